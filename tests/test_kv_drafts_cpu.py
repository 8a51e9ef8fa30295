"""Rotary frequencies, and the refusals of the calls on a draft, without a GPU."""
import ctypes
import math
import os
import subprocess
import types

import numpy as np
import pytest
import torch

import paper_2609_33224_gb300 as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def kv():
    P.build()
    from paper_2609_33224_gb300 import kvcache
    return kvcache


def test_frequencies(kv):
    f = [10000.0 ** (-2 * i / 64) for i in range(32)]
    near = lambda a, b: np.testing.assert_allclose(a, b, rtol=1e-14)  # noqa: E731
    near(kv.Rotary(64).frequencies, f)
    near(kv.Rotary(64, scaling="linear", factor=4).frequencies, [x / 4 for x in f])
    base = kv.Rotary(64, scaling="base", factor=4).frequencies
    assert base[0] == 1.0 and abs(base[-1] / (f[-1] / 4) - 1) < 1e-13 and (np.diff(base) < 0).all()
    got = kv.Rotary(64, scaling="rotations", factor=8, original=8192, low=1, high=4).frequencies
    for x, y in zip(f, got):
        turns = 8192 * x / (2 * math.pi)
        w = min(max((turns - 1) / 3, 0), 1)
        assert abs(y / (w * x + (1 - w) * x / 8) - 1) < 1e-14
    got = kv.Rotary(64, scaling="pairs", factor=8, original=4096, low=1, high=32).frequencies
    # the pair that makes r rotations in 4096 positions: 4096 / (2 pi 10000^(2 i / 64)) = r
    at = lambda r: 64 * math.log(4096 / (r * 2 * math.pi)) / (2 * math.log(10000))  # noqa: E731
    lo, hi = math.floor(at(32)), math.ceil(at(1))
    assert 0 < lo < hi < 32
    for i, (x, y) in enumerate(zip(f, got)):
        w = 1 - min(max((i - lo) / (hi - lo), 0), 1)
        assert abs(y / (w * x + (1 - w) * x / 8) - 1) < 1e-14
    near(kv.Rotary(16, frequencies=[0, 1, -2, 3, 1e9, 5, 6, 7]).frequencies, [0, 1, -2, 3, 1e9, 5, 6, 7])


def test_rotary_refusals(kv):
    for bad in (dict(dims=0), dict(dims=24), dict(dims=144), dict(dims=64, base=0.0), dict(dims=64, factor=-1.0, scaling="linear"),
                dict(dims=64, scaling="other"), dict(dims=64, scaling="rotations"), dict(dims=64, scaling="pairs", original=0),
                dict(dims=64, scaling="rotations", original=8192, low=4.0, high=4.0), dict(dims=64, frequencies=[1.0] * 31),
                dict(dims=16, frequencies=[math.nan] * 8), dict(dims=16, frequencies=[1.0] * 8, scaling="linear"),
                dict(dims=64, magnitude=math.inf), dict(dims=64, scaling="pairs", original=8192, base=1.0)):
        with pytest.raises(ValueError):
            kv.Rotary(**bad)
    r = kv.Rotary(64)
    with pytest.raises(ValueError):
        r.frequencies[0] = 2.0


def test_struct_layout_matches_c(kv, tmp_path):
    src = tmp_path / "layout.c"
    src.write_text("""
#include <stdio.h>
#include <stddef.h>
#include "packserve_kv.h"
int main(void) {
  printf("%zu %zu %zu %zu\\n", sizeof(ps_kv_rotary), offsetof(ps_kv_rotary, interleaved), offsetof(ps_kv_rotary, magnitude),
         offsetof(ps_kv_rotary, frequency));
  return 0;
}
""")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    R = P.PsKvRotary
    assert got == [ctypes.sizeof(R), R.interleaved.offset, R.magnitude.offset, R.frequency.offset]


def test_null_objects_are_refused(kv):
    L = P.lib()
    assert L.ps_kv_write_rotated(None, None, None, None, None, 0, None, None, None, 0, None) == 1
    assert L.ps_kv_move(None, None, None, 0, None, 0, None) == 1
    assert L.ps_kv_move_workspace(None, 0, None) == 1
    assert L.ps_kv_copy_blocks(None, None, None, None, 0, None) == 1
    assert L.ps_kv_tree_mask(None, None, 0, None, 0, None, None, 0, 0, None, None) == 1
    assert L.ps_kv_plan_set_masked(None, 0, None, 0, None, 0) == 1
    assert L.ps_kv_attend_masked(None, None, None, None, None, 1.0, None, 0, 0, None, 0, None) == 1


@pytest.fixture
def cache(kv, monkeypatch):
    """A cache on the host whose entry points record that they were reached."""
    c = kv.KVCache.__new__(kv.KVCache)
    c._h, c.device, c._device = ctypes.c_void_p(1), -1, torch.device("cpu")
    c.num_blocks, c.kv_heads, c.head_dim, c.fmt, c.dtype = 4, 2, 64, "bf16", torch.bfloat16
    c._args = (ctypes.c_char * (4 * kv._ROWS.size))()
    c._arg0 = ctypes.addressof(c._args)
    c._arg1, c._arg2, c._arg3 = (c._arg0 + i * kv._ROWS.size for i in (1, 2, 3))
    c._spaces, c.reached = {}, []
    monkeypatch.setattr(kv, "_stream", lambda d: 0)
    c._lib = types.SimpleNamespace(**{n: (lambda *a, n=n: c.reached.append(n) or 0) for n in (
        "ps_kv_write_rotated", "ps_kv_move", "ps_kv_copy_blocks", "ps_kv_tree_mask", "ps_kv_attend_masked", "ps_kv_attend")})
    yield c
    c._h = None


def test_calls_refuse_wrong_arguments(kv, cache):
    x, s = torch.zeros(5, 2, 64).bfloat16(), torch.arange(5)
    q, r = torch.zeros(5, 6, 64).bfloat16(), kv.Rotary(64)
    assert cache.write_rotated(x, x, s, s, r, q=q).shape == q.shape
    assert cache.write_rotated(x, x, s, s, r) is None
    cache.move(s, s)
    cache.copy_blocks(s, s)
    parents = torch.tensor([[-1, 0, 0]], dtype=torch.int32)
    assert [t.shape for t in cache.tree_mask(parents)] == [(3, 1), (3,)]
    assert len(cache.reached) == 5
    for args, kw in (((x, x, s, s[:4], r), {}), ((x, x, s, s.int(), r), {}), ((x, x, s, s, kv.Rotary(128)), {}),
                     ((x[:4], x, s, s, r), {}), ((x, x, s, s, r), dict(out=q)), ((x, x, s, s, r), dict(q=q[:, 0])),
                     ((x, x, s, s, r), dict(q=q[:, :0])), ((x, x, s, s, r), dict(q=q, out=q.float())),
                     ((x, x, s, s, r), dict(q=q, out=q[:, :5])), ((x, x, s[::1][None], s, r), {})):
        with pytest.raises(ValueError):
            cache.write_rotated(*args, **kw)
    for call in (cache.move, cache.copy_blocks):
        for a, b in ((s, s[:4]), (s.int(), s), (s, torch.arange(10)[::2]), (s[None], s)):
            with pytest.raises(ValueError):
                call(a, b)
    flat = parents[0]
    for args, kw in (((flat,), {}), ((parents.long(),), {}), ((parents, torch.tensor([0, 3])), {}), ((flat, torch.tensor([0, 3])), {}),
                     ((flat, torch.tensor([0, 3]), 9000), {}), ((parents,), dict(start=torch.zeros(2).long())),
                     ((flat, torch.zeros(0).long(), 4), {}), ((torch.zeros(4, 6).int()[:, ::2],), {})):
        with pytest.raises(ValueError):
            cache.tree_mask(*args, **kw)
    plan = types.SimpleNamespace(_open=lambda: 1, num_queries=5, q_heads=6, masked=40, workspace_bytes=0)
    ok = torch.zeros(5, 2, dtype=torch.int32)
    cache.attend(q, plan, mask=ok)
    for bad in (None, ok[:4], ok[:, :1], ok.long(), ok[0], torch.zeros(2, 5, dtype=torch.int32).T):
        with pytest.raises(ValueError):
            cache.attend(q, plan, mask=bad)
    assert cache.reached[5:] == ["ps_kv_attend_masked"]


def test_spans_of_drafts(kv):
    tables = [[1, 2, 3, 4, 5, 6], [1, 2, 3, 4, 9, 8]]
    for masked, want in ((True, [2, 2]), (False, [1, 1]), ([True, False], [2, 1])):
        order, spans, _ = kv.shared_spans(tables, [90, 92], [20, 3], masked=masked)
        own = {int(s["first_query"]): int(s["causal"]) for s in spans if s["causal"]}
        first = {i: sum([20, 3][j] for j in order[:x]) for x, i in enumerate(order)}
        assert [own[first[i]] for i in (0, 1)] == want
    with pytest.raises(ValueError):
        kv.shared_spans(tables, [90, 92], [20, 3], masked=[True])


def test_a_rotary_can_be_copied(kv):
    import copy
    r = copy.deepcopy(kv.Rotary(32, interleaved=True, magnitude=1.5, scaling="linear", factor=2.0))
    assert (r._c.dims, r._c.interleaved, r._c.magnitude) == (32, 1, 1.5)
    np.testing.assert_array_equal(list(r._c.frequency)[:16], r.frequencies)
