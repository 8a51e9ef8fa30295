"""Rotated writes against 64 bits: queries and keys turned by their positions, what the cache then holds."""
import math

import numpy as np
import pytest
import torch

from tests import kv_reference as ref
from tests.test_gpu_kv_store import _dtype, _same, kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


def turned(x, positions, rotary):
    """Rows [T, heads, D] turned in 64 bits, and elementwise the magnitudes |a| + |b| of what was mixed."""
    R = rotary.dims
    f = torch.from_numpy(rotary.frequencies.copy()).to(x.device)
    angle = positions.double()[:, None] * f
    c, s = (angle.cos() * rotary.magnitude)[:, None], (angle.sin() * rotary.magnitude)[:, None]
    x = x.double()
    lo, hi = (slice(0, R, 2), slice(1, R, 2)) if rotary.interleaved else (slice(0, R // 2), slice(R // 2, R))
    y, mag = x.clone(), x.abs()
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    both = (a.abs() + b.abs()) * abs(rotary.magnitude)
    mag[..., lo], mag[..., hi] = both, both
    return y, mag


def bound(want, mag, positions, rotary, fmt, quantised=False):
    """Off by half a step of the result's type (fp8: e4m3's 2^-4, or half of its smallest step 2^-9 times the row's scale,
    which is below 2 max / 448), and by the arithmetic before it: an angle is off by 2^-25 of a turn (2^-22 radians), or
    by p f 2^-51 where that is more (p f is as inexact here); sine and cosine, their product with the magnitude, and two
    products and a sum add less than 2^-21 of what is mixed."""
    far = (positions.double().abs()[:, None, None] * float(np.abs(rotary.frequencies).max())) * 2.0 ** -50
    slack = mag * (2.0 ** -20 + far)
    u = 2.0 ** -4 if quantised else 2.0 ** -11 if fmt == "fp16" else 2.0 ** -8
    tol = u * want.abs() * (1 + 2 * u) + slack * (1 + 2 * u)
    if quantised:
        tol = tol + 2.0 ** -10 * 2 / 448 * (want.abs() + slack).amax(-1, keepdim=True)
    elif fmt == "fp16":
        tol = tol + 2.0 ** -25
    return tol


def check(cache, rotary, q, k, v, slots, positions, got_q):
    gk, gv = cache.read(slots, dtype=torch.float32)
    _same(gv, ref.held(cache.fmt, v).float())
    want, mag = turned(k, positions, rotary)
    assert ((gk.double() - want).abs() <= bound(want, mag, positions, rotary, cache.fmt, cache.fmt == "fp8")).all()
    if q is not None:
        want, mag = turned(q, positions, rotary)
        assert got_q.dtype == cache.dtype
        assert ((got_q.double() - want).abs() <= bound(want, mag, positions, rotary, cache.fmt)).all()
    cache.check()


def _data(T, Hq, Hkv, D, src, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, Hq + 2 * Hkv, D, device="cuda", generator=g)
    x *= torch.exp2(torch.randint(-6, 7, (T, Hq + 2 * Hkv, 1), device="cuda", generator=g).float())
    x = x.to(_dtype(src))
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]  # slices of a fused projection


@pytest.mark.parametrize("fmt", ["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("src", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D,dims,interleaved", [(128, 128, False), (128, 128, True), (64, 64, False), (64, 32, True),
                                                (128, 16, False), (128, 48, False), (64, 16, True), (128, 112, True)])
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 64, 8), (37, 5, 1), (300, 7, 7)])
def test_against_64_bits(kv, fmt, src, D, dims, interleaved, T, Hq, Hkv):
    q, k, v = _data(T, Hq, Hkv, D, src, T + dims)
    rotary = kv.Rotary(dims, base=500000.0, interleaved=interleaved, scaling="rotations", factor=8.0, original=8192,
                       magnitude=1.25)
    positions = torch.randint(0, 131072, (T,), device="cuda")
    blocks = T // 16 + 9
    slots = torch.randperm(blocks * 16, device="cuda")[:T].contiguous()
    with kv.KVCache(blocks, Hkv, D, fmt=fmt) as c:
        got = c.write_rotated(k, v, slots, positions, rotary, q=q)
        check(c, rotary, q, k, v, slots, positions, got)


@pytest.mark.parametrize("T", [4000, 6001])
def test_many_tokens(kv, T):
    """Tokens whose rows several warps share, and a warp with several tokens."""
    q, k, v = _data(T, 12, 4, 128, "bf16", 3)
    rotary = kv.Rotary(128)
    positions = torch.arange(T, device="cuda") + 7
    slots = torch.randperm(T + 100, device="cuda")[:T].contiguous()
    with kv.KVCache((T + 100) // 16 + 1, 4, 128, fmt="fp8") as c:
        check(c, rotary, q, k, v, slots, positions, c.write_rotated(k, v, slots, positions, rotary, q=q))


def test_positions_of_any_size(kv):
    """Far and negative positions; position 0 changes nothing."""
    at = [0, 1, -1, 2 ** 31 - 1, -(2 ** 31), 10 ** 7 + 1, -12345, 2 ** 33 + 5, 0]
    T = len(at)
    q, k, v = _data(T, 3, 2, 64, "bf16", 4)
    positions = torch.tensor(at, device="cuda")
    slots = torch.arange(T, device="cuda")
    for rotary in (kv.Rotary(64), kv.Rotary(64, interleaved=True, frequencies=np.linspace(-7.0, 9.0, 32))):
        with kv.KVCache(2, 2, 64) as c:
            got = c.write_rotated(k, v, slots, positions, rotary, q=q)
            check(c, rotary, q, k, v, slots, positions, got)
            assert torch.equal(got[positions == 0], q[positions == 0])
            assert torch.equal(c.read(slots)[0][positions == 0], k[positions == 0])


def test_turning_back(kv):
    """A rotation and one by the negative position give the row again."""
    T = 50
    q, k, v = _data(T, 4, 2, 128, "fp32", 6)
    positions = torch.randint(0, 10 ** 6, (T,), device="cuda")
    slots = torch.arange(T, device="cuda")
    rotary = kv.Rotary(96, interleaved=True)
    with kv.KVCache(4, 2, 128) as c:
        there = c.write_rotated(k, v, slots, positions, rotary, q=q)
        kk, vv = c.read(slots)
        back = c.write_rotated(kk, vv, slots, -positions, rotary, q=there)
        for x, y in ((back, q), (c.read(slots)[0], k)):
            # two roundings of either element of a pair, by 2^-8 of it each, turned
            _, mag = turned(x, positions * 0, rotary)
            assert ((x.double() - y.double()).abs() <= 2.0 ** -6 * mag).all()


def test_in_place_strides_and_keys_alone(kv):
    T, Hq, Hkv, D = 70, 6, 2, 128
    rotary = kv.Rotary(D)
    positions = torch.randint(0, 5000, (T,), device="cuda")
    slots = torch.randperm(128, device="cuda")[:T].contiguous()
    q, k, v = _data(T, Hq, Hkv, D, "bf16", 7)
    with kv.KVCache(8, Hkv, D) as c:
        want = c.write_rotated(k, v, slots, positions, rotary, q=q)
        held = c.read(slots)
        assert c.write_rotated(k, v, slots, positions, rotary) is None
        for x, y in zip(c.read(slots), held):
            assert torch.equal(x, y)
        # heads first, a wider tensor around it
        wide = torch.full((Hq + 1, T + 2, D + 8), 9.0, device="cuda", dtype=torch.bfloat16)
        out = wide[:Hq, 1:T + 1, :D].transpose(0, 1)
        assert c.write_rotated(k, v, slots, positions, rotary, q=q, out=out) is out
        assert torch.equal(out, want)
        assert (wide[Hq:] == 9).all() and (wide[:, 0] == 9).all() and (wide[:, T + 1] == 9).all() and (wide[..., D:] == 9).all()
        # one key and value for all heads
        one = k[:, :1].expand(T, Hkv, D)
        c.write_rotated(one, one, slots, positions, rotary)
        check(c, rotary, None, one, one, slots, positions, None)
        assert c.write_rotated(k, v, slots, positions, rotary, q=q, out=q) is q
        assert torch.equal(q, want)
        for x, y in zip(c.read(slots), held):
            assert torch.equal(x, y)
        c.check()


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_skipped_tokens_and_values_that_are_not_finite(kv, fmt):
    import paper_2609_33224_gb300 as P
    T = 40
    q, k, v = (x.clone() for x in _data(T, 4, 2, 64, "bf16", 8))
    k[3, 0, 5] = math.nan
    k[4, 1, 60] = math.inf  # not turned
    q[5, 2, 1] = math.inf
    rotary = kv.Rotary(32)
    positions = torch.arange(T, device="cuda") + 1
    slots = torch.arange(T, device="cuda")
    slots[10:20] = -1
    with kv.KVCache(4, 2, 64, fmt=fmt) as c:
        got = c.write_rotated(k, v, slots, positions, rotary, q=q)
        c.check()
        held = c.read(torch.arange(T, device="cuda"))
        assert not held[0][10:20].any() and not held[1][10:20].any()
        want, _ = turned(q, positions, rotary)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
        bad = ~torch.isfinite(held[0])
        if fmt == "fp8":  # a row with a NaN is one whole, an infinity a large number
            assert bad[3, 0].all() and bad.sum() == 64
        else:
            assert bad[3, 0, [5, 21]].all() and torch.isposinf(held[0][4, 1, 60]) and bad.sum() == 3
        slots[7] = 64
        assert torch.equal(c.write_rotated(k, v, slots, positions, rotary, q=q)[6:], got[6:])
        with pytest.raises(P.PSError, match="outside the cache"):
            c.check()
        e = torch.zeros(0, dtype=torch.int64, device="cuda")
        assert c.write_rotated(k[:0], v[:0], e, e, rotary, q=q[:0]).shape == (0, 4, 64)
        c.check()


def test_captured_and_on_another_stream(kv):
    T = 33
    rotary = kv.Rotary(128, scaling="linear", factor=4.0)
    q, k, v = _data(T, 8, 2, 128, "fp32", 9)
    q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    positions = torch.randint(0, 5000, (T,), device="cuda")
    slots = torch.arange(T, device="cuda")
    c = kv.KVCache(3, 2, 128, fmt="fp8")
    out = torch.empty(T, 8, 128, device="cuda", dtype=torch.bfloat16)
    ko, vo = torch.empty(T, 2, 128, device="cuda"), torch.empty(T, 2, 128, device="cuda")
    c.write_rotated(k, v, slots, positions, rotary, q=q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.write_rotated(k, v, slots, positions, rotary, q=q, out=out)
        c.read(slots, k=ko, v=vo)
    turn, rotary = rotary, None  # the graph needs neither the rotary nor the cache
    with kv.KVCache(3, 2, 128, fmt="fp8") as d:
        s = torch.cuda.Stream()
        c.close()
        for i in range(3):
            q.copy_(torch.randn_like(q))
            k.copy_(torch.randn_like(k))
            positions += 1000 * i
            out.zero_()
            graph.replay()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                want = d.write_rotated(k, v, slots, positions, turn, q=q)
                wk, wv = d.read(slots, dtype=torch.float32)
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(ko, wk) and torch.equal(vo, wv)
        d.check()


def test_refusals(kv):
    import paper_2609_33224_gb300 as P
    with kv.KVCache(4, 2, 64) as c:
        q, k, v = _data(5, 4, 2, 64, "bf16", 1)
        s = torch.arange(5, device="cuda")
        r = kv.Rotary(64)
        with pytest.raises(ValueError, match="more dims"):
            c.write_rotated(k, v, s, s, kv.Rotary(128))
        for bad in (s[:4], s.int(), s.cpu()):
            with pytest.raises(ValueError):
                c.write_rotated(k, v, s, bad, r)
        with pytest.raises(ValueError, match="without q"):
            c.write_rotated(k, v, s, s, r, out=q)
        for bad in (q[:4], q[:, 0], q[:, :0], q.cpu()):
            with pytest.raises(ValueError):
                c.write_rotated(k, v, s, s, r, q=bad)
        with pytest.raises(ValueError, match="dtype"):
            c.write_rotated(k, v, s, s, r, q=q, out=torch.empty(5, 4, 64, device="cuda"))
        with pytest.raises(P.PSError, match="one element type"):
            c.write_rotated(k, v, s, s, r, q=q.float())
        with pytest.raises(P.PSError, match="overlap"):
            c.write_rotated(k, v, s, s, r, q=q, out=torch.empty(5, 1, 64, device="cuda", dtype=torch.bfloat16).expand(5, 4, 64))
        c.check()


@pytest.mark.parametrize("fmt", ["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("interleaved,magnitude", [(False, 1.0), (True, 1.0), (False, 1.375)])
def test_keys_are_rounded_once(kv, fmt, interleaved, magnitude):
    """What the cache holds is the exact key's rounding, but where that lies within 2^-22 of what is mixed from a border: sine
    and cosine are off by 2^-25 (with the magnitude 2^-24), a product and the sum of it and the other by as much again.
    An fp8 row's scale is the exact row's, but where its maximum lies within 2^-26 of a border."""
    T, H, D = 20000, 4, 128
    _, k, v = _data(T, 1, H, D, "fp32" if fmt == "fp16" else "bf16", 11)
    rotary = kv.Rotary(D, interleaved=interleaved, magnitude=magnitude)
    positions = torch.randint(0, 1 << 17, (T,), device="cuda")
    if fmt == "fp8":  # rows whose largest element, unturned, lies at a border of the scales or just beside it
        positions[::2] = 0
        k = k.float()
        k[::2] *= (448.0 / magnitude / k[::2].abs().amax(-1, keepdim=True)) * (1 + torch.randint(-3, 4, (T // 2, H, 1), device="cuda") * 2.0 ** -23)
        v = v.float()
    slots = torch.randperm(T + 8, device="cuda")[:T].contiguous()
    with kv.KVCache(T // 16 + 1, H, D, fmt=fmt) as c:
        c.write_rotated(k, v, slots, positions, rotary)
        got = c.read(slots, dtype=torch.float32)[0].double()
        c.check()
    want, mag = turned(k, positions, rotary)
    if fmt == "fp8":
        top = want.abs().amax(-1, keepdim=True)
        e, least = (torch.ceil(torch.log2(x / 448.0)) for x in (top * (1 + 2.0 ** -26), top * (1 - 2.0 ** -26)))
        same = (e == least).expand_as(want)
        unit = torch.exp2(e)
        step = lambda x: unit * torch.exp2(torch.floor(torch.log2((x / unit).abs().clamp(min=2.0 ** -6))) - 3)  # noqa: E731
    else:
        p, smallest = (8, -126) if fmt == "bf16" else (11, -14)  # significant bits, the smallest normal exponent
        same = torch.ones_like(want, dtype=torch.bool)
        step = lambda x: torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** smallest))) - (p - 1))  # noqa: E731
    low, high = (torch.round(x / step(x)) * step(x) for x in (want - mag * 2.0 ** -22, want + mag * 2.0 ** -22))
    clear = same & (low == high)
    assert clear.double().mean() > (0.5 if fmt == "fp8" else 0.99)
    assert torch.equal(got[clear], low[clear])
