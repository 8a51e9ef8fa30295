"""Writing keys and values into the block cache and reading them back: the held values are exact."""
import math

import numpy as np
import pytest

from tests.kv_reference import held

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for the gpu tests")
    import paper_2609_33224_gb300 as P
    P.build()
    from paper_2609_33224_gb300 import kvcache
    return kvcache


def _dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


def _same(a, b):
    import torch
    assert a.shape == b.shape
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    assert torch.equal(torch.nan_to_num(a, 7.0), torch.nan_to_num(b, 7.0))


def _data(T, H, D, src, seed):
    """Rows over many magnitudes, with the special ones first, as slices of a wider tensor (a fused projection)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, 3, H, D, device="cuda", generator=g)
    x *= torch.exp2(torch.randint(-20, 12, (T, 3, H, 1), device="cuda", generator=g).float())
    x = x.to(_dtype(src))
    if T > 12:
        x[0] = 0
        x[1, :, :, 3] = math.inf
        x[2, :, :, 5] = math.nan
        x[3] = torch.finfo(_dtype(src)).max
        x[4] = -torch.finfo(_dtype(src)).tiny
        x[5] = 448.0
        x[6] = 449.0
        x[7, :, :, 0] = -math.inf
        x[8] = torch.arange(D, device="cuda") * 2.0 ** -9  # subnormal codes and ties
        x[8, :, :, 0] = 448
        x[9] = (17 + torch.arange(D, device="cuda") * 0.5)  # ties between codes
        x[10] = 2.0 ** -24
        x[11] = 2.0 ** -126 if src != "fp16" else 2.0 ** -14
    return x[:, 1], x[:, 2]


@pytest.mark.parametrize("fmt", ["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("src", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D,H", [(128, 8), (64, 3), (128, 1)])
@pytest.mark.parametrize("T", [1, 16, 37, 1003])
def test_what_was_written_comes_back(kv, fmt, src, D, H, T):
    import torch
    k, v = _data(T, H, D, src, T + H)
    blocks = T // 16 + 20
    slots = torch.randperm(blocks * 16, device="cuda")[:T].contiguous()
    with kv.KVCache(blocks, H, D, fmt=fmt) as c:
        c.write(k, v, slots)
        for out in (torch.float32, torch.bfloat16, torch.float16):
            gk, gv = c.read(slots, dtype=out)
            # one rounding to the cache, one to the type asked for (which bf16 does not need for fp8 rows)
            _same(gk, held(fmt, k).to(torch.float32).to(out))
            _same(gv, held(fmt, v).to(torch.float32).to(out))
        c.check()


def test_rows_that_stay(kv):
    """A write changes its slots alone; unwritten slots are zero; negative slots are skipped and read as zero."""
    import torch
    H, D = 4, 128
    for fmt in ("bf16", "fp8"):
        with kv.KVCache(64, H, D, fmt=fmt) as c:
            k, v = _data(1000, H, D, "bf16", 1)
            all_slots = torch.arange(1024, device="cuda")
            a = torch.randperm(1024, device="cuda")[:1000].contiguous()
            c.write(k, v, a)
            before = c.read(all_slots)
            free = torch.ones(1024, dtype=torch.bool, device="cuda")
            free[a] = False
            assert not before[0][free].any() and not before[1][free].any()
            k2, v2 = _data(40, H, D, "bf16", 2)
            b = a[100:140].clone()
            b[::3] = -1
            c.write(k2, v2, b)
            after = c.read(all_slots)
            for x, y, new in ((before[0], after[0], k2), (before[1], after[1], v2)):
                want = x.clone()
                want[b[b >= 0]] = held(fmt, new[b >= 0]).to(want.dtype)
                _same(y, want)
            got = c.read(b)
            assert not got[0][b < 0].any() and not got[1][b < 0].any()
            c.check()


def test_slots_outside_the_cache_are_reported(kv):
    import torch

    import paper_2609_33224_gb300 as P
    with kv.KVCache(4, 2, 64, fmt="fp8") as c:
        k, v = _data(5, 2, 64, "bf16", 3)
        slots = torch.tensor([0, 64, 5, 1 << 40, 63], device="cuda")
        c.write(k, v, slots)
        with pytest.raises(P.PSError, match="outside the cache"):
            c.check()
        c.check()  # reported once
        ok = torch.tensor([0, 5, 63], device="cuda")
        _same(c.read(ok)[0], held("fp8", k[[0, 2, 4]]).bfloat16())
        got = c.read(slots)
        assert not got[0][[1, 3]].any()
        torch.cuda.synchronize()
        with pytest.raises(P.PSError, match="outside the cache"):
            c.read(ok)
        c.read(ok)


def test_offsets_past_32_bits(kv):
    """The last blocks of a cache of more than 2^32 bytes."""
    import torch
    H, D, blocks = 8, 128, 150000
    with kv.KVCache(blocks, H, D, fmt="fp8") as c:
        k, v = _data(200, H, D, "bf16", 4)
        slots = torch.arange(blocks * 16 - 200, blocks * 16, device="cuda")
        low = (slots * 33024 // 16 % (1 << 32)) * 16 // 33024  # where a 32-bit offset would land
        c.write(k, v, slots)
        _same(c.read(slots)[1], held("fp8", v).bfloat16())
        assert not c.read(low.contiguous())[0].any()
        c.check()


def test_another_stream_and_empty_calls(kv):
    import torch
    s = torch.cuda.Stream()
    with kv.KVCache(8, 2, 128) as c:
        k, v = _data(100, 2, 128, "fp32", 5)
        slots = torch.randperm(128, device="cuda")[:100].contiguous()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            c.write(k, v, slots)
            got = c.read(slots, dtype=torch.float32)
        torch.cuda.current_stream().wait_stream(s)
        _same(got[0], held("bf16", k).float())
        e = torch.zeros(0, dtype=torch.int64, device="cuda")
        c.write(k[:0], v[:0], e)
        assert c.read(e)[0].shape == (0, 2, 128)
        c.check()


def test_refusals(kv):
    import torch
    with pytest.raises(ValueError):
        kv.KVCache(8, 2, 96)
    with pytest.raises(ValueError):
        kv.KVCache(8, 2, 128, fmt="int8")
    with pytest.raises(ValueError):
        kv.KVCache(0, 2, 128)
    import paper_2609_33224_gb300 as P
    with kv.KVCache(8, 2, 128) as c:
        x = torch.zeros(4, 2, 128, device="cuda", dtype=torch.bfloat16)
        s = torch.arange(4, device="cuda")
        for bad in (x[:3], x.cpu(), x.int(), x[:, :1], torch.zeros(4, 128, 2, device="cuda").transpose(1, 2)):
            with pytest.raises(ValueError):
                c.write(bad, x, s)
        for bad in (s.int(), s.cpu(), torch.arange(8, device="cuda")[::2], s[None]):
            with pytest.raises(ValueError):
                c.write(x, x, bad)
        odd = torch.zeros(4 * 2 * 128 + 1, device="cuda", dtype=torch.bfloat16)[1:].view(4, 2, 128)
        with pytest.raises(P.PSError, match="16-byte"):
            c.write(odd, x, s)
        wide = torch.zeros(4, 2, 132, device="cuda", dtype=torch.bfloat16)[:, :, :128]
        with pytest.raises(P.PSError, match="strides"):
            c.write(wide, x, s)
        with pytest.raises(P.PSError, match="one element type"):
            c.write(x, x.float(), s)
        c.check()
    with pytest.raises(ValueError, match="closed"):
        c.read(s)
