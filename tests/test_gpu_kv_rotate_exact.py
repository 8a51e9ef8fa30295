"""Rotated writes where the last bits count: frequencies of either sign at far positions, fp8 rows whose turned maximum lies at
a border of the scales."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv_rotate import check, turned
from tests.test_gpu_kv_store import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
def test_negative_frequencies(kv, interleaved):  # noqa: F811
    """A negative frequency turns as its magnitude does at the negative position, in every bit, and as far as the latter is
    right; small ones at far positions too."""
    T, D = 200, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, 8, D, device="cuda", generator=g)
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    f = np.concatenate([10.0 ** -np.linspace(6, 12, 24), 10.0 ** -np.linspace(13, 18, 8)])
    positions = torch.randint(-(1 << 40), 1 << 40, (T,), device="cuda", generator=g)
    slots = torch.arange(T, device="cuda")
    with kv.KVCache(T // 16 + 1, 2, D, fmt="fp16") as c:
        rotary = kv.Rotary(D, interleaved=interleaved, frequencies=-f)
        got = c.write_rotated(k, v, slots, positions, rotary, q=q)
        held = c.read(slots)[0]
        check(c, rotary, q, k, v, slots, positions, got)
        again = c.write_rotated(k, v, slots, -positions, kv.Rotary(D, interleaved=interleaved, frequencies=f), q=q)
        assert torch.equal(got, again) and torch.equal(held, c.read(slots)[0])
        c.check()


@pytest.mark.parametrize("T,Hq,Hkv", [(3, 0, 6), (3, 5, 6), (37, 9, 3), (6000, 2, 5)])
@pytest.mark.parametrize("D,dims", [(128, 128), (128, 48), (64, 64), (64, 16)])
@pytest.mark.parametrize("interleaved,magnitude", [(False, 1.0), (True, 1.0), (False, 1.375), (True, 0.8125)])
def test_rows_at_a_border_of_the_scales(kv, T, Hq, Hkv, D, dims, interleaved, magnitude):  # noqa: F811
    """Every key's maximum, turned by any angle, lies within 2^-20 of 448 times a power of two: its row is turned to 2^-28 of
    what is mixed.  Its scale is the exact row's, but where the maximum lies within 2^-26 of the border, and each code is the
    exact element's, but where that lies within 2^-26 of what is mixed from the middle of two.  A few tokens, whose rows
    several warps share, and many; with queries and without."""
    g = torch.Generator(device="cuda").manual_seed(T + dims)
    rotary = kv.Rotary(dims, interleaved=interleaved, magnitude=magnitude)
    x = torch.randn(T, Hq + 2 * Hkv, D, device="cuda", generator=g)
    positions = torch.randint(0, 1 << 17, (T,), device="cuda", generator=g)
    top = turned(x, positions, rotary)[0].abs().amax(-1, keepdim=True)
    near = 1 + torch.randint(-3, 4, top.shape, device="cuda", generator=g) * 2.0 ** -23
    x = (x.double() * (448.0 * torch.exp2(torch.randint(-12, 5, top.shape, device="cuda", generator=g).double()) * near / top)).float()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    want, mag = turned(k, positions, rotary)
    top = want.abs().amax(-1, keepdim=True)
    # a float's rounding moves an element by 2^-24 of itself, the maximum by less than twice that of it (two elements are mixed)
    border = 448.0 * torch.exp2(torch.round(torch.log2(top / 448.0)))
    assert ((top / border - 1).abs() < 2.0 ** -20).all()
    slots = torch.randperm(T + 16, device="cuda", generator=g)[:T].contiguous()
    with kv.KVCache(T // 16 + 2, Hkv, D, fmt="fp8") as c:
        c.write_rotated(k, v, slots, positions, rotary, q=q if Hq else None)
        got = c.read(slots, dtype=torch.float32)[0].double()
        c.check()
    e, least = (torch.ceil(torch.log2(y / 448.0)) for y in (top * (1 + 2.0 ** -26), top * (1 - 2.0 ** -26)))
    unit = torch.exp2(e)

    def code(y):
        step = unit * torch.exp2(torch.floor(torch.log2((y / unit).abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(y / step) * step

    low, high = (code(want + s * mag * 2.0 ** -26) for s in (-1, 1))
    clear = (e == least).expand_as(want) & (low == high)
    assert clear.double().mean() > 0.5
    assert torch.equal(got[clear], low[clear])
