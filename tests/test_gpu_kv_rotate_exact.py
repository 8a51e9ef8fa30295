"""Rotated writes where angles or scales are near a border: frequencies of either sign at far positions."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv_rotate import check
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
