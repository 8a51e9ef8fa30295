"""fp8 caches and queries whose elements span more than fp16 does, in attention of few rows."""
import math

import pytest
import torch

from tests import kv_reference as ref
from tests.test_gpu_kv_attend import Batch, kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,g", [(128, 8), (64, 4)])
@pytest.mark.parametrize("big", [2.0 ** 20, 2.0 ** 36, 2.0 ** 60, 2.0 ** 122])
def test_a_large_element_that_no_key_has(kv, D, g, big):
    """One element of the queries is far larger than the others; the keys' are zero there."""
    T = 4
    b = Batch(kv, "fp8", 2, g, D, [(0, T, 300, 0)] + [(i, 1, 20 + 9 * i, 1) for i in range(T)], T, seed=61)
    b.q[1:, :, 5] = big
    k = b.k.clone()
    k[:, :, 5] = torch.where(torch.isnan(k[:, :, 5]), k[:, :, 5], 0.0)
    b.cache.write(k, b.v, torch.arange(k.shape[0], device="cuda"))
    b.k = k
    b.check(*b.run())


@pytest.mark.parametrize("up", [-100, 90, 100, 118])
def test_large_queries_on_small_keys(kv, up):
    """Scores of common size from queries and keys of extreme magnitudes."""
    T = 3
    b = Batch(kv, "fp8", 1, 8, 128, [(0, T, 200, 0), (0, T, 33, 1)], T, seed=67)
    down = min(max(up, -100), 95)
    b.q = (b.q.double() * 2.0 ** up).to(b.q.dtype)
    b.k = (b.k.double() * 2.0 ** -down).to(b.k.dtype)
    b.cache.write(b.k, b.v, torch.arange(b.k.shape[0], device="cuda"))
    scale = 128 ** -0.5 * 2.0 ** (down - up)
    b.check(*b.run(scale=scale), scale=scale)


def test_a_key_with_a_nan_beside_a_large_query(kv):
    """In the wide form too a masked key's NaN stays with the queries that see it."""
    n = 30
    b = Batch(kv, "fp8", 1, 8, 64, [(0, n, n + 4, 1)], n, seed=71)
    b.q[:, :, 5] = 2.0 ** 50
    k = b.k.clone()
    k[:, :, 5] = torch.where(torch.isnan(k[:, :, 5]), k[:, :, 5], 0.0)
    clean = k.clone()
    k[b.slots_of[0][4 + 20], :, 9] = math.nan
    b.cache.write(k, b.v, torch.arange(k.shape[0], device="cuda"))
    out, _ = b.run()
    assert torch.isnan(out[20:]).all() and torch.isfinite(out[:20]).all()
    want, _, A, mag, cnt = ref.attend(b.q, ref.held("fp8", clean), ref.held("fp8", b.v), b.spans, b.slots_of, 64 ** -0.5)
    tol, _ = ref.bounds("fp8", 64, want, A, mag, cnt, 0.0)
    assert ((out[:20].double() - want[:20]).abs() <= tol[:20]).all()
