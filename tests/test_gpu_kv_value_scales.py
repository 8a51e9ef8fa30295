"""fp8 values whose scales lie far apart, in attention of few rows: what a query does not see, or hardly weighs, must
not cost the precision of what it does."""
import math

import pytest
import torch

from tests import kv_reference as ref
from tests.test_gpu_kv_attend import Batch, kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


def _check(b, k, v, out, lse, skip=None):
    """Against 64 bits, elementwise.  Beside the roundings of kv_reference.bounds, probabilities in fp16, taken relative
    to value scales that lie within 2^11 of each other, lose at most 2^-25 of 2^5 of the largest scale: 2^-20 of the key's
    own value, where the largest probability counts 1 or more.  Keys further above the smallest scale are held
    without such a floor.  skip[t, h, d]: elements that are not compared."""
    scale = b.D ** -0.5
    hk, hv = ref.held("fp8", k), ref.held("fp8", v)
    want, wl, A, mag, cnt = ref.attend(b.q, hk, hv, b.spans, b.slots_of, scale)
    tol, tl = ref.bounds("fp8", b.D, want, A, mag, cnt, 0.0)
    amax = hv.abs().amax(-1)
    seen = torch.cat([s for s in b.slots_of]).unique()
    least = amax[seen][amax[seen] > 0].min()
    plain = torch.where((amax <= 2.0 ** 11 * least)[..., None], hv.abs(), 0.0)
    # sum_j |v_j| / sum_j e^(z_j - max): a uniform sum over the seen keys times e^(max - lse)
    g = b.Hq // k.shape[1]
    for t in range(b.T):
        sel = [sl[:max(0, ln - n + (t - f) + 1) if c else ln] for (f, n, ln, c, *_), sl in zip(b.spans, b.slots_of) if f <= t < f + n]
        sel = torch.cat(sel) if sel else torch.zeros(0, dtype=torch.int64, device="cuda")
        if sel.numel():
            z = torch.einsum("hd,lhd->hl", b.q[t].double(), hk[sel].repeat_interleave(g, 1)) * scale
            tol[t] += 2.0 ** -20 * plain[sel].sum(0).repeat_interleave(g, 0) * torch.exp(z.amax(-1) - wl[t])[:, None]
    ok = (out.double() - want).abs() <= tol
    if skip is not None:
        ok |= skip
    assert ok.all(), ((out.double() - want).abs() / tol)[~ok].max().item()
    seen = cnt > 0
    assert ((lse.double() - wl).abs() <= tl)[seen].all()


def _put(b, k, v):
    b.cache.write(k, v, torch.arange(k.shape[0], device="cuda"))


@pytest.mark.parametrize("D,g", [(128, 8), (64, 4), (128, 1)])
@pytest.mark.parametrize("big", [2.0 ** 14, 2.0 ** 30, 2.0 ** 100, math.inf])
def test_a_large_value_that_earlier_queries_do_not_see(kv, D, g, big):
    """Causal: a token's value row is far larger than all others (or one of its elements infinite, held as the largest
    number); the queries before it do not see it."""
    n = 40
    b = Batch(kv, "fp8", 2, g, D, [(0, n, n + 9, 1)], n, seed=41)
    k, v = b.k.clone(), b.v.clone()
    at = b.slots_of[0][9 + 20]
    skip = None
    if math.isinf(big):
        v[at, :, 3] = big
        skip = torch.zeros(n, b.Hq, D, dtype=torch.bool, device="cuda")
        skip[20:, :, 3] = True  # sums of the largest float may overflow
    else:
        v[at] *= big
    _put(b, k, v)
    out, lse = b.run()
    _check(b, k, v, out, lse, skip)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("big", [2.0 ** 12, 2.0 ** 30, 2.0 ** 60])
def test_a_large_value_of_no_weight(kv, D, big):
    """Rows of large values whose scores are very low: they lie before, between and behind the others."""
    T = 3
    b = Batch(kv, "fp8", 2, 4, D, [(i, 1, 700, 0) for i in range(T)], T, seed=43)
    b.q = b.q.abs() + 0.5
    k, v = b.k.clone(), b.v.clone()
    for sl, at in zip(b.slots_of, ([0, 1, 300], [305], [690, 699])):
        k[sl[at]] = -6.0 * (64 / D) ** 0.5  # scores below -50
        v[sl[at]] *= big
    _put(b, k, v)
    out, lse = b.run()
    _check(b, k, v, out, lse)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("order", ["up", "down", "random", "small", "far"])
def test_scales_that_differ(kv, D, order):
    """Value scales that grow, fall or jump along the keys, small ones and rows of zeros among them."""
    T, n = 5, 400
    b = Batch(kv, "fp8", 1, 4, D, [(0, T, n, 0), (1, 3, 45, 1)], T, seed=47)
    k, v = b.k.clone(), b.v.clone()
    gen = torch.Generator(device="cuda").manual_seed(1)
    sl = b.slots_of[0]
    i = torch.arange(n, device="cuda")
    e = {"up": i // 16 * 3 - 40, "down": 30 - i // 16 * 3,
         "random": torch.randint(-30, 31, (n,), device="cuda", generator=gen),
         "small": torch.where(i % 50 == 7, -15, 0), "far": torch.where(i < 100, -90, torch.where(i < 200, 90, 0))}[order]
    v[sl] = (v[sl].float() * torch.exp2(e.float())[:, None, None]).to(v.dtype)
    v[sl[5::37]] = 0
    _put(b, k, v)
    out, lse = b.run()
    _check(b, k, v, out, lse)


def test_a_marked_row_beside_a_large_one(kv):
    """A value row with a NaN and one of large values: queries that see the NaN get it, the others neither."""
    n = 33
    b = Batch(kv, "fp8", 1, 8, 128, [(0, n, 100, 0), (0, n, n, 1)], n, seed=53)
    k, v = b.k.clone(), b.v.clone()
    sl = b.slots_of[1]
    v[sl[20]] *= 2.0 ** 40
    v[sl[22], :, 5] = math.nan
    v[sl[24]] *= 2.0 ** 40
    _put(b, k, v)
    out, lse = b.run()
    assert torch.isnan(out[22:]).all() and torch.isfinite(out[:22]).all()
    v2 = v.nan_to_num(0.0)
    skip = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    skip[22:] = True
    _check(b, k, v2, out, lse, skip)
