"""Joining the parts of queries with many heads on one key/value head, whose rows lie in several tiles."""
import pytest
import torch

from tests import kv_reference as ref
from tests.test_gpu_kv_attend import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("g,T,mixed", [(128, 20, False), (100, 9, True), (33, 30, True), (65535, 17, False), (65535, 17, True)])
def test_every_row_is_joined(kv, g, T, mixed):
    """A shared span and a causal span per query: every row has two parts.  mixed: one query without a key, whose heads
    need no cut."""
    D, shared, own = 64, 64, 40
    gen = torch.Generator(device="cuda").manual_seed(g)
    n = T - 1 if mixed else T
    blocks = 4 + 3 * T
    k, v = (torch.randn(blocks * 16, 1, D, device="cuda", generator=gen).bfloat16() for _ in range(2))
    q = (torch.randn(T, g, D, device="cuda", generator=gen) * 0.7).bfloat16()
    spans = [(0, n, shared, 0, 0)] + [(i, 1, own, 1, 4 + 3 * i) for i in range(n)]
    with kv.KVCache(blocks, 1, D) as c:
        c.write(k, v, torch.arange(blocks * 16, device="cuda"))
        plan = kv.AttentionPlan(c, g, T, len(spans), blocks)
        plan.set(T, spans, list(range(blocks)))
        out = torch.full_like(q, 77.0)
        lse = torch.full((T, g), 77.0, device="cuda")
        c.attend(q, plan, out=out, lse=lse)
        c.check()
    for t in range(T):
        if t >= n:
            assert not out[t].any() and torch.isneginf(lse[t]).all()
            continue
        sel = torch.cat([torch.arange(shared, device="cuda"), torch.arange(own, device="cuda") + 16 * (4 + 3 * t)])
        K, V, x = k[sel, 0].double(), v[sel, 0].double(), q[t].double()
        z = x @ K.T * D ** -0.5
        w = torch.softmax(z, -1)
        mag = (x.abs() @ K.abs().T).amax(-1) * D ** -0.5
        tol, tl = ref.bounds("bf16", D, w @ V, w @ V.abs(), mag, None, 0.0)
        assert ((out[t].double() - w @ V).abs() <= tol).all(), t
        assert ((lse[t].double() - torch.logsumexp(z, -1)).abs() <= tl).all(), t
