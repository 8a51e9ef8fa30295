"""Tensors that receive results: rows that overlap are refused, strides of every other kind taken."""
import itertools

import pytest
import torch

from tests.test_gpu_kv_attend import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


def _overlap(n, heads, ts, hs, D):
    rows = sorted(t * ts + h * hs for t in range(n) for h in range(heads))
    return any(b - a < D for a, b in zip(rows, rows[1:]))


def test_results_in_strided_tensors(kv):
    import paper_2609_33224_gb300 as P
    H, D, n = 2, 64, 4
    with kv.KVCache(8, H, D) as c:
        k, v = (torch.randn(n, H, D, device="cuda").bfloat16() for _ in range(2))
        slots = torch.arange(n, device="cuda")
        c.write(k, v, slots)
        plan = kv.AttentionPlan(c, H, n, 1, 8)
        plan.set(n, [(0, n, n, 0, 0)], [0])
        q = torch.randn(n, H, D, device="cuda").bfloat16()
        want = c.attend(q, plan)
        refused = 0
        for ts, hs in itertools.product((0, 8, 56, 64, 72, 96, 128, 192, 256, 320, 512), repeat=2):
            hold = [torch.zeros(2048 + D, device="cuda", dtype=torch.bfloat16) for _ in range(3)]
            a, b, o = (x.as_strided((n, H, D), (ts, hs, 1)) for x in hold)
            if _overlap(n, H, ts, hs, D):
                refused += 1
                good = torch.zeros_like(k)
                for kk, vv in ((a, good), (good, b)):
                    with pytest.raises(P.PSError, match="overlap"):
                        c.read(slots, k=kk, v=vv)
                with pytest.raises(P.PSError, match="overlap"):
                    c.attend(q, plan, out=o)
            else:
                c.read(slots, k=a, v=b)
                c.attend(q, plan, out=o)
                assert torch.equal(a, k) and torch.equal(b, v) and torch.equal(o, want)
        assert 40 < refused < 100
        c.check()


def test_single_rows_and_repeated_inputs(kv):
    """A lone token's or head's stride is no matter; what is read may repeat a row."""
    D = 128
    with kv.KVCache(8, 1, D) as c:
        x = torch.randn(1, 1, D, device="cuda").bfloat16()
        slots = torch.arange(5, device="cuda")
        c.write(x.expand(5, 1, D), x.expand(5, 1, D), slots)
        k, v = c.read(slots)
        assert torch.equal(k, x.expand(5, 1, D).contiguous()) and torch.equal(v, k)
        one = torch.zeros(1, 1, D, device="cuda").bfloat16().as_strided((1, 1, D), (0, 0, 1))
        c.read(slots[:1], k=one, v=torch.empty_like(x))
        assert torch.equal(one, x)
        e = torch.zeros(0, 1, D, device="cuda").bfloat16()
        c.read(slots[:0], k=e, v=e)
        plan = kv.AttentionPlan(c, 2, 3, 1, 8)
        plan.set(3, [(0, 3, 5, 0, 0)], [0])
        q = torch.randn(1, 2, D, device="cuda").bfloat16().expand(3, 2, D)
        out = c.attend(q, plan)
        assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
        c.check()
