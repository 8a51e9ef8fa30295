"""A batch without a key inside a CUDA graph: the join is the call's first kernel and follows nodes of any kind."""
import pytest
import torch

from tests.test_gpu_kv_attend import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("before", ["copy", "zero", "nothing"])
@pytest.mark.parametrize("spans", [[], [(0, 3, 0, 0, 0), (1, 4, 0, 1, 0)]])
def test_no_key_in_a_graph(kv, before, spans):
    T, HQ, D = 5, 8, 64
    with kv.KVCache(4, 2, D, fmt="fp16") as c:
        plan = kv.AttentionPlan(c, HQ, T, 4, 4)
        plan.set(T, spans, [])
        q = torch.randn(T, HQ, D, device="cuda").half()
        other = torch.full_like(q, 77.0)
        out, lse = torch.empty_like(q), torch.empty(T, HQ, device="cuda")
        c.attend(q, plan, out=out, lse=lse)
        c.check()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            if before == "copy":
                out.copy_(other)
            elif before == "zero":
                lse.zero_()
            c.attend(q, plan, out=out, lse=lse)
            after = out.clone()
        for _ in range(5):
            out.fill_(3.0)
            lse.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert not out.any() and not after.any() and torch.isneginf(lse).all()
        graph.reset()
        c.check()
