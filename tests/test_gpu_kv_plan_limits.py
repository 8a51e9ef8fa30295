"""Batches that are refused because the plan's 32-bit indexes would not hold them."""
import pytest

from tests.test_gpu_kv_attend import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


def test_spans_over_more_queries_than_a_plan_counts(kv):
    """2^27 queries under 32 spans: the list of each query's spans would have 2^32 entries."""
    import paper_2609_33224_gb300 as P
    T = 1 << 27
    with kv.KVCache(4, 1, 64) as c:
        plan = kv.AttentionPlan(c, 1, T, 64, 64)
        with pytest.raises(P.PSError, match="too large"):
            plan.set(T, [(0, T, 1, 0, 0)] * 32, [0])
        plan.set(2, [(0, 2, 1, 0, 0)] * 32, [0])
