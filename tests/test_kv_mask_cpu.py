"""A mask that the batch would not look at is refused, not dropped."""
import types

import pytest
import torch

from tests.test_kv_drafts_cpu import cache, kv  # noqa: F401 (fixtures)


def test_a_mask_without_masked_spans_is_refused(kv, cache):  # noqa: F811
    q, mask = torch.zeros(5, 6, 64).bfloat16(), torch.zeros(5, 1, dtype=torch.int32)
    plan = types.SimpleNamespace(_open=lambda: 1, num_queries=5, q_heads=6, masked=0, workspace_bytes=0)
    with pytest.raises(ValueError, match="no masked span"):
        cache.attend(q, plan, mask=mask)
    assert cache.reached == []
    cache.attend(q, plan)
    plan.num_queries = 0  # an empty batch's mask has no row
    cache.attend(q[:0], plan, mask=mask[:0])
    plan.num_queries, plan.masked = 5, 3
    cache.attend(q, plan, mask=mask)
    assert cache.reached == ["ps_kv_attend", "ps_kv_attend", "ps_kv_attend_masked"]
