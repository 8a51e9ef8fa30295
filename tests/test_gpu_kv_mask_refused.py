"""A mask that the batch would not look at is refused, not dropped."""
import ctypes

import pytest
import torch

from tests.test_gpu_kv_store import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


def test_a_mask_without_masked_spans_is_refused(kv):  # noqa: F811
    """A tree's mask with spans that are causal by mistake, or a plan that was set without masked spans."""
    import paper_2609_33224_gb300 as P
    with kv.KVCache(8, 2, 128) as c:
        p = kv.AttentionPlan(c, 4, 4, 1, 8)
        q = torch.zeros(4, 4, 128, device="cuda", dtype=torch.bfloat16)
        o = torch.empty_like(q)
        mask = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
        for causal, masked in ((1, False), (1, True), (0, True)):
            p.set(4, [(0, 4, 50, causal, 0)], range(8), masked=masked)
            with pytest.raises(ValueError, match="no masked span"):
                c.attend(q, p, mask=mask)
            c.attend(q, p)
            rows, out = (P.PsKvRows(x.data_ptr(), 512, 128, 0) for x in (q, o))
            ws = torch.empty(max(256, p.workspace_bytes), dtype=torch.uint8, device="cuda")
            call = lambda m, words: P.lib().ps_kv_attend_masked(  # noqa: E731
                c._h, p._h, ctypes.addressof(rows), ctypes.addressof(out), None, 1.0, m, 1, words, ws.data_ptr(), ws.numel(), None)
            assert call(mask.data_ptr(), 1) == 1 and b"no masked span" in P.lib().ps_kv_last_error(c._h)
            assert call(None, 0) == 0
        p.set(4, [(0, 4, 50, 2, 0)], range(8), masked=True)
        c.attend(q, p, mask=mask)
        p.set(0, [], [], masked=True)
        assert c.attend(q[:0], p, mask=mask[:0]).shape == (0, 4, 128)
        c.check()
