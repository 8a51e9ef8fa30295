"""A captured call's workspace belongs to its graph, whichever device is current (torch's CUDA state is faked)."""
import contextlib
import types

import pytest
import torch


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("captures", [0, 1, None])
def test_the_caches_stream_is_asked(monkeypatch, current, captures):
    from paper_2609_33224_gb300 import kvcache
    now = [current]

    @contextlib.contextmanager
    def device(d):
        was, now[0] = now[0], d
        yield
        now[0] = was

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: now[0] == captures)
    plan = kvcache.AttentionPlan.__new__(kvcache.AttentionPlan)
    plan._h, plan._spaces = None, {}
    plan.cache = types.SimpleNamespace(device=1, _device=torch.device("cpu"))
    a, b = plan._workspace(7, 100), plan._workspace(7, 100)
    assert now[0] == current
    if captures == 1:
        assert not plan._spaces and a.data_ptr() != b.data_ptr()
    else:
        assert a is b and plan._spaces[7] is a
