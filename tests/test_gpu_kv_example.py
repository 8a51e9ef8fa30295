"""The example that takes a scheduled window through the block cache and the attention on it."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("fmt", ["fp8", "bf16"])
def test_window_to_attention(fmt):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for the gpu tests")
    import __graft_entry__ as g
    g.build()
    spec = importlib.util.spec_from_file_location("instance_step", os.path.join(ROOT, "examples", "instance_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.main(fmt)
    assert r["requests"] > 1 and r["prefill_tokens"] > 0 and r["cached_tokens"] > 0
    # probabilities and output are rounded to bf16 once each: at most 2^-8 of sum p |v|, in the norm far less
    assert r["error"] < 2 * 2.0 ** -8
