"""Moves on both sides of the numbers of tokens where another form begins: a thread's second token, and the workspace."""
import ctypes

import pytest
import torch

from tests.test_gpu_kv_copies import SHAPES, test_moves_are_as_if_all_were_read_first as moved
from tests.test_gpu_kv_store import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,H,D", SHAPES)
@pytest.mark.parametrize("n", [255, 256, 257, 511, 512, 513])
def test_moves_are_as_if_all_were_read_first(kv, fmt, H, D, n):  # noqa: F811
    moved(kv, fmt, H, D, n)


@pytest.mark.parametrize("fmt,D", [("bf16", 128), ("fp8", 64)])
def test_the_binding_asks_for_what_the_library_needs(kv, fmt, D):  # noqa: F811
    """Up to 512 tokens need no workspace; KVCache.move asks for none up to 256."""
    import paper_2609_33224_gb300 as P
    with kv.KVCache(8, 2, D, fmt=fmt) as c:
        got = ctypes.c_uint64()
        for n, some in ((1, False), (256, False), (257, False), (512, False), (513, True), (5000, True)):
            assert P.lib().ps_kv_move_workspace(c._h, n, ctypes.byref(got)) == 0 and (got.value > 0) == some
