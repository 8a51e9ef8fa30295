"""Masked attention in the rarer forms of its kernels: pieces of drafts that are split by the parity of their steps, and joins
by entries.  That the batches reach them is tests/test_kv_plan_shapes_host.py's to check."""
import math
import random

import pytest
import torch

from tests import test_kv_plan_shapes_host as shapes
from tests.test_gpu_kv_drafts import Drafts, rows_of, tree
from tests.test_gpu_kv_store import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


def drafts(kv, fmt, D, shape, seed):  # noqa: F811
    H, g, T, spans = shape
    rng = random.Random(seed)
    sees = []
    for _, n, _, kind in spans:
        if kind:
            sees += [s for s, _ in rows_of(tree(rng, n, "near"))] if kind == 2 else [set()] * n
    return Drafts(kv, fmt, H, g, D, spans, T, sees, seed=seed)


@pytest.mark.parametrize("fmt,name", [(f, n) for f in ("bf16", "fp16", "fp8") for n in shapes.SPLIT] + [("bf16", n) for n in shapes.SPLIT_LONG])
def test_pieces_split_by_steps(kv, fmt, name):  # noqa: F811
    """Finite values first; then a NaN and an infinity among the drafted tokens on either side of the multiple of 128 that
    they straddle, which reach the queries that see them, in their columns, and nothing else."""
    d = drafts(kv, fmt, 128, {**shapes.SPLIT, **shapes.SPLIT_LONG}[name], seed=len(name))
    out, lse = d.run()
    d.check(out, lse)
    d.check(*d.run(scale=-0.1), scale=-0.1)
    clean, _, tol, _, _ = d.expected()
    for (f, n, length, _, _), sl in zip(d.spans, d.slots_of):
        border = length // 128 * 128  # the first key of the last step
        assert length - n < border < length
        d.v[sl[length - n], :, 7] = math.nan
        d.v[sl[border], :, 70] = math.nan
        if fmt != "fp8":  # (an infinity is held as a large finite number there)
            d.v[sl[border - 1], :, 71] = math.inf
            d.v[sl[length - 1], :, 8] = -math.inf
    d.write()
    dirty, _, _, _, _ = d.expected()
    odd = ~torch.isfinite(dirty)
    assert odd.any() and not odd.all()
    bad, again = d.run()
    assert torch.equal(torch.isnan(bad), torch.isnan(dirty)) and torch.equal(torch.isinf(bad), torch.isinf(dirty))
    inf = torch.isinf(dirty)
    assert torch.equal(bad[inf].double(), dirty[inf])
    assert ((bad.double() - clean).abs() <= tol)[~odd].all()
    assert torch.equal(again, lse)
    d.cache.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("name", list(shapes.ENTRIES))
def test_joins_by_entries(kv, fmt, name):  # noqa: F811
    (D, *shape), _, _ = shapes.ENTRIES[name]
    d = drafts(kv, fmt, D, shape, seed=len(name))
    plain = all(s[3] != 2 for s in shape[-1])
    out, lse = d.run(**({"mask": None} if plain else {}))
    d.check(out, lse)
    d.cache.close()
