"""A whole step with drafted tokens captured into one graph: masks and positions, rotated writes, attention, moves, block copies
and a read, replayed with other trees, tokens and moves beside the same calls made eagerly on another stream."""
import random

import numpy as np
import pytest
import torch

from tests.test_gpu_kv_drafts import tree
from tests.test_gpu_kv_store import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,D,nodes", [("fp8", 128, [33, 9, 20]), ("bf16", 64, [150, 200, 250]), ("fp16", 128, [64] * 12)])
def test_replays_are_what_eager_calls_give(kv, fmt, D, nodes):  # noqa: F811
    rng = random.Random(len(nodes))
    H, g, context = 2, 8, 333
    T, R = sum(nodes), len(nodes)
    per = -(-(context + max(nodes)) // 16)
    blocks = R * per + 10
    gen = torch.Generator(device="cuda").manual_seed(3)
    dt = torch.float16 if fmt == "fp16" else torch.bfloat16
    rand = lambda n, h: torch.randn(n, h, D, device="cuda", generator=gen).to(dt)  # noqa: E731
    tables = [list(range(i * per, (i + 1) * per)) for i in range(R)]
    order, spans, ids = kv.shared_spans(tables, [context + n for n in nodes], nodes, masked=True)
    assert list(order) == list(range(R))
    a, b = (kv.KVCache(blocks, H, D, fmt=fmt) for _ in range(2))
    every = torch.arange(blocks * 16, device="cuda")
    k0, v0 = rand(blocks * 16, H), rand(blocks * 16, H)
    plans = []
    for c in (a, b):
        c.write(k0, v0, every)
        plans.append(kv.AttentionPlan(c, H * g, T, len(spans), len(ids)))
        plans[-1].set(T, spans, ids, masked=True)
    slots = torch.cat([torch.arange(i * per * 16 + context, i * per * 16 + context + n, device="cuda") for i, n in enumerate(nodes)])
    offsets = torch.tensor(np.cumsum([0] + nodes)).cuda()
    rotary = kv.Rotary(D)
    # what changes from step to step
    parents = torch.empty(T, dtype=torch.int32, device="cuda")
    start = torch.empty(R, dtype=torch.int64, device="cuda")
    src, dst = torch.empty_like(slots), torch.empty_like(slots)
    q, k, v = rand(T, H * g), rand(T, H), rand(T, H)
    fork, to = torch.empty(5, dtype=torch.int64, device="cuda"), torch.empty(5, dtype=torch.int64, device="cuda")

    def new():
        parents.copy_(torch.tensor(sum((tree(rng, n, rng.choice(["any", "near", "early", "chain"])) for n in nodes), []), dtype=torch.int32))
        start.copy_(torch.tensor([rng.randrange(10 ** 6) for _ in nodes]))
        src.copy_(slots[torch.randperm(T, device="cuda", generator=gen)])
        dst.copy_(slots[torch.randperm(T, device="cuda", generator=gen)])
        dst[torch.rand(T, device="cuda", generator=gen) < 0.3] = -1
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda", generator=gen))
        fork.copy_(torch.randperm(R * per, device="cuda", generator=gen)[:5])
        to.copy_(R * per + torch.randperm(10, device="cuda", generator=gen)[:5])

    def step(c, plan):
        mask, positions = c.tree_mask(parents, offsets, max(nodes), start)
        turned = c.write_rotated(k, v, slots, positions, rotary, q=q)
        out = c.attend(turned, plan, mask=mask)
        c.move(src, dst)
        c.copy_blocks(fork, to)
        return mask, positions, turned, out, *c.read(every)

    new()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a, plans[0])
    s = torch.cuda.Stream()
    for _ in range(4):
        new()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            want = step(b, plans[1])
        graph.replay()
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(got, want)):
            assert torch.equal(x, y), i
    a.check()
    b.check()
    a.close()
    b.close()
