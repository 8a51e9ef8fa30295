"""A CUDA graph keeps the cache's blocks and the plan's arrays that its calls read."""
import gc
import time

import pytest
import torch

from tests.test_gpu_kv_attend import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu

H, HQ, D, BLOCKS, T = 2, 8, 128, 4096, 6


def _captured(kv, blocks=BLOCKS):
    """A graph of a write, an attention and a read, its inputs and outputs, and its cache and plan."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    cache = kv.KVCache(blocks, H, D, fmt="fp8")
    n = 3000
    k, v = (torch.randn(n, H, D, device="cuda", generator=gen).bfloat16() for _ in range(2))
    slots = torch.randperm(blocks * 16, device="cuda", generator=gen)[:n].contiguous()
    every = torch.randn(BLOCKS * 16, H, D, device="cuda", generator=gen).bfloat16()
    cache.write(every, every, torch.arange(BLOCKS * 16, device="cuda"))
    plan = kv.AttentionPlan(cache, HQ, T, T + 1, BLOCKS)
    spans = [(0, T, 20000, 0, 0)] + [(i, 1, 700 + i, 1, 2000 + 50 * i) for i in range(T)]
    plan.set(T, spans, list(range(BLOCKS)))
    q = torch.randn(T, HQ, D, device="cuda", generator=gen).bfloat16()
    cache.write(k, v, slots)
    want = (cache.attend(q, plan), *cache.read(slots))
    cache.check()
    out = torch.empty_like(q)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.write(k, v, slots)
        cache.attend(q, plan, out=out)
        cache.read(slots, k=ko, v=vo)
    return graph, (k, v, slots, q), (out, ko, vo), want, cache, plan


@pytest.mark.parametrize("order", ["plan", "cache", "collected"])
def test_replay_after_release(kv, order):
    graph, inputs, got, want, cache, plan = _captured(kv)
    if order == "plan":
        plan.close()
    elif order == "cache":
        cache.close()  # and its plan
    else:
        del cache, plan
        gc.collect()
    # what would take freed memory, filled with other things
    others = []
    for _ in range(4):
        c = kv.KVCache(BLOCKS, H, D, fmt="fp8")
        x = torch.randn(BLOCKS * 16, H, D, device="cuda").bfloat16()
        c.write(x, x, torch.arange(BLOCKS * 16, device="cuda"))
        p = kv.AttentionPlan(c, HQ, T, T + 1, BLOCKS)
        p.set(T, [(0, T, 3, 0, 7)], list(range(BLOCKS))[::-1])
        others.append((c, p, c.attend(inputs[3], p)))
    for _ in range(3):
        for x in got:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)
    for c, p, y in others:
        assert torch.equal(c.attend(inputs[3], p), y)
        c.check()


def test_memory_is_freed_with_the_graph(kv):
    """Kept while the graph is, then freed by a later call; without a graph freed at once."""
    big = 1 << 18  # 2.2 GB
    torch.cuda.synchronize()
    kv.KVCache(1, 1, 64).close()
    torch.cuda.empty_cache()
    free = lambda: torch.cuda.mem_get_info()[0]
    before = free()
    cache = kv.KVCache(big, H, D, fmt="fp8")
    size = before - free()
    assert size > 2 << 30
    cache.close()
    assert free() > before - size // 2
    graph, *rest = _captured(kv, big)
    rest[-2].close()
    assert free() < before - size // 2
    graph.replay()
    torch.cuda.synchronize()
    graph.reset()
    del graph, rest
    gc.collect()
    for _ in range(100):  # the driver gives the reference up on a thread of its own
        kv.KVCache(1, 1, 64).close()
        if free() > before - size // 2:
            break
        time.sleep(0.05)
    assert free() > before - size // 2


def test_a_captured_plan_stays_as_it_is(kv):
    """A refused set leaves the plan's batch in place, for eager calls and for replays."""
    import paper_2609_33224_gb300 as P
    graph, inputs, got, want, cache, plan = _captured(kv)
    with pytest.raises(P.PSError, match="PS_ERR_STATE"):
        plan.set(1, [(0, 1, 5, 0, 0)], [0])
    assert torch.equal(cache.attend(inputs[3], plan), want[0])
    got[0].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0])


def test_a_plan_is_free_again_after_its_graph(kv):
    import paper_2609_33224_gb300 as P
    graph, inputs, got, want, cache, plan = _captured(kv)
    span = [(0, T, 700, 0, 0)]
    with pytest.raises(P.PSError, match="PS_ERR_STATE"):
        plan.set(T, span, list(range(BLOCKS)))
    graph.replay()
    torch.cuda.synchronize()
    graph.reset()
    for _ in range(100):  # the driver gives the reference up on a thread of its own
        try:
            plan.set(T, span, list(range(BLOCKS)))
            break
        except P.PSError:
            time.sleep(0.05)
    other = kv.AttentionPlan(cache, HQ, T, 1, BLOCKS)
    other.set(T, span, list(range(BLOCKS)))
    assert torch.equal(cache.attend(inputs[3], plan), cache.attend(inputs[3], other))
    cache.check()


def test_a_plan_without_spans(kv):
    """Limits of zero: a batch without a key."""
    with kv.KVCache(4, H, D) as c:
        plan = kv.AttentionPlan(c, HQ, T, 0, 0)
        for n in (0, T, 0, 1):
            plan.set(n, [], [])
            q = torch.ones(n, HQ, D, device="cuda").bfloat16()
            assert not c.attend(q, plan).any()
        c.check()
