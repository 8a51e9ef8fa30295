"""Attention of a batch over the block cache against a 64-bit form, within elementwise bounds derived from the
arithmetic (tests/kv_reference.py)."""
import math

import numpy as np
import pytest

from tests import kv_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for the gpu tests")
    import paper_2609_33224_gb300 as P
    P.build()
    from paper_2609_33224_gb300 import kvcache
    return kvcache


class Batch:
    """A cache filled at random with the tokens of spans (first, queries, length, causal), blocks in random order,
    the unused slots of last blocks holding other tokens, NaNs and infinities among them."""

    def __init__(self, kv, fmt, Hkv, g, D, spans, T, seed=0, qscale=1.0):
        import torch
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.kv, self.fmt, self.T, self.D, self.Hq = kv, fmt, T, D, Hkv * g
        need = [-(-s[2] // 16) for s in spans]
        total = sum(need)
        blocks = total + 5
        ids = rng.permutation(blocks)[:total].astype(np.uint32)
        at = np.concatenate([[0], np.cumsum(need)]).astype(int)
        self.spans = [(*s, int(a)) for s, a in zip(spans, at)]
        self.ids = ids
        slots = (torch.from_numpy(ids.astype(np.int64)).cuda()[:, None] * 16 + torch.arange(16, device="cuda")).reshape(-1)
        self.slots_of = [slots[16 * a:16 * a + s[2]] for s, a in zip(spans, at)]
        dt = torch.float16 if fmt == "fp16" else torch.bfloat16
        k = torch.randn(blocks * 16, Hkv, D, device="cuda", generator=gen)
        k *= torch.exp2(torch.randint(-2, 3, (blocks * 16, Hkv, 1), device="cuda", generator=gen).float())
        v = torch.randn(blocks * 16, Hkv, D, device="cuda", generator=gen)
        self.q = (torch.randn(T, self.Hq, D, device="cuda", generator=gen) * qscale).to(dt)
        self.k, self.v = k.to(dt), v.to(dt)
        # what lies in the blocks' other slots must not matter
        free = torch.ones(blocks * 16, dtype=torch.bool, device="cuda")
        for s in self.slots_of:
            free[s] = False
        self.k[free] = math.nan
        self.v[free] = torch.where(torch.rand(int(free.sum()), Hkv, D, device="cuda", generator=gen) < 0.5, math.inf, math.nan).to(dt)
        self.cache = kv.KVCache(blocks, Hkv, D, fmt=fmt)
        self.cache.write(self.k, self.v, torch.arange(blocks * 16, device="cuda"))
        self.plan = kv.AttentionPlan(self.cache, self.Hq, max(T, 1), max(len(spans), 1), max(total, 1))
        self.plan.set(T, self.spans, ids)

    def run(self, **kw):
        import torch
        lse = torch.full((self.T, self.Hq), 77.0, device="cuda")
        out = self.cache.attend(self.q, self.plan, lse=lse, **kw)
        self.cache.check()
        return out, lse

    def check(self, out, lse, scale=None):
        import torch
        scale = self.D ** -0.5 if scale is None else scale
        k, v = ref.held(self.fmt, self.k), ref.held(self.fmt, self.v)
        want, wl, A, mag, cnt = ref.attend(self.q, k, v, self.spans, self.slots_of, scale)
        vmax = max((v[s].abs().max().item() for s in self.slots_of if s.numel()), default=0.0)
        tol, tl = ref.bounds(self.fmt, self.D, want, A, mag, cnt, vmax)
        none = cnt == 0
        assert not out[none].any() and torch.isneginf(lse[none]).all()
        assert torch.isfinite(out).all()
        over = (out.double() - want).abs() / tol.clamp(min=1e-30)
        assert over.max() <= 1.0 if over.numel() else True, over.max().item()
        d = ((lse.double() - wl).abs() / tl)[~none]
        assert d.max() <= 1.0 if d.numel() else True, d.max().item()


LAYOUTS = {
    # one token alone, around the block size
    "one": lambda: (5, [(i, 1, n, 0) for i, n in enumerate((1, 15, 16, 17, 1000))]),
    # a shared prefix and the requests' own tokens, none for some
    "shared": lambda: (9, [(0, 9, 321, 0)] + [(i, 1, n, 1) for i, n in enumerate((1, 16, 0, 33, 0, 100, 7, 250, 2))]),
    # three levels, a query that nothing covers, an empty prefix
    "tree": lambda: (12, [(0, 11, 40, 0), (0, 5, 129, 0), (5, 6, 0, 0)] + [(i, 1, 3 * i + 1, 1) for i in range(11)]),
    # several new tokens per request on a prefix; fewer tokens than queries leaves the first rows empty
    "extend": lambda: (5 + 40 + 1 + 17, [(0, 45, 200, 0), (0, 5, 3, 1), (5, 40, 77, 1), (45, 1, 1, 1), (46, 17, 17, 1)]),
    "extend_empty": lambda: (30, [(0, 20, 4, 1), (20, 10, 0, 1)]),
    # a long batch of many queries: every way of tiling, odd sizes
    "wide": lambda: (150, [(0, 150, 700, 0), (3, 147, 290, 1)]),
    # long chains cut over many workers
    "long": lambda: (3, [(0, 3, 20011, 0), (0, 1, 9000, 1), (2, 1, 30001, 1)]),
}


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("fmt,Hkv,g,D", [("bf16", 2, 8, 128), ("fp8", 2, 8, 128), ("fp16", 3, 1, 64), ("bf16", 1, 5, 64),
                                         ("fp8", 1, 16, 64), ("fp8", 1, 21, 128), ("fp16", 2, 4, 128)])
def test_against_64_bits(kv, layout, fmt, Hkv, g, D):
    T, spans = LAYOUTS[layout]()
    b = Batch(kv, fmt, Hkv, g, D, spans, T, seed=len(layout) + g)
    b.check(*b.run())


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_peaked_scores_and_scales(kv, fmt):
    """Scores of some hundreds: the running maximum moves a lot; a negative and a zero scale."""
    T, spans = LAYOUTS["shared"]()
    b = Batch(kv, fmt, 2, 4, 128, spans, T, seed=3, qscale=8.0)
    for scale in (None, -0.3, 0.0):
        b.check(*b.run(scale=scale), scale=scale)


@pytest.mark.parametrize("fmt", ["bf16", "fp16", "fp8"])
def test_later_tokens_that_are_not_finite(kv, fmt):
    """A NaN or an infinity in a key or value reaches the queries that see it and no other."""
    import torch
    n = 40
    b = Batch(kv, fmt, 1, 4, 64, [(0, n, 100, 0), (0, n, n + 9, 1)], n, seed=5)
    clean, _ = b.run()
    k, v = b.k.clone(), b.v.clone()
    sl = b.slots_of[1]
    v[sl[9 + 20], :, 7] = math.nan     # seen by queries 20..
    v[sl[9 + 25], :, 9] = math.inf     # seen by queries 25..
    k[sl[9 + 30]] = math.nan           # seen by queries 30..
    b.cache.write(k, v, torch.arange(k.shape[0], device="cuda"))
    out, _ = b.run()
    assert torch.equal(out[:20], clean[:20])
    assert torch.isnan(out[20:, :, 7]).all()
    assert torch.isnan(out[30:]).all()
    keep = [d for d in range(64) if d not in (7, 9)]
    if fmt == "fp8":  # a row with a NaN is NaN whole; an infinity is held as a large number
        assert torch.isnan(out[20:]).all()
    else:
        assert torch.isposinf(out[25:30, :, 9]).all()
        want, _, A, mag, cnt = ref.attend(b.q, ref.held(fmt, k).nan_to_num(0, 0, 0), ref.held(fmt, v).nan_to_num(0, 0, 0),
                                          b.spans, b.slots_of, 64 ** -0.5)
        tol, _ = ref.bounds(fmt, 64, want, A, mag, cnt, 8.0)
        assert ((out[:30].double() - want[:30]).abs() <= tol[:30])[:, :, keep].all()


def test_shared_and_unshared_agree(kv):
    """The prefix as one span for all, and as a span of its own per request."""
    import torch
    T, P0 = 24, 333
    b = Batch(kv, "bf16", 2, 8, 128, [(0, T, P0, 0)] + [(i, 1, 5 + i, 1) for i in range(T)], T, seed=9)
    out, lse = b.run()
    alone = [(i, 1, P0, 0, 0) for i in range(T)] + b.spans[1:]
    p2 = kv.AttentionPlan(b.cache, 16, T, len(alone), len(b.ids))
    p2.set(T, alone, b.ids)
    b.plan = p2
    out2, lse2 = b.run()
    b.check(out2, lse2)
    b.check(out, lse)


def test_strided_tensors_and_reuse_of_a_plan(kv):
    """q as a slice of a fused projection, out and lse given; a plan set again for longer spans; results do not
    depend on what ran before."""
    import torch
    T, spans = LAYOUTS["shared"]()
    b = Batch(kv, "bf16", 2, 4, 128, spans, T, seed=11)
    first, _ = b.run()
    wide = torch.randn(T, 3, 8, 128, device="cuda").to(torch.bfloat16)
    wide[:, 1] = b.q
    hold = torch.zeros(T, 8, 2, 128, device="cuda", dtype=torch.bfloat16)
    r = b.cache.attend(wide[:, 1], b.plan, out=hold[:, :, 1])
    assert r.data_ptr() == hold[:, :, 1].data_ptr()
    assert torch.equal(hold[:, :, 1], first) and not hold[:, :, 0].any()
    for n in (1, 300, 17, 321):
        sp = [(0, T, n, 0, 0)]
        b.plan.set(T, sp, b.ids)
        b.spans, keep = [s + () for s in sp], b.slots_of
        b.slots_of = [keep[0][:n]]
        b.check(*b.run())
        b.slots_of = keep
    b.plan.set(T, [(*s, a) for s, a in zip(spans, np.concatenate([[0], np.cumsum([-(-s[2] // 16) for s in spans])]))], b.ids)
    assert torch.equal(b.run()[0], first)
    b.plan.set(0, [], [])
    assert b.cache.attend(b.q[:0], b.plan).shape == (0, 8, 128)


def test_streams_and_graphs(kv):
    import torch

    import paper_2609_33224_gb300 as P
    T, spans = LAYOUTS["tree"]()
    b = Batch(kv, "fp8", 2, 4, 128, spans, T, seed=13)
    want, _ = b.run()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for i in range(9):
        s = streams[i % 3]
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(b.cache.attend(b.q, b.plan))
    b.plan.set(T, b.spans, b.ids)  # while calls may still run
    got.append(b.cache.attend(b.q, b.plan))
    torch.cuda.synchronize()
    for g in got:
        assert torch.equal(g, want)
    out = torch.empty_like(b.q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.cache.attend(b.q, b.plan, out=out)
    for seed in range(3):
        q2 = torch.randn(b.q.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(b.q.dtype)
        b.q.copy_(q2)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, b.cache.attend(b.q, b.plan))
    with pytest.raises(P.PSError, match="PS_ERR_STATE"):
        b.plan.set(T, b.spans, b.ids)
    del graph


def test_blocks_past_32_bits(kv):
    import torch
    H, D, blocks = 8, 128, 150000
    with kv.KVCache(blocks, H, D, fmt="fp8") as c:
        n = 50
        k = torch.randn(n, H, D, device="cuda").bfloat16()
        v = torch.randn(n, H, D, device="cuda").bfloat16()
        ids = np.array([blocks - 1, 3, blocks - 2, 140000], np.uint32)
        slots = (torch.from_numpy(ids.astype(np.int64)).cuda()[:, None] * 16 + torch.arange(16, device="cuda")).reshape(-1)[:n]
        c.write(k, v, slots.contiguous())
        q = torch.randn(1, 16, D, device="cuda").bfloat16()
        p = kv.AttentionPlan(c, 16, 1, 1, 4)
        p.set(1, [(0, 1, n, 0, 0)], ids)
        out = c.attend(q, p)
        want, _, A, mag, cnt = ref.attend(q, ref.held("fp8", k), ref.held("fp8", v), [(0, 1, n, 0)],
                                          [torch.arange(n, device="cuda")], D ** -0.5)
        tol, _ = ref.bounds("fp8", D, want, A, mag, cnt, 8.0)
        assert ((out.double() - want).abs() <= tol).all()
        c.check()


def test_refusals(kv):
    import torch

    import paper_2609_33224_gb300 as P
    with kv.KVCache(8, 2, 128) as c:
        with pytest.raises(P.PSError, match="multiple of kv_heads"):
            kv.AttentionPlan(c, 3, 4, 4, 8)
        p = kv.AttentionPlan(c, 4, 4, 2, 8)
        q = torch.zeros(4, 4, 128, device="cuda", dtype=torch.bfloat16)
        with pytest.raises(P.PSError, match="no batch"):
            c.attend(q[:0], p)
        bad = [((5, [], []), "max_queries"), ((4, [(0, 1, 1, 0, 0)] * 3, [0]), "max_spans"), ((4, [], [0] * 9), "max_blocks"),
               ((4, [(0, 5, 1, 0, 0)], [0]), "inside the batch"), ((4, [(3, 2, 1, 0, 0)], [0]), "inside the batch"),
               ((4, [(0, 1, 17, 0, 0)], [0]), "block array"), ((4, [(0, 1, 1, 0, 1)], [0]), "block array"),
               ((4, [(0, 1, 1, 2, 0)], [0]), "causal"), ((4, [(0, 1, 1 << 30, 0, 0)], [0]), "2\\^30"),
               ((4, [(0, 1, 1, 0, 0)], [8]), "outside the cache")]
        for args, msg in bad:
            with pytest.raises(P.PSError, match=msg):
                p.set(*args)
            with pytest.raises(P.PSError, match="no batch"):
                c.attend(q[:0], p)
        with pytest.raises(ValueError):
            p.set(4, [(0, -1, 1, 0, 0)], [0])
        with pytest.raises(ValueError):
            p.set(4, [(0, 1, 1, 0, 0)], [-1])
        p.set(4, [(0, 4, 20, 0, 0)], [2, 5])
        for x in (q[:3], q[:, :2], q.float().cpu(), q.transpose(0, 1)[:4, :4, :64]):
            with pytest.raises(ValueError):
                c.attend(x, p)
        with pytest.raises(P.PSError, match="16-bit type"):
            c.attend(q.half(), p)
        with pytest.raises(P.PSError, match="finite"):
            c.attend(q, p, scale=math.inf)
        with pytest.raises(ValueError):
            c.attend(q, p, lse=torch.zeros(4, 4, device="cuda", dtype=torch.float64))
        with kv.KVCache(8, 2, 64) as other, kv.KVCache(4, 2, 128) as small:
            with pytest.raises(P.PSError, match="another shape"):
                other.attend(q[:, :, :64].contiguous(), p)
            with pytest.raises(P.PSError, match="another shape"):
                small.attend(q, p)
        c.attend(q, p)
        c.check()
    with pytest.raises(ValueError, match="closed"):
        c.attend(q, p)


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(kv, seed):
    """Random spans, formats, groups and head sizes: rows and tiles, joins of every kind."""
    import random
    rng = random.Random(seed)
    D, fmt = rng.choice([64, 128]), rng.choice(["bf16", "fp16", "fp8"])
    Hkv, g = rng.choice([1, 2, 3]), rng.choice([1, 2, 4, 5, 8, 16])
    T = rng.choice([3, 40, 130])
    spans = [(0, T, rng.choice([0, 37, 1200, 5000]), 0)]
    first = 0
    while first < T:
        n = min(T - first, rng.choice([1, 1, 7, 70]))
        if rng.random() < 0.9:
            spans.append((first, n, rng.choice([0, n, n + 15, n + 300, 900, max(1, n - 2)]), 1))
        if n > 1 and rng.random() < 0.3:
            spans.append((first, n, rng.randrange(1, 700), 0))
        first += n
    b = Batch(kv, fmt, Hkv, g, D, spans, T, seed=100 + seed)
    b.check(*b.run())


@pytest.mark.parametrize("fmt,D", [("bf16", 128), ("fp8", 128), ("fp16", 64), ("fp8", 64)])
def test_one_tile_over_many_keys(kv, fmt, D):
    """A few queries on a long prefix: one tile of rows, its steps cut over many workers and by parity."""
    T = 40
    b = Batch(kv, fmt, 2, 4, D, [(0, T, 40003, 0)] + [(i, 1, 5, 1) for i in range(T)], T, seed=7)
    b.check(*b.run())


@pytest.mark.parametrize("fmt,D", [("bf16", 128), ("fp8", 128), ("fp16", 64), ("fp8", 64)])
def test_tiles_scales_and_values_that_are_not_finite(kv, fmt, D):
    """The tile kernel: negative and zero scales, a length that ends inside a block, and a NaN or an infinity in a
    token that every query sees."""
    import torch
    T, n = 200, 1001
    b = Batch(kv, fmt, 2, 4, D, [(0, T, n, 0)], T, seed=17)
    for scale in (None, -0.3, 0.0):
        b.check(*b.run(scale=scale), scale=scale)
    k, v = b.k.clone(), b.v.clone()
    v[b.slots_of[0][1000], 0, 5] = math.nan
    v[b.slots_of[0][7], 1, 6] = math.inf
    b.cache.write(k, v, torch.arange(k.shape[0], device="cuda"))
    out, _ = b.run()
    if fmt == "fp8":  # a row with a NaN is NaN whole; an infinity is held as a large number
        assert torch.isnan(out[:, :4]).all() and torch.isfinite(out[:, 4:]).all()
    else:
        assert torch.isnan(out[:, :4, 5]).all() and torch.isposinf(out[:, 4:, 6]).all()
        keep = torch.ones(D, dtype=torch.bool, device="cuda")
        keep[[5, 6]] = False
        assert torch.isfinite(out[:, :, keep]).all()
    k[b.slots_of[0][300], 1] = math.nan
    b.cache.write(k, v, torch.arange(k.shape[0], device="cuda"))
    assert torch.isnan(b.run()[0][:, 4:]).all()


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_back_to_back_calls(kv, fmt):
    """Calls queued one behind the other, with the queries, cached tokens and the plan changed in between: each gives
    what it gives alone."""
    import torch
    T = 60
    spans = [(0, T, 700, 0)] + [(i, 1, 30 + i, 1) for i in range(T)]
    b = Batch(kv, fmt, 2, 8, 128, spans, T, seed=23)
    gen = torch.Generator(device="cuda").manual_seed(4)
    n = 25
    qs = torch.randn(n, *b.q.shape, device="cuda", generator=gen).to(b.q.dtype)
    sl = b.slots_of[0][:200].contiguous()
    ks = torch.randn(n, 200, 2, 128, device="cuda", generator=gen).to(b.q.dtype)
    lens = [700 if i % 3 else 512 for i in range(n)]
    q = torch.empty_like(b.q)

    def step(i):
        q.copy_(qs[i])
        b.cache.write(ks[i], ks[i], sl)
        b.plan.set(T, [(0, T, lens[i], 0, 0)] + b.spans[1:], b.ids)
        return b.cache.attend(q, b.plan), b.cache.attend(q, b.plan, scale=0.05)

    torch.cuda.synchronize()
    got = [step(i) for i in range(n)]
    b.cache.check()
    for i in range(n):
        torch.cuda.synchronize()
        want = step(i)
        torch.cuda.synchronize()
        assert torch.equal(got[i][0], want[0]) and torch.equal(got[i][1], want[1])


@pytest.mark.parametrize("fmt,D", [("bf16", 128), ("fp8", 128), ("fp16", 64)])
def test_many_tiles_per_worker(kv, fmt, D):
    """Each worker of the tile kernel has several pieces, whose queries and results pass through the same memory, its
    warps at different pieces."""
    import random
    rng = random.Random(5)
    spans, first = [], 0
    for _ in range(30):
        n = rng.choice([64, 64, 33, 50])
        spans.append((first, n, rng.choice([300, 450, 640]), 0))
        first += n
    b = Batch(kv, fmt, 8, 8, D, spans, first, seed=31)
    out, lse = b.run()
    b.check(out, lse)
    for _ in range(10):
        import torch
        assert torch.equal(b.run()[0], out)
