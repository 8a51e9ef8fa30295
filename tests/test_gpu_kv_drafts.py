"""Trees of drafted tokens: masks and positions from parents, and attention of masked spans against 64 bits."""
import math
import random

import numpy as np
import pytest
import torch

from tests import kv_reference as ref
from tests.test_gpu_kv_store import kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


# ---- masks and positions

def tree(rng, n, kind):
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "star":
        return [-1] + [0] * (n - 1)
    if kind == "roots":
        return [-1] * n
    p = [rng.randint(-1, i - 1) if kind == "any" else max(-1, i - 1 - rng.randint(0, 5)) for i in range(n)]
    if kind == "early":  # the last nodes are none
        end = rng.randint(0, n)
        p[end:] = [-2 - rng.randint(0, 3)] * (n - end)
    return p


def rows_of(p):
    """[(ancestors and itself, depth)] of a tree."""
    out = []
    for i, x in enumerate(p):
        out.append((set(), 0) if x < -1 else ({i}, 0) if x == -1 else (out[x][0] | {i}, out[x][1] + 1))
    return out


def bits(sets, words):
    m = np.zeros((len(sets), words), np.uint32)
    for i, s in enumerate(sets):
        for j in s:
            m[i, j // 32] |= np.uint32(1 << (j % 32))
    return torch.from_numpy(m.view(np.int32)).cuda()


@pytest.fixture(scope="module")
def cache(kv):  # noqa: F811
    with kv.KVCache(1, 1, 64) as c:
        yield c


@pytest.mark.parametrize("kind", ["chain", "star", "roots", "any", "near", "early"])
@pytest.mark.parametrize("trees,n", [(1, 1), (3, 31), (2, 32), (5, 33), (2, 64), (40, 65), (1, 257), (2, 1000)])
def test_masks_of_equal_trees(cache, kind, trees, n):
    rng = random.Random(n)
    ps = [tree(rng, n, kind) for _ in range(trees)]
    start = [rng.randrange(1 << 40) for _ in ps]
    want = [rows_of(p) for p in ps]
    mask, pos = cache.tree_mask(torch.tensor(ps, dtype=torch.int32).cuda(), start=torch.tensor(start).cuda())
    cache.check()
    assert torch.equal(mask, bits([s for w in want for s, _ in w], -(-n // 32)))
    assert pos.tolist() == [a + d for a, w in zip(start, want) for _, d in w]
    assert cache.tree_mask(torch.tensor(ps, dtype=torch.int32).cuda())[1].tolist() == [d for w in want for _, d in w]


def test_masks_of_uneven_trees(cache):
    rng = random.Random(1)
    sizes = [5, 0, 1, 70, 33, 0, 128, 2]
    ps = [tree(rng, n, "any") for n in sizes]
    off = torch.tensor(np.cumsum([0] + sizes)).cuda()
    parents = torch.tensor(sum(ps, []), dtype=torch.int32).cuda()
    mask, pos = cache.tree_mask(parents, offsets=off, max_nodes=128)
    cache.check()
    want = [r for p in ps for r in rows_of(p)]
    assert mask.shape == (sum(sizes), 4) and torch.equal(mask, bits([s for s, _ in want], 4))
    assert pos.tolist() == [d for _, d in want]
    # rows of no tree
    mask, pos = cache.tree_mask(parents, offsets=off[3:5].contiguous(), max_nodes=128)
    assert not mask[:6].any() and not mask[76:].any() and not pos[76:].any() and mask[6:76].any(1).all()
    for shape in ((0, 5), (3, 0)):
        mask, pos = cache.tree_mask(torch.zeros(shape, dtype=torch.int32, device="cuda"))
        assert mask.shape == (0, 1) and pos.shape == (0,)
    mask, _ = cache.tree_mask(torch.arange(-1, 8191, dtype=torch.int32, device="cuda")[None])
    assert mask.shape == (8192, 256) and (mask[-1] == -1).all() and mask[0, 0] == 1 and not mask[0, 1:].any()
    cache.check()


def test_wrong_trees_are_reported(cache):
    import paper_2609_33224_gb300 as P
    ok = [-1, 0, 1, 0]

    def reported(call):
        call()
        with pytest.raises(P.PSError, match="parent"):
            cache.check()
        cache.check()

    t = lambda rows: torch.tensor(rows, dtype=torch.int32, device="cuda")  # noqa: E731
    for bad in ([0, 0, 1, 0], [-1, 2, 1, 0], [-1, 0, 1, 1 << 30], [-2, 0, 1, 0]):
        reported(lambda: cache.tree_mask(t([ok, bad])))
    for off in ([0, 2, 9], [0, 3, 2], [-1, 2, 4], [0, 1 << 60, 4]):
        reported(lambda: cache.tree_mask(t(ok), offsets=torch.tensor(off).cuda(), max_nodes=4))
    reported(lambda: cache.tree_mask(t([-1] * 33), offsets=torch.tensor([0, 33]).cuda(), max_nodes=20))
    # the other trees' rows are right
    mask, pos = cache.tree_mask(t([ok, [3, 0, 1, 0], ok]))
    assert mask[:4, 0].tolist() == mask[8:, 0].tolist() == [1, 3, 7, 9] and pos[8:].tolist() == [0, 1, 2, 1]
    with pytest.raises(P.PSError, match="parent"):
        cache.check()
    for bad in (dict(parents=t(ok)), dict(parents=t([ok]).long()), dict(parents=t([ok]).cpu()), dict(parents=t([ok] * 4).T),
                dict(parents=t(ok), offsets=torch.tensor([0, 4]).cuda()), dict(parents=t([ok]), start=torch.zeros(2).long().cuda()),
                dict(parents=t(ok), offsets=torch.tensor([0, 4]).cuda(), max_nodes=8193),
                dict(parents=t(ok), offsets=torch.zeros(0, dtype=torch.int64, device="cuda"), max_nodes=4)):
        with pytest.raises(ValueError):
            cache.tree_mask(**bad)


def test_captured_masks(cache):
    """A replay reads the parents' memory anew; on another stream, beside calls on this one."""
    parents = torch.empty(6, 100, dtype=torch.int32, device="cuda")
    start = torch.arange(6, device="cuda") * 1000
    rng = random.Random(3)
    trees = [torch.tensor([tree(rng, 100, k) for _ in range(6)], dtype=torch.int32).cuda() for k in ("any", "near", "early", "chain")]
    want = [cache.tree_mask(t, start=start) for t in trees]
    parents.copy_(trees[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mask, pos = cache.tree_mask(parents, start=start)
    s = torch.cuda.Stream()
    for i in (1, 0, 3, 2):
        parents.copy_(trees[i])
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            graph.replay()
        other = cache.tree_mask(trees[3 - i], start=start)
        torch.cuda.synchronize()
        assert torch.equal(mask, want[i][0]) and torch.equal(pos, want[i][1])
        assert torch.equal(other[0], want[3 - i][0]) and torch.equal(other[1], want[3 - i][1])
    cache.check()


# ---- attention

class Drafts:
    """A cache filled at random with the tokens of spans (first, queries, length, kind), and masks of the queries: sees[t],
    the own tokens that query t sees.  Unused slots hold NaNs and infinities."""

    def __init__(self, kv, fmt, Hkv, g, D, spans, T, sees, seed=0, words=None, cache=None, qscale=1.0):  # noqa: F811
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.kv, self.fmt, self.T, self.D, self.Hq, self.sees = kv, fmt, T, D, Hkv * g, sees
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
        free = torch.ones(blocks * 16, dtype=torch.bool, device="cuda")
        for s in self.slots_of:
            free[s] = False
        self.k[free] = math.nan
        self.v[free] = torch.where(torch.rand(int(free.sum()), Hkv, D, device="cuda", generator=gen) < 0.5, math.inf, math.nan).to(dt)
        self.cache = kv.KVCache(blocks, Hkv, D, fmt=fmt)
        self.write()
        most = max([s[1] for s in spans if s[3] == 2], default=0)
        self.mask = bits(sees, words or max(1, -(-most // 32)))
        # bits that are not to be looked at
        for first, n, _, kind in spans:
            if kind == 2 and n % 32:
                self.mask[first:first + n, n // 32] |= -1 << (n % 32)
                self.mask[first:first + n, n // 32 + 1:] = -1
        self.plan = kv.AttentionPlan(self.cache, self.Hq, max(T, 1), max(len(spans), 1), max(total, 1))
        self.plan.set(T, self.spans, ids, masked=True)

    def write(self):
        self.cache.write(self.k, self.v, torch.arange(self.k.shape[0], device="cuda"))

    def run(self, **kw):
        lse = torch.full((self.T, self.Hq), 77.0, device="cuda")
        out = self.cache.attend(self.q, self.plan, lse=lse, **{"mask": self.mask, **kw})
        self.cache.check()
        return out, lse

    def seen(self, t):
        """The slots that query t sees."""
        got = [torch.zeros(0, dtype=torch.int64, device="cuda")]
        for (f, n, length, kind, *_), sl in zip(self.spans, self.slots_of):
            if not f <= t < f + n:
                continue
            if kind == 2:
                got += [sl[:length - n], sl[sorted(length - n + j for j in self.sees[t])]]
            else:
                got.append(sl[:max(0, length - n + t - f + 1) if kind else length])
        return torch.cat(got)

    def expected(self, scale=None):
        """Output, logarithms, their bounds, and which queries see nothing."""
        scale = self.D ** -0.5 if scale is None else scale
        k, v = ref.held(self.fmt, self.k), ref.held(self.fmt, self.v)
        slots = [self.seen(t) for t in range(self.T)]
        want, wl, A, mag, cnt = ref.attend(self.q, k, v, [(t, 1, s.numel(), 0) for t, s in enumerate(slots)], slots, scale)
        vmax = max((v[s].abs().max().item() for s in slots if s.numel()), default=0.0)
        return (want, wl, *ref.bounds(self.fmt, self.D, want, A, mag, cnt, vmax), cnt == 0)

    def check(self, out, lse, scale=None):
        want, wl, tol, tl, none = self.expected(scale)
        assert not out[none].any() and torch.isneginf(lse[none]).all()
        assert torch.isfinite(out).all()
        over = (out.double() - want).abs() / tol.clamp(min=1e-30)
        assert over.max() <= 1.0 if over.numel() else True, over.max().item()
        d = ((lse.double() - wl).abs() / tl)[~none]
        assert d.max() <= 1.0 if d.numel() else True, d.max().item()


def batch(sizes, shared=0, kind="near", seed=0):
    """(T, spans, sees) of requests (context, nodes), all on a shared prefix."""
    rng = random.Random(seed)
    T = sum(n for _, n in sizes)
    spans, sees, first = [(0, T, shared, 0)] if shared else [], [], 0
    for own, n in sizes:
        spans.append((first, n, own + n, 2))
        first += n
        if kind == "mask":  # any at all: some see nothing, some what comes after them
            sees += [set(rng.sample(range(n), rng.choice([0, rng.randint(0, n)]))) for _ in range(n)]
        else:
            sees += [s for s, _ in rows_of(tree(rng, n, kind))]
    return T, spans, sees


LAYOUTS = {
    "one": lambda: batch([(1000, 1)]),
    "draft": lambda: batch([(333, 16)]),
    # no context: a root sees itself alone, a node of "early" nothing
    "bare": lambda: batch([(0, 7), (0, 1), (0, 33)]),
    "bare_any": lambda: batch([(0, 40), (0, 3)], kind="mask"),
    "early": lambda: batch([(0, 20), (17, 20), (0, 64)], kind="early", seed=1),
    # around the block and word sizes
    "edges": lambda: batch([(15, 1), (16, 16), (17, 31), (31, 32), (1, 33), (40, 17)]),
    "mask": lambda: batch([(100, 65), (3, 129)], kind="mask"),
    "shared": lambda: batch([(rng, 1 + rng % 9) for rng in (0, 5, 16, 100, 7, 33)], shared=500, kind="any"),
    "wide": lambda: batch([(2500, 150)], shared=700, kind="any"),
    "chain": lambda: batch([(300, 100), (0, 50)], kind="chain"),
}


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("fmt,Hkv,g,D", [("bf16", 2, 8, 128), ("fp8", 2, 8, 128), ("fp16", 3, 1, 64), ("bf16", 1, 5, 64),
                                         ("fp8", 1, 16, 64), ("fp8", 1, 21, 128), ("fp16", 2, 4, 128)])
def test_against_64_bits(kv, layout, fmt, Hkv, g, D):  # noqa: F811
    T, spans, sees = LAYOUTS[layout]()
    d = Drafts(kv, fmt, Hkv, g, D, spans, T, sees, seed=len(layout) + g)
    d.check(*d.run())
    d.cache.close()


@pytest.mark.parametrize("fmt,D", [("bf16", 128), ("fp8", 128), ("fp16", 64), ("fp8", 64)])
def test_many_rows_and_long_contexts(kv, fmt, D):  # noqa: F811
    """Contexts that the tile kernel takes, of lengths that end anywhere in a block, with scales of either sign."""
    T, spans, sees = batch([(3000, 40), (2049, 64), (1500 + 15, 33), (16 * 90, 64)], kind="any", seed=3)
    d = Drafts(kv, fmt, 4, 8, D, spans, T, sees, seed=11, qscale=2.0)
    for scale in (None, -0.1, 0.0):
        d.check(*d.run(scale=scale), scale=scale)
    d.cache.close()


@pytest.mark.parametrize("fmt,Hkv,g,D", [("bf16", 1, 8, 128), ("fp8", 2, 2, 128), ("fp16", 1, 4, 64)])
@pytest.mark.parametrize("n", [256, 257, 600])
def test_large_drafts(kv, fmt, Hkv, g, D, n):  # noqa: F811
    """As many own tokens as the tile kernel takes, and more, over several of its steps."""
    for own in (0, 777):
        T, spans, sees = batch([(own, n), (1500, 3)], kind="mask" if own else "any", seed=n)
        d = Drafts(kv, fmt, Hkv, g, D, spans, T, sees, seed=n + own)
        d.check(*d.run())
        d.cache.close()


@pytest.mark.parametrize("fmt,D", [("bf16", 128), ("fp8", 128), ("fp16", 64)])
@pytest.mark.parametrize("shared,own", [(600, 40), (9000, 700)])
def test_many_rows_to_join(kv, fmt, D, shared, own):  # noqa: F811
    """More than 16384 rows with a few parts each; some queries see nothing at all."""
    T, spans, sees = batch([(own, 29)] * 9 + [(0, 3)], kind="any", seed=12)
    T2 = T + 2
    spans = [(0, T - 3, shared, 0)] + spans
    d = Drafts(kv, fmt, 8, 8, D, spans, T2, sees[:-3] + [set(), {0}, set()] + [set()] * 2, seed=13)
    d.check(*d.run())
    d.cache.close()


@pytest.mark.parametrize("fmt,D,g", [("bf16", 128, 16), ("fp8", 128, 16), ("fp16", 128, 8), ("fp16", 64, 8), ("fp8", 64, 8)])
def test_many_small_drafts(kv, fmt, D, g):  # noqa: F811
    """Several pieces of one tile of rows a worker of the tile kernel, of uneven lengths, two at a time; then with values of
    drafted tokens that are not finite, which reach the queries that see them and no other."""
    rng = random.Random(6)
    T, spans, sees = batch([(rng.choice([130, 300, 700, 1000]) + rng.randrange(40), rng.randrange(8, 16)) for _ in range(30)],
                           kind="any", seed=14)
    d = Drafts(kv, fmt, 8, g, D, spans, T, sees, seed=16)
    out, lse = d.run()
    d.check(out, lse)
    for _ in range(5):
        assert torch.equal(d.run()[0], out)
    hit = torch.zeros(T, dtype=torch.bool, device="cuda")
    for (f, n, length, kind, _), sl in zip(d.spans, d.slots_of):
        for j in rng.sample(range(n), 2):
            d.v[sl[length - n + j], :, rng.randrange(D)] = math.nan
            hit |= torch.tensor([f <= t < f + n and j in sees[t] for t in range(T)], device="cuda")
    d.write()
    bad, _ = d.run()
    assert torch.isnan(bad).any(-1).all(-1)[hit].all()
    want, _, tol, _, _ = d.expected()
    assert ((bad.double() - want).abs() <= tol)[~hit].all()
    d.cache.close()


def test_mixed_with_causal_spans(kv):  # noqa: F811
    """A batch of prefills, single tokens and drafts."""
    T, spans, sees = batch([(70, 20), (9, 40)], kind="any", seed=4)
    more = [(T, 30, 100, 1), (T + 30, 1, 55, 1), (T + 31, 3, 2, 1)]
    spans = [(0, T + 34, 333, 0)] + spans + more
    for fmt, D, g in (("bf16", 128, 8), ("fp8", 64, 3)):
        d = Drafts(kv, fmt, 2, g, D, spans, T + 34, sees + [set()] * 34, seed=5)
        d.check(*d.run())
        d.cache.close()


@pytest.mark.parametrize("seed", range(16))
def test_random_batches(kv, seed):  # noqa: F811
    rng = random.Random(seed)
    D, fmt = rng.choice([64, 128]), rng.choice(["bf16", "fp16", "fp8"])
    Hkv, g = rng.choice([1, 2, 3]), rng.choice([1, 2, 4, 5, 8, 16])
    sizes = [(rng.choice([0, 1, 16, rng.randrange(2000)]), rng.choice([1, rng.randrange(1, 70)])) for _ in range(rng.randint(1, 8))]
    T, spans, sees = batch(sizes, rng.choice([0, 37, 1200, 5000]), rng.choice(["any", "near", "mask", "early"]), seed)
    d = Drafts(kv, fmt, Hkv, g, D, spans, T, sees, seed=100 + seed, words=rng.choice([None, 5]))
    d.check(*d.run())
    d.cache.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("D,g,own", [(64, 4, 9), (128, 8, 9), (128, 8, 2000), (64, 16, 1500)])
def test_tokens_that_are_not_finite(kv, fmt, D, g, own):  # noqa: F811
    """A NaN or an infinity in a drafted token's key or value reaches the queries that see it and no other."""
    n = 40
    rng = random.Random(2)
    sees = [s for s, _ in rows_of(tree(rng, n, "near"))]
    d = Drafts(kv, fmt, 1, g, D, [(0, n, 100, 0), (0, n, own + n, 2)], n, sees, seed=5)
    clean, _ = d.run()
    want, _, tol, _, _ = d.expected()
    nodes = [5, 9, 12, 39]
    sl = d.slots_of[1]
    d.v[sl[own + 5], 0, 7] = math.nan
    d.v[sl[own + 9], 0, 9] = math.inf
    d.v[sl[own + 39]] = -math.inf
    d.k[sl[own + 12]] = math.nan
    d.write()
    out, _ = d.run()
    sees_one = lambda x: torch.tensor([x in s for s in sees], device="cuda")  # noqa: E731
    touched = torch.zeros(n, dtype=torch.bool, device="cuda")
    for x in nodes:
        touched |= sees_one(x)
    # What sees none of them is as it was; in fp8, where an infinity is a large number whose scale is far from the others',
    # the probabilities of the rows beside it may be rounded to 8 bits instead of 11, which the bounds allow for.
    if fmt == "fp8":
        assert ((out.double() - want).abs() <= tol)[~touched].all()
    else:
        assert torch.equal(out[~touched], clean[~touched])
    assert torch.isnan(out[sees_one(12)]).all()
    five = sees_one(5) & ~sees_one(12)
    if fmt == "fp8":  # (an infinity is held as 448 * 2^119, of which a sum in 32 bits, with weights up to 2^8, may be one)
        assert torch.isnan(out[five]).all() and not torch.isnan(out[~sees_one(12) & ~sees_one(5)]).any()
    else:
        assert torch.isnan(out[five][..., 7]).all()
        only = five & ~sees_one(9) & ~sees_one(39)
        keep = torch.arange(D, device="cuda") != 7
        assert torch.isfinite(out[only][..., keep]).all()
        only = sees_one(9) & ~five & ~sees_one(12) & ~sees_one(39)
        assert torch.isposinf(out[only][..., 9]).all() and torch.isfinite(out[only][..., torch.arange(D, device="cuda") != 9]).all()
        only = sees_one(39) & ~five & ~sees_one(12) & ~sees_one(9)
        assert torch.isneginf(out[only]).all()
    d.cache.close()


@pytest.mark.parametrize("n,own", [(200, 3000), (2500, 333)])
@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_a_chain_is_a_causal_span(kv, fmt, n, own):  # noqa: F811
    """A tree that is a chain sees what a causal span of the same tokens sees."""
    D = 64
    sees = [set()] * n
    d = Drafts(kv, fmt, 1, 2, D, [(0, n, own + n, 2)], n, sees, seed=15)
    mask, pos = d.cache.tree_mask(torch.arange(-1, n - 1, dtype=torch.int32, device="cuda")[None])
    assert torch.equal(pos, torch.arange(n, device="cuda"))
    out, lse = d.run(mask=mask)
    causal = kv.AttentionPlan(d.cache, d.Hq, n, 1, len(d.ids))
    causal.set(n, [(0, n, own + n, 1, 0)], d.ids)
    lse2 = torch.empty_like(lse)
    want = d.cache.attend(d.q, causal, lse=lse2)
    d.cache.check()
    # either is off by its own rounding and its probabilities', 2^-8 of the largest value each; scores are off by
    # (D + 3) 2^-24 of sum |q| |k|, which the same fp32 products and sums bound by 2^-14 here
    vmax = ref.held(fmt, d.v)[d.slots_of[0]].abs().max()
    assert (out.double() - want.double()).abs().max() <= 4 * 2.0 ** -8 * 1.05 * vmax
    assert (lse - lse2).abs().max() <= 2.0 ** -12
    d.cache.close()


def test_one_plan_on_two_streams(kv):  # noqa: F811
    T, spans, sees = batch([(900, 50), (2000, 64), (10, 9)], shared=300, kind="any", seed=21)
    d = Drafts(kv, "fp8", 2, 8, 128, spans, T, sees, seed=22)
    masks = [d.mask, torch.randint(-(1 << 31), 1 << 31, d.mask.shape, device="cuda").int()]
    want = [d.cache.attend(d.q, d.plan, mask=m) for m in masks]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(d.cache.attend(d.q, d.plan, mask=masks[i]))
    torch.cuda.synchronize()
    d.cache.check()
    for i in range(2):
        for x in got[i]:
            assert torch.equal(x, want[i])
    d.cache.close()


def test_strided_masks(kv):  # noqa: F811
    T, spans, sees = batch([(50, 40), (20, 7)], kind="mask", seed=6)
    d = Drafts(kv, "bf16", 2, 4, 128, spans, T, sees, seed=7)
    out, _ = d.run()
    wide = torch.full((T, 9), -1, dtype=torch.int32, device="cuda")
    wide[:, 3:3 + d.mask.shape[1]] = d.mask
    assert torch.equal(d.run(mask=wide[:, 3:3 + d.mask.shape[1]])[0], out)
    assert torch.equal(d.run(mask=wide[:, 3:])[0], out)
    # one row for all
    one = d.mask[:1].expand(T, -1)
    assert torch.equal(d.run(mask=one)[0], d.run(mask=one.contiguous())[0])
    d.cache.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_captured_with_masks_that_change(kv, fmt):  # noqa: F811
    """A replayed graph reads the mask's memory anew; eager calls of another plan go on beside it on another stream."""
    T, spans, sees = batch([(2000, 50), (300, 64)], shared=200, kind="any", seed=8)
    d = Drafts(kv, fmt, 2, 8, 128, spans, T, sees, seed=9)
    other = kv.AttentionPlan(d.cache, d.Hq, T, len(spans), len(d.ids))
    other.set(T, d.spans, d.ids, masked=True)
    mask, out = d.mask.clone(), torch.empty_like(d.q)
    d.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.cache.attend(d.q, d.plan, out=out, mask=mask)
    masks = [d.mask, torch.randint(-(1 << 31), 1 << 31, mask.shape, device="cuda").int(), torch.zeros_like(mask)]
    want = [d.cache.attend(d.q, other, mask=m) for m in masks]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    for i in (0, 1, 2, 1, 0):
        mask.copy_(masks[i])
        with torch.cuda.stream(s):
            beside = [d.cache.attend(d.q, other, mask=masks[(i + 1) % 3]) for _ in range(3)]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
        for x in beside:
            assert torch.equal(x, want[(i + 1) % 3])
    d.cache.check()


def test_a_draft_step(kv):  # noqa: F811
    """The calls as they are used together: masks and positions, rotated writes, attention, and the accepted path's rows to
    the front, which then is what writing that path alone gives."""
    rng = random.Random(4)
    H, g, D, fmt = 2, 4, 128, "fp8"
    gen = torch.Generator(device="cuda").manual_seed(1)
    context, nodes = [5, 37, 100], [33, 9, 20]  # in the order that shared_spans gives them
    ps = [tree(rng, n, "near") for n in nodes]
    T = sum(nodes)
    tables = [list(range(10 * i, 10 * i + 10)) for i in range(3)]
    rand = lambda n, h: torch.randn(n, h, D, device="cuda", generator=gen).bfloat16()  # noqa: E731
    slot = lambda i, a, b: torch.tensor([tables[i][t // 16] * 16 + t % 16 for t in range(a, b)], dtype=torch.int64).cuda()  # noqa: E731
    rotary = kv.Rotary(D)
    with kv.KVCache(30, H, D, fmt=fmt) as c, kv.KVCache(30, H, D, fmt=fmt) as alone:
        for i, n in enumerate(context):
            k, v = rand(n, H), rand(n, H)
            for x in (c, alone):
                x.write_rotated(k, v, slot(i, 0, n), torch.arange(n, device="cuda"), rotary)
        # one step of the drafted trees
        parents = torch.tensor(sum(ps, []), dtype=torch.int32).cuda()
        mask, pos = c.tree_mask(parents, torch.tensor(np.cumsum([0] + nodes)).cuda(), max(nodes), torch.tensor(context).cuda())
        slots = torch.cat([slot(i, a, a + n) for i, (a, n) in enumerate(zip(context, nodes))])
        q, k, v = rand(T, H * g), rand(T, H), rand(T, H)
        turned = c.write_rotated(k, v, slots, pos, rotary, q=q)
        order, spans, blocks = kv.shared_spans(tables, [a + n for a, n in zip(context, nodes)], nodes, masked=True)
        plan = kv.AttentionPlan(c, H * g, T, 8, 64)
        plan.set(T, spans, blocks, masked=True)
        assert list(order) == [0, 1, 2]
        out = c.attend(turned, plan, mask=mask)
        # a path of each tree, written alone and attended to causally, gives the same
        src, dst, path = [], [], []
        first = np.cumsum([0] + nodes)
        for i, p in enumerate(ps):
            j, way = max(range(nodes[i]), key=lambda x: rows_of(p)[x][1]), []
            while j >= 0:
                way.insert(0, j)
                j = p[j]
            path.append(way)
            src += [int(slots[first[i] + j]) for j in way]
            dst += slot(i, context[i], context[i] + len(way)).tolist()
        at = torch.tensor([first[i] + j for i, way in enumerate(path) for j in way]).cuda()
        to = torch.tensor(dst).cuda()
        again = alone.write_rotated(k[at], v[at], to, pos[at], rotary, q=q[at])
        assert torch.equal(again, turned[at])
        c.move(torch.tensor(src).cuda(), to)
        for x, y in zip(c.read(to), alone.read(to)):
            assert torch.equal(x, y)
        n = [len(w) for w in path]
        order, spans, blocks = kv.shared_spans(tables, [a + b for a, b in zip(context, n)], n)
        other = kv.AttentionPlan(alone, H * g, sum(n), 8, 64)
        other.set(sum(n), spans, blocks)
        want = alone.attend(again, other)
        # the same keys and values; each result is off by at most 2^-8 of itself (its rounding) and by 2^-8 of the largest
        # value (a probability's rounding, sums of weights 1)
        vmax = v.abs().max().double()
        assert (out[at].double() - want.double()).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -7) * 1.1 * vmax
        # a fork of the last request at an open block
        c.copy_blocks(torch.tensor([tables[2][6]]).cuda(), torch.tensor([9]).cuda())
        for x, y in zip(c.read(slot(2, 96, 112)), c.read(torch.arange(9 * 16, 10 * 16, device="cuda"))):
            assert torch.equal(x, y)
        c.check()
        alone.check()


def test_refusals(kv):  # noqa: F811
    import paper_2609_33224_gb300 as P
    with kv.KVCache(8, 2, 128) as c:
        p = kv.AttentionPlan(c, 4, 40, 4, 8)
        q = torch.zeros(40, 4, 128, device="cuda", dtype=torch.bfloat16)
        with pytest.raises(P.PSError, match="0 or 1"):
            p.set(4, [(0, 4, 5, 2, 0)], [0])
        with pytest.raises(P.PSError, match="0, 1 or 2"):
            p.set(4, [(0, 4, 5, 3, 0)], [0], masked=True)
        with pytest.raises(P.PSError, match="its queries' tokens"):
            p.set(4, [(0, 4, 3, 2, 0)], [0], masked=True)
        p.set(40, [(0, 4, 50, 0, 0), (0, 40, 60, 2, 4)], range(8), masked=True)
        ok = torch.zeros(40, 2, dtype=torch.int32, device="cuda")
        with pytest.raises(ValueError, match="needs a mask"):
            c.attend(q, p)
        for bad in (ok[:39], ok[:, :1], ok.long(), ok.cpu(), ok[None], ok.T.contiguous().T):
            with pytest.raises(ValueError):
                c.attend(q, p, mask=bad)
        c.attend(q, p, mask=ok)
        p.set(4, [(0, 4, 50, 1, 0)], range(8), masked=True)  # none of them is
        a = c.attend(q[:4], p)
        assert torch.equal(a, c.attend(q[:4], p, mask=None))
        c.check()
        L = P.lib()
        rows = P.PsKvRows(q.data_ptr(), 512, 128, 0)
        import ctypes
        at = ctypes.addressof(rows)
        p.set(40, [(0, 40, 60, 2, 4)], range(8), masked=True)
        ws = torch.empty(max(256, p.workspace_bytes), dtype=torch.uint8, device="cuda")
        args = (c._h, p._h, at, at, None, 1.0)
        assert L.ps_kv_attend(*args, ws.data_ptr(), ws.numel(), None) == 1
        for m in ((None, 2, 2), (ok.data_ptr() + 2, 2, 2), (ok.data_ptr(), 2, 1)):
            assert L.ps_kv_attend_masked(*args, *m, ws.data_ptr(), ws.numel(), None) == 1
