"""Cases of a step with drafted tokens on the paged key/value cache, and of copies inside and between caches.

An instance that drafts tokens ahead builds a tree of candidates per request, gives every node the position of its depth,
rotates the nodes' queries and keys by their positions and writes the keys and values into the cache's 16-token blocks,
attends from every node to the request's context and the node's ancestors, and moves the rows of the accepted nodes to
where the context goes on.  Blocks are copied where a request is forked or handed to another cache, and cleared where
they are given back.

Kinds of cases:
- "rotate": `tokens` new tokens with `q_heads` queries: queries and keys are rotated by their positions (`dims` elements
  of the head, pairs interleaved or half a head apart, frequencies scaled for long contexts), keys and values written
  into the cache, and what the cache now holds for them is read back;
- "mask":   `requests` trees of up to `nodes` nodes, given by their parents: masks of ancestors, and positions;
- "tree":   attention of `requests` trees of `nodes_lo` to `nodes` nodes, all on a shared prefix of `shared` tokens, each
  on a context of `own_lo` to `own_hi` tokens of its own;
- "move":   the drafted tokens of `requests` trees of `nodes` nodes are written, up to `depth` accepted ones of each are
  moved to the front, and all of them read back;
- "copy":   `count` blocks are copied (within a cache, or from another one), a share `cleared` of them cleared, and read
  back.
"""
import math
import random

import torch

own = False

BLOCK = 16  # tokens of a cache block
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EXP_MIN, EXP_MAX, EXP_NAN = -110, 119, 255  # exponents that a row's scale can have; the mark of a row with a NaN
ORIGINAL, LOW, HIGH, FACTOR = 8192, 1.0, 4.0, 8.0  # long contexts: the trained one, rotations in it, and the extension

_CACHE = dict(kv_heads=8, head_dim=128, fmt="bf16", src="bf16", lengths=1)
_ROTATE = dict(_CACHE, kind="rotate", tokens=1, q_heads=64, dims=128, interleaved=False, base=500000.0, scaling="rotations",
               far=131072, blocks=4096)
_MASK = dict(kind="mask", requests=1, nodes=16, width=8, padded=False)
_TREE = dict(_CACHE, kind="tree", q_heads=64, requests=1, shared=0, own_lo=1, own_hi=512, nodes_lo=1, nodes=16, width=8)
_MOVE = dict(_CACHE, kind="move", requests=1, nodes=16, depth=8, blocks=4096)
_COPY = dict(_CACHE, kind="copy", count=1, cleared=0.0, between=False, blocks=64)


def listed():
    return [
        # one request decodes: its newest token's queries and key
        dict(_ROTATE, name="rotate_1_fp8", fmt="fp8"),
        # a prefill chunk of an engine that computes in 32 bits; small heads, a part of each rotated, pairs interleaved
        dict(_ROTATE, name="rotate_2047_part_fp16", tokens=2047, kv_heads=4, q_heads=28, head_dim=64, dims=32,
             interleaved=True, base=10000.0, scaling="linear", src="fp32", fmt="fp16"),
        # the prefills of a whole arrival window (a 64 Ki-token budget) into an 8-bit cache
        dict(_ROTATE, name="rotate_65536_fp8", tokens=65536, fmt="fp8", blocks=8192),
        # one request's draft
        dict(_MASK, name="mask_1x24", nodes=24),
        # a full batch's drafts, some of which ended early
        dict(_MASK, name="mask_256x200", requests=256, nodes=200, width=25, padded=True),
        # one request verifies its draft alone: latency
        dict(_TREE, name="tree_1x16_on_4096_bf16", own_lo=4096, own_hi=4096, nodes_lo=16),
        # a batch of sessions with contexts of their own
        dict(_TREE, name="tree_32x64_on_5000_bf16", requests=32, own_lo=3000, own_hi=5000, nodes_lo=40, nodes=64, lengths=2),
        # an agent fleet verifies drafts on a shared prompt, 8-bit cache
        dict(_TREE, name="tree_60x31_share_16384_fp8", requests=60, shared=16384, own_hi=700, nodes=31, fmt="fp8", lengths=3),
        # one request's accepted tokens
        dict(_MOVE, name="move_1x16_fp8", fmt="fp8"),
        # a batch's
        dict(_MOVE, name="move_64x60_bf16", requests=64, nodes=60, depth=7),
        # eight requests are forked at their open blocks
        dict(_COPY, name="copy_8_bf16", count=8),
        # a long chain is handed to another cache, 8-bit
        dict(_COPY, name="copy_8192_fp8", count=8192, between=True, cleared=0.05, fmt="fp8", blocks=9000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "mask", "tree", "tree", "tree", "move", "copy"])
    if kind == "mask":
        nodes = _log(rng, 1, 300)
        return dict(_MASK, requests=_log(rng, 1, max(1, 30000 // nodes)), nodes=nodes, width=rng.randint(1, max(1, nodes // 3)),
                    padded=rng.random() < 0.5)
    D = rng.choice([64, 128])
    fmt = rng.choice(["bf16", "fp8", "fp8", "fp16"])
    kv = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 3, 4, 5, 7, 8, 16])
    while kv * group > 64:
        group = max(1, group // 2)
    c = dict(kind=kind, kv_heads=kv, head_dim=D, fmt=fmt, src="fp16" if fmt == "fp16" else "bf16", lengths=rng.randint(0, 1 << 20))
    if kind == "rotate":
        src = rng.choice([c["src"], "fp32"])
        tokens = _log(rng, 1, 40000 if src == "fp32" else 65536)
        return dict(_ROTATE, **c | dict(tokens=tokens, q_heads=kv * group, dims=16 * rng.randint(1, D // 16),
                    interleaved=rng.random() < 0.5, base=rng.choice([10000.0, 500000.0]),
                    scaling=rng.choice(["none", "linear", "rotations"]), far=_log(rng, 2, 10000000),
                    src=src, blocks=-(-tokens // BLOCK) + rng.randint(1, 4096)))
    if kind == "move":
        nodes = rng.randint(2, 100)
        requests = _log(rng, 1, 40)
        return dict(_MOVE, **c | dict(requests=requests, nodes=nodes, depth=rng.randint(1, min(nodes, 12)),
                    blocks=requests * (nodes // BLOCK + 2) + rng.randint(1, 2000)))
    if kind == "copy":
        count = _log(rng, 1, 4096)
        return dict(_COPY, **c | dict(count=count, cleared=rng.choice([0.0, 0.2]), between=rng.random() < 0.5,
                    blocks=2 * count + rng.randint(1, 100)))
    nodes = _log(rng, 1, 120)
    requests = _log(rng, 1, 60)
    while requests * nodes > 2000:
        requests = max(1, requests // 2)
    hi = _log(rng, 1, max(2, min(30000, 120000 // requests)))
    return dict(_TREE, **c | dict(q_heads=kv * group, requests=requests, nodes_lo=max(1, nodes // rng.choice([1, 2, 4])),
                nodes=nodes, width=rng.randint(1, max(1, nodes // 2)), shared=rng.choice([0, 0, _log(rng, 16, 8000)]),
                own_lo=hi // rng.choice([1, 2, 50]), own_hi=hi))


# ---- sizes ---------------------------------------------------------------------------------------------------

def _held_bytes(case):
    """Bytes of a token's K and V in one head of the cache."""
    return 2 * case["head_dim"] + 2 if case["fmt"] == "fp8" else 4 * case["head_dim"]


def _sizes(case):
    """[(own context, nodes) per request] of a tree case."""
    rng = random.Random(case["lengths"])
    return [(rng.randint(case["own_lo"], case["own_hi"]), rng.randint(case["nodes_lo"], case["nodes"]))
            for _ in range(case["requests"])]


def _parents(gen, sizes, width):
    """Parents of trees in order of depth: node i's lies about `width` nodes before it (-1: a root)."""
    dev = gen.device
    i = torch.cat([torch.arange(n, device=dev) for n in sizes])
    u = torch.rand(i.numel(), generator=gen, device=dev)
    return torch.clamp(i - 1 - (u * 2 * width).long(), min=-1).to(torch.int32)


def work(case):
    kind = case["kind"]
    if kind == "mask":
        T = case["requests"] * case["nodes"]
        return {"bytes": T * (4 + 4 * -(-case["nodes"] // 32) + 8) + 8 * case["requests"], "flops": T}
    D, H, held = case["head_dim"], case["kv_heads"], _held_bytes(case)
    if kind == "rotate":
        T, src = case["tokens"], DTYPES[case["src"]].itemsize
        return {"bytes": T * (case["q_heads"] * D * (src + 2) + H * (2 * D * src + 2 * held + 4 * D) + 16),
                "flops": 3 * T * (case["q_heads"] + H) * case["dims"]}
    if kind == "move":
        T, m = case["requests"] * case["nodes"], case["requests"] * case["depth"]
        return {"bytes": H * (T * (2 * D * DTYPES[case["src"]].itemsize + 2 * held + 4 * D) + 2 * m * held) + 8 * T + 16 * m,
                "flops": T * H * D}
    if kind == "copy":
        T = case["count"] * BLOCK
        return {"bytes": T * H * (3 * held + 4 * D) + 16 * case["count"], "flops": T * H * D}
    sizes = _sizes(case)
    T = sum(n for _, n in sizes)
    keys = case["shared"] + sum(o + n for o, n in sizes)
    # a node has about i / width ancestors before it
    pairs = sum(n * (case["shared"] + o) + sum(1 + i // case["width"] for i in range(n)) for o, n in sizes)
    return {"bytes": keys * H * held + 2 * T * case["q_heads"] * D * 2 + T * -(-case["nodes"] // 32) * 4,
            "flops": 4 * D * case["q_heads"] * pairs}


# ---- inputs --------------------------------------------------------------------------------------------------

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _rows(gen, tokens, heads, D, dtype, parts=2):
    """Rows as a fused projection leaves them: side by side in one tensor, some channels far larger than others."""
    x = torch.randn(tokens, parts, heads, D, generator=gen, device=gen.device)
    x[:, 0, :, ::29] *= 5.0
    x *= torch.exp2(torch.randint(-2, 3, (tokens, 1, heads, 1), generator=gen, device=gen.device).float()) ** 0.5
    return x.to(dtype).unbind(1)


def _inputs(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    kind = case["kind"]
    if kind == "mask":
        B, n = case["requests"], case["nodes"]
        parents = _parents(gen, [n] * B, case["width"]).reshape(B, n)
        if case["padded"]:  # trees that ended early
            size = torch.randint(1, n + 1, (B, 1), generator=gen, device=dev)
            parents = torch.where(torch.arange(n, device=dev) < size, parents, -2).to(torch.int32)
        return dict(parents=parents, start=torch.randint(0, 131072, (B,), generator=gen, device=dev))
    D, H = case["head_dim"], case["kv_heads"]
    dtype = DTYPES[case["src"]]
    spread = torch.arange(BLOCK, device=dev)

    def some(n):  # slots of n blocks
        return (torch.randperm(case["blocks"], generator=gen, device=dev)[:n, None] * BLOCK + spread).reshape(-1)

    if kind == "rotate":
        T = case["tokens"]
        k, v = _rows(gen, T, H, D, dtype)
        q, = _rows(gen, T, case["q_heads"], D, dtype, 1)
        # prompts of up to 4096 tokens, each somewhere in its context
        first = torch.randint(0, case["far"], (-(-T // 4096),), generator=gen, device=dev)
        t = torch.arange(T, device=dev)
        return dict(q=q, k=k, v=v, slots=some(-(-T // BLOCK))[:T].contiguous(), positions=first[t // 4096] + t % 4096)
    if kind == "move":
        B, n, depth = case["requests"], case["nodes"], case["depth"]
        per = n // BLOCK + 1
        k, v = _rows(gen, B * n, H, D, dtype)
        slots = some(B * per).reshape(B, per * BLOCK)[:, :n].contiguous()
        # the accepted nodes in order of depth, padded to `depth` with -1
        path = torch.rand(B, n, generator=gen, device=dev).argsort(1)[:, :depth].sort(1).values
        took = torch.randint(0, depth + 1, (B, 1), generator=gen, device=dev)
        live = torch.arange(depth, device=dev) < took
        src = torch.where(live, slots.gather(1, path), -1).reshape(-1)
        dst = torch.where(live, slots[:, :depth], -1).reshape(-1)
        return dict(k=k, v=v, slots=slots.reshape(-1), src=src, dst=dst, path=path, live=live)
    if kind == "copy":
        n = case["count"]
        perm = torch.randperm(case["blocks"], generator=gen, device=dev)
        here, dst = perm[:n], perm[-n:].contiguous()
        clear = torch.rand(n, generator=gen, device=dev) < case["cleared"]
        k, v = _rows(gen, n * BLOCK, H, D, dtype)
        return dict(k=k, v=v, from_slots=(here[:, None] * BLOCK + spread).reshape(-1), clear=clear, dst=dst,
                    src=torch.where(clear, -1, here), slots=(dst[:, None] * BLOCK + spread).reshape(-1))
    sizes = _sizes(case)
    T = sum(n for _, n in sizes)
    # spans: (first query, queries, tokens, kind: 0 all see all of it, 2 the last tokens are the queries' own, masked)
    first, spans = 0, [(0, T, case["shared"], 0)] if case["shared"] else []
    for o, n in sizes:
        spans.append((first, n, o + n, 2))
        first += n
    need = [-(-s[2] // BLOCK) for s in spans]
    total = sum(need)
    blocks = total + 37
    ids = torch.randperm(blocks, generator=gen, device=dev)[:total]
    k, v = _rows(gen, total * BLOCK, H, D, dtype)
    q = (torch.randn(T, case["q_heads"], D, generator=gen, device=dev) * 0.6).to(dtype)
    return dict(k=k, v=v, q=q, slots=(ids[:, None] * BLOCK + spread).reshape(-1), ids=ids, spans=spans, need=need,
                blocks=blocks, T=T, sizes=[n for _, n in sizes], parents=_parents(gen, [n for _, n in sizes], case["width"]))


# ---- plain form ----------------------------------------------------------------------------------------------

def _quantise(x):
    """e4m3 codes and scale exponents (biased by 127) of rows [..., D]."""
    x = x.float()
    big = torch.finfo(torch.float32).max
    amax = x.nan_to_num(0.0, big, -big).abs().amax(-1)
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (m > 0.875).int(), EXP_MIN).clamp(EXP_MIN, EXP_MAX)
    code = torch.ldexp(x, -e[..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return code, torch.where(x.isnan().any(-1), EXP_NAN, e + 127).to(torch.uint8)


def _value(code, exp):
    e = exp.int()
    x = torch.ldexp(code.float(), (e - 127)[..., None])
    return torch.where((e == EXP_NAN)[..., None], math.nan, x)


def _plain_cache(case, blocks, dev):
    """Rows of all slots and one more, which takes what is skipped."""
    shape = (blocks * BLOCK + 1, case["kv_heads"], case["head_dim"])
    if case["fmt"] == "fp8":
        return [torch.zeros(shape, dtype=torch.uint8, device=dev), torch.zeros(shape[:2], dtype=torch.uint8, device=dev)]
    return [torch.zeros(shape, dtype=DTYPES[case["fmt"]], device=dev)]


def _plain_write(cache, x, slots):
    if len(cache) == 2:
        code, exp = _quantise(x)
        cache[0][slots] = code.view(torch.uint8)
        cache[1][slots] = exp
    else:
        cache[0][slots] = x.to(cache[0].dtype)


def _plain_read(cache, slots):
    """The cached rows at `slots`, in 32 bits."""
    if len(cache) == 2:
        return _value(cache[0][slots].view(torch.float8_e4m3fn), cache[1][slots])
    return cache[0][slots].float()


def _frequencies(case, dev):
    i = torch.arange(0, case["dims"], 2, dtype=torch.float64, device=dev)
    f = case["base"] ** (-i / case["dims"])
    if case["scaling"] == "linear":
        return f / FACTOR
    if case["scaling"] == "rotations":
        w = ((ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        return f * (w + (1 - w) / FACTOR)
    return f


def _plain_rotate(case, x, angle):
    """Rows [T, heads, D] rotated by the angles [T, pairs], in 32 bits."""
    x, R = x.float(), case["dims"]
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if case["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((y, x[..., R:]), -1)


def _plain_mask(parents, start):
    """Masks of ancestors [B * n, words] and positions [B * n] of trees [B, n], by doubling the length of paths."""
    B, n = parents.shape
    p = parents.long()
    real = p >= -1
    one = torch.arange(n, device=p.device)
    path = ((p[..., None] == one) | (one[:, None] == one)).float()
    for _ in range((n - 1).bit_length()):
        path = (path @ path).clamp(max=1.0)
    seen = (path > 0) & real[..., None]
    depth = torch.where(real, seen.sum(-1) - 1, 0)
    words = -(-n // 32)
    bits = torch.nn.functional.pad(seen, (0, words * 32 - n)).reshape(B * n, words, 32).long()
    word = (bits << torch.arange(32, device=p.device)).sum(-1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32), (start[:, None] + depth).reshape(-1)


def _level(q, s, seen):
    """One level of spans: q [T, H, g, D]; each span has its queries' rows and its tokens, both padded to the level's
    longest.  Returns the running maximum, sum and weighted values of every query."""
    rows, tok, mask = seen  # [N, Q], [N, L], [N, Q, L]
    k, v = (_plain_read(c, tok) for c in (s["kc"], s["vc"]))  # [N, L, H, D]
    z = torch.einsum("nqhgd,nlhd->nhgql", q[rows], k).mul_(s["scale"])
    z.masked_fill_(~mask[:, None, None], -math.inf)
    m = z.amax(-1)
    z = z.sub_(m.clamp(min=-1e30)[..., None]).exp_()
    l = z.sum(-1)
    a = torch.einsum("nhgql,nlhd->nqhgd", z, v)
    live = mask.any(-1)  # padded rows see nothing
    at = rows[live]
    M = torch.full(q.shape[:3], -math.inf, device=q.device)
    S = torch.zeros(q.shape[:3], device=q.device)
    A = torch.zeros(q.shape, device=q.device)
    M[at], S[at], A[at] = m.permute(0, 3, 1, 2)[live], l.permute(0, 3, 1, 2)[live], a[live]
    return M, S, A


def _plain_attend(s):
    case, q = s["case"], s["q"]
    H = case["kv_heads"]
    x = q.float().reshape(q.shape[0], H, q.shape[1] // H, -1)
    M, S, A = (torch.stack(t) for t in zip(*[_level(x, s, seen) for seen in s["levels"]]))
    w = (M - M.amax(0).clamp(min=-1e30)).exp()
    S, A = (w * S).sum(0), (w[..., None] * A).sum(0)
    return torch.where(S[..., None] > 0, A / S[..., None], 0.0).reshape(q.shape).to(q.dtype)


def _plain_levels(inp):
    """The spans by level (those of a level cover different queries), padded: rows, tokens and masks."""
    dev = inp["slots"].device
    at, starts = 0, []
    for n in inp["need"]:
        starts.append(at * BLOCK)
        at += n
    N = max(inp["sizes"])
    par = torch.full((len(inp["sizes"]), N), -2, device=dev)
    par[torch.arange(N, device=dev) < torch.tensor(inp["sizes"], device=dev)[:, None]] = inp["parents"].long()
    i = torch.arange(N, device=dev)
    path = ((par[..., None] == i) | (i[:, None] == i)).float()
    for _ in range((N - 1).bit_length()):
        path = (path @ path).clamp(max=1.0)
    out = []
    for kind in (0, 2):
        spans = [(f, n, length, start) for (f, n, length, c), start in zip(inp["spans"], starts) if c == kind]
        if not spans:
            continue
        f, n, length, start = (torch.tensor(c, device=dev)[:, None] for c in zip(*spans))
        qi, kj = torch.arange(int(n.max()), device=dev), torch.arange(int(length.max()), device=dev)
        rows = (f + qi).clamp(max=inp["T"] - 1)
        tok = inp["slots"][(start + torch.minimum(kj, length - 1))]
        mask = (kj < length)[:, None] & (qi < n)[..., None]  # [N, Q, L]
        if kind == 2:
            j = kj - (length - n)  # the own token's number
            tree = path.gather(2, j.clamp(0, N - 1)[:, None].expand(-1, N, -1)) > 0
            mask = mask & ((j < 0)[:, None] | tree)
        out.append((rows, tok, mask))
    return out


# ---- states and passes ---------------------------------------------------------------------------------------

def prepare(case, seed):
    inp = _inputs(case, seed)
    kind = case["kind"]
    if kind == "mask":
        s = dict(case=case, **inp)
        if own:
            from paper_2609_33224_gb300 import kvcache
            s["cache"] = kvcache.KVCache(1, 1, 64)
        return s
    dev = inp["slots"].device
    s = dict(case=case, **{x: inp[x] for x in ("q", "k", "v", "slots", "positions", "src", "dst") if x in inp})
    s["out"] = torch.float16 if case["fmt"] == "fp16" else torch.bfloat16
    blocks = inp["blocks"] if kind == "tree" else case["blocks"]
    if own:
        from paper_2609_33224_gb300 import kvcache

        def cache():
            return kvcache.KVCache(blocks, case["kv_heads"], case["head_dim"], fmt=case["fmt"])

        s["cache"] = cache()
        if kind == "rotate":
            s["rotary"] = kvcache.Rotary(case["dims"], base=case["base"], interleaved=case["interleaved"],
                                         scaling=None if case["scaling"] == "none" else case["scaling"], factor=FACTOR,
                                         original=ORIGINAL, low=LOW, high=HIGH)
    else:
        s["kc"], s["vc"] = (_plain_cache(case, blocks, dev) for _ in range(2))
        if kind == "rotate":
            s["freq"] = _frequencies(case, dev)
    if kind == "copy":
        if own:
            s["source"] = cache() if case["between"] else s["cache"]
            s["source"].write(s["k"], s["v"], inp["from_slots"])
        else:
            s["ks"], s["vs"] = (_plain_cache(case, blocks, dev) if case["between"] else s[c] for c in ("kc", "vc"))
            _plain_write(s["ks"], s["k"], inp["from_slots"])
            _plain_write(s["vs"], s["v"], inp["from_slots"])
    if kind == "tree":
        if own:
            s["cache"].write(s["k"], s["v"], s["slots"])
        else:
            _plain_write(s["kc"], s["k"], s["slots"])
            _plain_write(s["vc"], s["v"], s["slots"])
        s["scale"] = case["head_dim"] ** -0.5
        if own:
            import numpy as np
            n = len(inp["spans"])
            spans, at = np.zeros(n, kvcache.SPAN_DTYPE), 0
            for i, (x, b) in enumerate(zip(inp["spans"], inp["need"])):
                spans[i] = (*x, at)
                at += b
            ids = inp["ids"].cpu().numpy().astype(np.uint32)
            s["plan"] = kvcache.AttentionPlan(s["cache"], case["q_heads"], max_queries=inp["T"], max_spans=n, max_blocks=len(ids))
            s["plan"].set(inp["T"], spans, ids, masked=True)
            offsets = torch.tensor([0] + inp["sizes"], device=dev).cumsum(0)
            s["mask"], _ = s["cache"].tree_mask(inp["parents"], offsets=offsets, max_nodes=case["nodes"])
        else:
            s["levels"] = _plain_levels(inp)
    if kind in ("tree", "copy"):
        del s["k"], s["v"]
    return s


def run(state):
    s = state
    case = s["case"]
    kind = case["kind"]
    if own:
        cache = s["cache"]
        if kind == "mask":
            return cache.tree_mask(s["parents"], start=s["start"])
        if kind == "tree":
            return cache.attend(s["q"], s["plan"], scale=s["scale"], mask=s["mask"])
        if kind == "rotate":
            q = cache.write_rotated(s["k"], s["v"], s["slots"], s["positions"], s["rotary"], q=s["q"])
            return (q, *cache.read(s["slots"], dtype=s["out"]))
        if kind == "move":
            cache.write(s["k"], s["v"], s["slots"])
            cache.move(s["src"], s["dst"])
        else:
            cache.copy_blocks(s["src"], s["dst"], source=s["source"])
        return cache.read(s["slots"], dtype=s["out"])
    if kind == "mask":
        return _plain_mask(s["parents"], s["start"])
    if kind == "tree":
        return _plain_attend(s)
    caches = (s["kc"], s["vc"])
    if kind == "rotate":
        angle = s["positions"].double()[:, None] * s["freq"]
        _plain_write(s["kc"], _plain_rotate(case, s["k"], angle), s["slots"])
        _plain_write(s["vc"], s["v"], s["slots"])
        q = _plain_rotate(case, s["q"], angle).to(s["out"])
        return (q, *(_plain_read(c, s["slots"]).to(s["out"]) for c in caches))
    if kind == "move":
        _plain_write(s["kc"], s["k"], s["slots"])
        _plain_write(s["vc"], s["v"], s["slots"])
        src, dst = s["src"], torch.where(s["dst"] < 0, case["blocks"] * BLOCK, s["dst"])
        parts = [x for c in caches for x in c]
        for x, y in zip(parts, [x[src] for x in parts]):
            x[dst] = y
    else:
        clear = s["src"] < 0
        for to, source in zip(caches, (s["ks"], s["vs"])):
            for x, y in zip(to, source):
                shape = (case["blocks"], BLOCK, *x.shape[1:])
                got = y[:-1].view(shape)[s["src"].clamp(min=0)]
                x[:-1].view(shape)[s["dst"]] = torch.where(clear.view(-1, *[1] * (len(shape) - 1)), 0, got)
    return tuple(_plain_read(c, s["slots"]).to(s["out"]) for c in caches)


# ---- 64 bits -------------------------------------------------------------------------------------------------

def _held(case, x):
    """What the cache holds for rows x [..., D], in 64 bits, from the format's definition."""
    if case["fmt"] != "fp8":
        return x.to(DTYPES[case["fmt"]]).double()
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(amax / 448.0)).clamp(EXP_MIN, EXP_MAX)
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, e)
    e = torch.where((amax <= 448.0 * torch.exp2(e - 1)) & (e > EXP_MIN), e - 1, e)
    y = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def _exact_rotation(case, x, positions):
    """Each pair as a complex number, times e^(i angle)."""
    R = case["dims"]
    freq = []
    for i in range(R // 2):
        f = math.exp(-2.0 * i / R * math.log(case["base"]))
        if case["scaling"] == "linear":
            f /= FACTOR
        elif case["scaling"] == "rotations":
            turns = ORIGINAL * f / math.tau
            keep = 0.0 if turns < LOW else 1.0 if turns > HIGH else (turns - LOW) / (HIGH - LOW)
            f = keep * f + (1.0 - keep) * f / FACTOR
        freq.append(f)
    angle = positions.double()[:, None] * torch.tensor(freq, dtype=torch.float64, device=x.device)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    y = x.double().clone()
    lo, hi = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
    z = torch.complex(y[..., lo], y[..., hi]) * turn
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


def exact(case, seed):
    kind = case["kind"]
    cpu = _device() == "cpu"
    if cpu and kind == "tree" and work(case)["flops"] > 2e10 or cpu and kind != "tree" and work(case)["bytes"] > 1e8:
        return None
    inp = _inputs(case, seed)
    if kind == "mask":
        parents, start = inp["parents"].tolist(), inp["start"].tolist()
        words = -(-case["nodes"] // 32)
        masks, positions = [], []
        for tree, first in zip(parents, start):
            rows = []
            for i, p in enumerate(tree):
                m, depth = (0, 0) if p < -1 else (1 << i, 0) if p < 0 else (rows[p][0] | 1 << i, rows[p][1] + 1)
                rows.append((m, depth))
                positions.append(first + depth)
                masks.append([((m >> 32 * w & 0xFFFFFFFF) ^ 1 << 31) - (1 << 31) for w in range(words)])
        dev = inp["start"].device
        return torch.tensor(masks, dtype=torch.int32, device=dev), torch.tensor(positions, device=dev)
    if kind == "rotate":
        q, k = (_exact_rotation(case, inp[x], inp["positions"]) for x in "qk")
        return q, _held(case, k), _held(case, inp["v"])
    if kind == "copy":
        return tuple(torch.where(inp["clear"].repeat_interleave(BLOCK)[:, None, None], 0.0, _held(case, inp[x])) for x in "kv")
    if kind == "move":
        B, n, depth = case["requests"], case["nodes"], case["depth"]
        node = torch.arange(n, device=inp["slots"].device).repeat(B, 1)
        node[:, :depth] = torch.where(inp["live"], inp["path"], node[:, :depth])
        node = (node + torch.arange(B, device=node.device)[:, None] * n).reshape(-1)
        return tuple(_held(case, inp[x])[node] for x in "kv")
    q = inp["q"]
    T, Hq, D = q.shape
    H = case["kv_heads"]
    g = Hq // H
    starts, at = [], 0
    for b in inp["need"]:
        starts.append(at * BLOCK)
        at += b
    parents = inp["parents"].tolist()
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=q.device)
    den = torch.zeros(T, Hq, dtype=torch.float64, device=q.device)
    # scores of this data stay below 600, so that exp needs no maximum in 64 bits
    for (f, n, length, kind), start in zip(inp["spans"], starts):
        seen = None
        if kind == 2:
            seen = torch.ones(n, length, dtype=torch.bool)
            base = length - n
            seen[:, base:] = False
            for i in range(n):
                j = i
                while j >= 0:
                    seen[i, base + j] = True
                    j = parents[f + j]
            seen = seen.to(q.device).repeat_interleave(g, 0)
        for a in range(0, length, 32768):
            b = min(length, a + 32768)
            k, v = (_held(case, inp[c][start + a:start + b]) for c in "kv")
            for h in range(H):
                x = q[f:f + n, h * g:(h + 1) * g].double().reshape(n * g, D)
                w = torch.exp(x @ k[:, h].T * D ** -0.5)
                if seen is not None:
                    w = torch.where(seen[:, a:b], w, 0.0)
                out[f:f + n, h * g:(h + 1) * g] += (w @ v[:, h]).reshape(n, g, D)
                den[f:f + n, h * g:(h + 1) * g] += w.sum(-1).reshape(n, g)
    return torch.where(den[..., None] > 0, out / den[..., None], 0.0)
