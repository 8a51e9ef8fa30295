"""A window of requests from the scheduler's decision to an instance's attention.

The scheduler assigns a window; the instance that got the most requests then does what its next steps need: it
writes the keys and values of the tokens that it did not have cached into 16-token blocks, attends from them to
the cached prefixes (each shared prefix once for all requests on it), and decodes a few tokens for the whole batch.

    python examples/instance_step.py [fp8|bf16|fp16]

Keys, values and queries are random (there is no model here); the last step is checked against 64 bits.
"""
from __future__ import annotations

import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

Q_HEADS, KV_HEADS, HEAD_DIM, STEPS = 32, 8, 128, 4


def main(fmt: str = "fp8") -> dict:
    import numpy as np
    import torch

    import paper_2609_33224_gb300 as P
    import workload as W
    from paper_2609_33224_gb300.kvcache import AttentionPlan, KVCache, shared_spans

    # ---- the scheduler's part: which instance, and how much of each prompt it has cached
    wl = W.generate(0)
    with P.scheduler_for(wl, device=0) as s:
        dec = s.schedule_window(wl.window)
    admitted = dec["path"] < 2
    inst = int(np.bincount(dec["assign"][admitted]).argmax())
    mine = np.flatnonzero(admitted & (dec["assign"] == inst))
    off, hashes = wl.window.chain_off.astype(np.int64), wl.window.chain_hash
    lengths = [int(wl.window.prompt_tokens[r]) for r in mine]

    # ---- the instance's part: a cache block per distinct block hash, one more per request for its open end
    ids: dict = {}
    tables, new = [], []
    for r, n in zip(mine, lengths):
        chain = [ids.setdefault(int(h), len(ids)) for h in hashes[off[r]:off[r + 1]]]
        hit = min(int(dec["hit_chosen"][r]), len(chain), (n - 1) // 16)  # at least the last token is computed
        new.append(n - 16 * hit)
        tables.append(chain)
    spare = iter(range(len(ids), 1 << 31))
    for t, n in zip(tables, lengths):
        t.extend(next(spare) for _ in range(-(-(n + STEPS) // 16) - len(t)))
    num_blocks = max(max(t) for t in tables) + 1

    dev = torch.device("cuda", 0)
    gen = torch.Generator(device=dev).manual_seed(1)
    dtype = torch.float16 if fmt == "fp16" else torch.bfloat16
    k_all, v_all = (torch.randn(num_blocks * 16, KV_HEADS, HEAD_DIM, device=dev, generator=gen).to(dtype) for _ in range(2))

    def slots(table, a, b):  # of a request's tokens a .. b - 1
        t = np.arange(a, b)
        return np.asarray(table, np.int64)[t // 16] * 16 + t % 16

    def write(cache, parts):
        where = torch.from_numpy(np.unique(np.concatenate(parts))).to(dev)  # requests of a window share new blocks too
        cache.write(k_all[where], v_all[where], where)

    with KVCache(num_blocks, KV_HEADS, HEAD_DIM, fmt=fmt, device=0) as cache:
        plan = AttentionPlan(cache, Q_HEADS, max_queries=sum(new), max_spans=4 * len(tables) + 1,
                             max_blocks=sum(len(t) for t in tables))
        cached = [slots(t, 0, n - q) for t, n, q in zip(tables, lengths, new)]
        if sum(c.size for c in cached):
            write(cache, cached)  # what earlier requests left
        result = {"requests": len(tables), "prefill_tokens": sum(new), "cached_tokens": sum(lengths) - sum(new)}

        # ---- prefill of what was not cached, then decode steps
        for step in range(1 + STEPS):
            if step:
                lengths, new = [n + 1 for n in lengths], [1] * len(new)
            write(cache, [slots(t, n - q, n) for t, n, q in zip(tables, lengths, new)])
            order, spans, blocks = shared_spans(tables, lengths, new)
            plan.set(sum(new), spans, blocks)
            q = torch.randn(sum(new), Q_HEADS, HEAD_DIM, device=dev, generator=gen).to(dtype)
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            out = cache.attend(q, plan)
            b.record()
            cache.check()
            result["prefill_ms" if step == 0 else "decode_ms"] = a.elapsed_time(b)
        result["spans"], result["shared"] = len(spans), int((spans["causal"] == 0).sum())

        # ---- the last decode step against 64 bits
        worst = 0.0
        for at, i in enumerate(order):
            k, v = cache.read(torch.from_numpy(slots(tables[i], 0, lengths[i])).to(dev), dtype=torch.float32)
            x = q[at].double().view(KV_HEADS, Q_HEADS // KV_HEADS, HEAD_DIM)
            w = torch.softmax(torch.einsum("hgd,lhd->hgl", x, k.double()) * HEAD_DIM ** -0.5, -1)
            want = torch.einsum("hgl,lhd->hgd", w, v.double()).reshape(Q_HEADS, HEAD_DIM)
            worst = max(worst, float((out[at].double() - want).norm() / want.norm()))
        result["error"] = worst
    return result


if __name__ == "__main__":
    r = main(*sys.argv[1:2])
    print(", ".join(f"{k} {v:.4g}" if isinstance(v, float) else f"{k} {v}" for k, v in r.items()))
