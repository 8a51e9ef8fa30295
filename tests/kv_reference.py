"""Plain 64-bit forms of the serving operators, for the tests: what the cache holds of a row, and attention
of spans, with elementwise error bounds of the kernels' arithmetic."""
import math

import torch

TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.bfloat16}


def held(fmt, x):
    """The values the cache holds of rows x [..., D], as float64 (a row with a NaN: NaN whole, fp8 only)."""
    if fmt != "fp8":
        return x.to(TORCH[fmt]).double()
    big = torch.finfo(torch.float32).max
    y = x.double().clamp(-big, big)
    nan = torch.isnan(y).any(-1, keepdim=True)
    y = torch.where(torch.isnan(y), 0.0, y)
    amax = y.abs().amax(-1, keepdim=True)
    e = torch.full_like(amax, -110.0)
    for k in range(-110, 119):  # the smallest e with amax <= 448 * 2^e
        e = torch.where(amax > 448.0 * 2.0 ** k, k + 1.0, e)
    s = torch.exp2(e)
    u = (y / s).clamp(-448.0, 448.0)
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.where(nan, math.nan, torch.round(u / step) * step * s)  # torch.round: ties to even


def attend(q, k, v, spans, slots_of, scale):
    """q [T, Hq, D]; k, v [slots, Hkv, D] float64 cached values; spans (first, n, length, causal, ...);
    slots_of[i]: the slots of span i's tokens.  Returns out, lse, and A = sum p |v| / sum p (for the bounds), the
    largest sum |q||k| of a row's scores, and the number of keys a row sees."""
    T, Hq, D = q.shape
    g = Hq // k.shape[1]
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=q.device)
    A = torch.zeros_like(out)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    mag = torch.zeros((T, Hq), dtype=torch.float64, device=q.device)
    cnt = torch.zeros(T, dtype=torch.int64)
    for t in range(T):
        sel = []
        for (f, n, length, causal, *_), sl in zip(spans, slots_of):
            if f <= t < f + n:
                m = length - n + (t - f) + 1 if causal else length
                sel.append(sl[:max(0, m)])
        sel = torch.cat(sel) if sel else torch.zeros(0, dtype=torch.int64, device=q.device)
        cnt[t] = sel.numel()
        if not sel.numel():
            continue
        K, V = (x[sel].repeat_interleave(g, 1).transpose(0, 1) for x in (k, v))  # [Hq, L, D]
        x = q[t].double()
        z = torch.einsum("hd,hld->hl", x, K) * scale
        m = z.amax(-1, keepdim=True)
        w = torch.exp(z - m)
        l = w.sum(-1, keepdim=True)
        out[t] = torch.einsum("hl,hld->hd", w, V) / l
        A[t] = torch.einsum("hl,hld->hd", w, V.abs()) / l
        lse[t] = (m + torch.log(l))[:, 0]
        mag[t] = torch.einsum("hd,hld->hl", x.abs(), K.abs()).amax(-1) * abs(scale)
    return out, lse, A, mag, cnt.to(q.device)


def bounds(fmt, D, out, A, mag, cnt, vmax):
    """Elementwise bounds.  Scores are sums of D exact products in 32 bits: off by at most (D + 3) 2^-24 mag, which moves
    every probability by that relative amount; ex2, scale factors and the sums add less than 2^-18.  A probability and
    the output are each rounded once to 8 (bf16) or 11 bits (fp16); fp16 probabilities below 2^-14 are off by up to 2^-25
    of a sum that is at least 1."""
    u = 2.0 ** -11 if fmt == "fp16" else 2.0 ** -8  # 2^-p of p significant bits
    # a last-bit tie may fall to the other side of the output's rounding: the slack of the bracket covers it
    z = (D + 3) * 2.0 ** -24 * mag
    tol = u * out.abs() * (1 + 2 * u) + (u + 2.0 ** -18 + 2 * z)[..., None] * A
    if fmt == "fp16":
        tol = tol + (cnt * 2.0 ** -25 * vmax)[:, None, None] + 2.0 ** -25
    tol_lse = z + 2.0 ** -18 + 2.0 ** -22 * mag
    return tol, tol_lse
