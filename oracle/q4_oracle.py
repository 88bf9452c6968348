"""Plain definitions of the 4-bit operators (include/coreinfer.h), NumPy: groups of 4-bit numbers, products with them,
attention over a cache of them, and eviction by accumulated weight.

Which of its sixteen values an element is held as is decided in 32 bits, as the definition says; everything after
that is float64.  Nothing here is shared with the kernels.
"""

import numpy as np


def hold(x, group):
    """x [..., n] as groups along the last axis: codes (0 .. 15), step and low spread over their groups (float64)."""
    x = np.asarray(x, dtype=np.float32)
    n = x.shape[-1]
    codes, steps, lows = np.zeros(x.shape), np.zeros(x.shape), np.zeros(x.shape)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        for a in range(0, n, group):
            part = x[..., a:a + group]
            lo, hi = part.min(-1, keepdims=True), part.max(-1, keepdims=True)   # a NaN takes them over
            step = np.minimum((hi - lo) / np.float32(15.0), np.float32(65504.0)).astype(np.float16)
            low = np.clip(lo, np.float32(-65504.0), np.float32(65504.0)).astype(np.float16)
            s32, l32 = step.astype(np.float32), low.astype(np.float32)
            code = np.clip(np.rint((part - l32) / s32), 0, 15)
            code = np.where(s32 > 0, code, 0.0)
            codes[..., a:a + group] = code
            steps[..., a:a + group] = step.astype(np.float64)
            lows[..., a:a + group] = low.astype(np.float64)
    return codes, steps, lows


def held_values(x, group):
    codes, steps, lows = hold(x, group)
    return lows + steps * codes


def silu(z):
    return z / (1.0 + np.exp(-z))


def matvec(x, w, gate=None, bias=None, act="none"):
    """x [M, C] and the held values w [R, C]."""
    y = x @ w.T
    if bias is not None:
        y = y + bias
    if act == "relu":
        return np.maximum(y, 0.0)
    return silu(x @ gate.T) * y if act == "swiglu" else y


def attend(q, k, v, lens, scale):
    """q [B, S, Hq, D]; held values k, v [B, H, T, D].  Returns out, lse [B, S, Hq] and the weight that the call adds to
    each slot [B, H, T]."""
    B, S, Hq, D = q.shape
    H, T = k.shape[1:3]
    G = Hq // H
    out, lse, weight = np.zeros(q.shape), np.full((B, S, Hq), -np.inf), np.zeros((B, H, T))
    for b in range(B):
        for s in range(S):
            seen = min(lens[b], lens[b] - S + s + 1)
            if seen <= 0:
                continue
            for i in range(Hq):
                z = scale * (k[b, i // G, :seen] @ q[b, s, i])
                top = z.max()
                e = np.exp(z - top)
                p = e / e.sum()
                out[b, s, i] = p @ v[b, i // G, :seen]
                lse[b, s, i] = top + np.log(e.sum())
                weight[b, i // G, :seen] += p
    return out, lse, weight


def evict_head(weight, pos, length, next_pos, budget, recent):
    """One head.  Returns the slot that each of the first min(length, budget) slots takes its contents from."""
    if length <= budget:
        return list(range(length))

    def order(t):
        w = float(weight[t])
        if pos[t] >= next_pos - recent:
            return (0, 0.0, t)
        return (2, 0.0, t) if w != w else (1, -w, t)
    kept = set(sorted(range(length), key=order)[:budget])
    moving = iter([t for t in sorted(kept) if t >= budget])
    return [t if t in kept else next(moving) for t in range(budget)]
