"""Plain definitions of rotary positions and of a cache in pages (include/coreinfer.h), NumPy float64, row by row.  Nothing here is
shared with the kernels."""

import math

import numpy as np


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original=0.0, fast=32.0, slow=1.0):
    """Radians a position of each pair."""
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        g = np.clip((original * f / (2 * math.pi) - slow) / (fast - slow), 0.0, 1.0)
        f = f * g + f / factor * (1 - g)
    return f


def rope(x, pos, f=(), style="half", scale=1.0, norm=None, eps=0.0, backward=False):
    """x [T, H, D] float64."""
    x = np.array(x, dtype=np.float64)
    if norm is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * norm
    n = len(f)
    if n == 0:
        return x
    angle = np.asarray(pos, dtype=np.float64)[:, None, None] * np.asarray(f)
    c, s = np.cos(angle) * scale, np.sin(angle) * scale * (-1.0 if backward else 1.0)
    first, second = (np.arange(n), np.arange(n) + n) if style == "half" else (2 * np.arange(n), 2 * np.arange(n) + 1)
    y = x.copy()
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    return y


def slots(first, lens):
    """(row, sentence, slot) of every packed row that belongs to a sentence."""
    for b, n in enumerate(lens):
        for i in range(first[b], first[b + 1]):
            yield i, b, n - (first[b + 1] - i)


def seen(p, length, window, sinks):
    return [t for t in range(min(length, p + 1)) if window == 0 or t > p - window or t < sinks]


def attend(q, k, v, table, first, lens, window=0, sinks=0, scale=1.0):
    """q [T, Hq, D]; k, v [pages, H, page, D].  Returns out and lse, and for error bounds the sum of p |v| and the largest
    scale sum |q| |k| of a row; NaN rows of out: not computed."""
    T, Hq, D = q.shape
    pages, H, page = k.shape[:3]
    G = Hq // H
    out, lse = np.full(q.shape, np.nan), np.full((T, Hq), np.nan)
    size, reach = np.zeros(q.shape), np.zeros((T, Hq))
    gathered = {}
    for b, n in enumerate(lens):
        at = [(table[b][t // page], t % page) for t in range(max(n, 0))]
        ok = np.array([0 <= g < pages for g, _ in at], dtype=bool)
        g = np.array([g if good else 0 for (g, _), good in zip(at, ok)], dtype=int)
        s = np.array([s for _, s in at], dtype=int)
        gathered[b] = (k[g, :, s], v[g, :, s], ok) if len(at) else (None, None, ok)
    for r, b, p in slots(first, lens):
        kk, vv, ok = gathered[b]
        t = [t for t in seen(p, lens[b], window, sinks) if ok[t]]
        out[r], lse[r] = 0.0, -np.inf
        if not t:
            continue
        for i in range(Hq):
            kt, vt = kk[t, i // G], vv[t, i // G]
            z = scale * (kt @ q[r, i])
            top = z.max()
            e = np.exp(z - top)
            w = e / e.sum()
            out[r, i] = w @ vt
            lse[r, i] = top + np.log(e.sum())
            size[r, i] = w @ np.abs(vt)
            reach[r, i] = scale * (np.abs(kt) @ np.abs(q[r, i])).max()
    return out, lse, size, reach
