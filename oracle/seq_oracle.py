"""Attention over token sequences in 64 bits, with the bounds that rounding puts on a computation of it (include/seq.h).

Test infrastructure: plain numpy, one batch item and head at a time.  ``attention`` returns, next to each result, how far a
computation may be from it that rounds the weights and their gradients once to a type of unit roundoff ``u`` (half a step) where they enter a
product, and the result once, and that carries ``e`` of relative error in everything it holds in fp32:

A result is off by u of itself, or where the type has no smaller step (fp16 below 2^-14: multiples of 2^-24) by half of that step, `tiny` / 2.

  out = sum P v        each P off by (u + e) P and by `tiny` (the type's smallest step)     (u + e) sum P |v| + tiny sum |v| + u |out|
  delta = <dout, out>  out off by u |out| and the products by e                             d_delta = (u + e) sum |dout| |out|
  dS = P (dP - delta)  t = |P| (|dP| + |delta|), rounded                                    u |dS| + e t' + P d_delta, e t' with sum |dout| |v| in place of |dP|
"""
from __future__ import annotations

import numpy as np

INF = float("inf")


def visible(Lq, Lk, causal=False, window=None, documents=None, prefix=None):
    """bool [Lq, Lk] of one batch item."""
    pos = np.arange(Lq) + Lk - Lq
    far = pos[:, None] - np.arange(Lk)[None]
    see = np.ones_like(far, dtype=bool)
    if causal:
        see &= far >= 0
    if window is not None:
        see &= np.abs(far) < window
    if prefix is not None:
        see |= prefix.astype(bool)[None]
    if documents is not None:
        mine = np.where(pos >= 0, documents[np.maximum(pos, 0)], -1)
        see &= (mine[:, None] == documents[None]) & (documents >= 0)[None]
    return see


def head(q, k, v, dout, see, *, scale, softcap=None, slope=0.0, u=0.0, e=0.0, tiny=0.0):
    """One head: q [Lq, D], k and v [Lk, D], dout [Lq, D] or None, see [Lq, Lk] -> dict of results and dict of bounds."""
    Lq, Lk = see.shape
    live_q, live_k = see.any(1), see.any(0)
    q, k, v = (np.where(alive[:, None], x, 0.0) for x, alive in ((q, live_q), (k, live_k), (v, live_k)))   # the rest may be anything
    raw = scale * (q @ k.T)
    t = np.tanh(raw / softcap) if softcap else None
    s = softcap * t if softcap else raw
    far = np.abs(np.arange(Lq)[:, None] + Lk - Lq - np.arange(Lk)[None])
    s = np.where(see, s - slope * far, -INF)
    m = np.where(live_q, s.max(1, initial=-INF), 0.0)
    p = np.exp(s - m[:, None])
    total = p.sum(1)
    p = p / np.where(total == 0, 1.0, total)[:, None]
    out = p @ v
    with np.errstate(divide="ignore"):
        lse = np.where(live_q, m + np.log(np.where(total == 0, 1.0, total)), -INF)
    res, bound = {"out": out, "lse": lse}, {"out": (u + e) * (p @ np.abs(v)) + tiny * (see @ np.abs(v)) + u * np.abs(out) + tiny / 2, "lse": e * (1 + np.abs(np.where(live_q, lse, 0.0)))}
    if dout is None:
        return res, bound
    dout = np.where(live_q[:, None], dout, 0.0)
    dp, delta = dout @ v.T, (dout * out).sum(1)
    through = 1 - t * t if softcap else 1.0
    ds = p * (dp - delta[:, None]) * through
    size = np.abs(dout) @ np.abs(v).T + (np.abs(dout) * np.abs(out)).sum(1)[:, None]
    off = u * np.abs(ds) + e * p * size + p * ((u + e) * (np.abs(dout) * np.abs(out)).sum(1))[:, None] + tiny * see * np.abs(dout).max(1, initial=0.0)[:, None]
    res.update(dq=scale * ds @ k, dk=scale * ds.T @ q, dv=p.T @ dout)
    bound.update(dq=abs(scale) * off @ np.abs(k), dk=abs(scale) * off.T @ np.abs(q), dv=((u + e) * p + tiny * see).T @ np.abs(dout))
    return res, bound


def attention(q, k, v, dout=None, *, causal=False, window=None, softcap=None, slopes=None, documents=None, prefix=None, scale=None, u=0.0, e=0.0, tiny=0.0):
    """q [B, heads, Lq, D], k and v [B, kv_heads, Lk, D], float64 -> (results, bounds), each a dict of out, lse, dq, dk, dv."""
    B, heads, Lq, D = q.shape
    kv, Lk = k.shape[1:3]
    scale = D ** -0.5 if scale is None else scale
    names = {"out": q.shape, "lse": q.shape[:3], **({} if dout is None else {"dq": q.shape, "dk": k.shape, "dv": v.shape})}
    res, bound = ({n: np.zeros(s) for n, s in names.items()} for _ in range(2))
    for b in range(B):
        see = visible(Lq, Lk, causal, window, None if documents is None else documents[b], None if prefix is None else prefix[b])
        for h in range(heads):
            g = h // (heads // kv)
            r, o = head(q[b, h], k[b, g], v[b, g], None if dout is None else dout[b, h], see, scale=scale, softcap=softcap,
                        slope=0.0 if slopes is None else float(slopes[h]), u=u, e=e, tiny=tiny)
            for n in names:
                at = (b, g) if n in ("dk", "dv") else (b, h)
                res[n][at] += r[n]
                bound[n][at] += o[n]
    for n in ("dq", "dk", "dv"):
        if n in names:
            bound[n] += u * np.abs(res[n]) + tiny / 2
    return res, bound


# ---- the cache ---------------------------------------------------------------------------------------------------------

def append(cells, scales, x, table, lengths, counts=None):
    """cells int8 [pages, kv, page, D], scales float32 [pages, kv], x float32 [B, kv, n, D]: both with the new tokens, in the
    fp32 steps of the definition (include/seq.h), a page at a time."""
    cells, scales, page = cells.copy(), scales.copy(), cells.shape[2]
    pages, f32 = cells.shape[0], np.float32
    for b, L in enumerate(lengths):
        n = x.shape[2] if counts is None else min(int(counts[b]), x.shape[2])
        for at in range(L // page, (L + n - 1) // page + 1) if n > 0 and L >= 0 else ():
            lo, hi = max(L, at * page), min(L + n, (at + 1) * page)
            if at >= table.shape[1] or not 0 <= table[b, at] < pages:
                continue
            i, old = table[b, at], lo - at * page
            new = np.nan_to_num(x[b, :, lo - L:hi - L].astype(f32), nan=0.0, posinf=np.finfo(f32).max, neginf=np.finfo(f32).min)
            for h in range(cells.shape[1]):
                before = scales[i, h] if old else f32(0)
                scale = max(before, np.abs(new[h]).max() / f32(127))
                by = scale if scale > 0 else f32(1)
                if old and scale != before:
                    cells[i, h, :old] = np.rint(cells[i, h, :old].astype(f32) * (before / by))
                cells[i, h, old:old + hi - lo] = np.clip(np.rint(new[h] / by), -127, 127)
                scales[i, h] = scale
    return cells, scales


def gather(cells, scales, table, lengths, first, n):
    """[B, kv, n, D] float64."""
    pages, kv, page, D = cells.shape
    out = np.zeros((len(lengths), kv, n, D))
    for b, L in enumerate(lengths):
        for i in range(n):
            t = int(first[b]) + i
            if 0 <= t < L and t // page < table.shape[1] and 0 <= table[b, t // page] < pages:
                p = table[b, t // page]
                out[b, :, i] = cells[p, :, t % page].astype(np.float64) * scales[p].astype(np.float64)[:, None]
    return out


def present(pages, page, table, L):
    """bool [L]: which positions of a sequence lie in a page that is one."""
    return np.array([t // page < len(table) and 0 <= table[t // page] < pages for t in range(L)], dtype=bool)
