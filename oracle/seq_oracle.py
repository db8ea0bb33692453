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


def head(q, k, v, dout, see, *, scale, softcap=None, slope=0.0, u=0.0, e=0.0, tiny=0.0, far=None):
    """One head: q [Lq, D], k and v [Lk, D], dout [Lq, D] or None, see [Lq, Lk], far [Lq, Lk] (None: of tokens in a row) -> dict of results and dict of bounds."""
    Lq, Lk = see.shape
    live_q, live_k = see.any(1), see.any(0)
    q, k, v = (np.where(alive[:, None], x, 0.0) for x, alive in ((q, live_q), (k, live_k), (v, live_k)))   # the rest may be anything
    raw = scale * (q @ k.T)
    t = np.tanh(raw / softcap) if softcap else None
    s = softcap * t if softcap else raw
    far = np.abs(np.arange(Lq)[:, None] + Lk - Lq - np.arange(Lk)[None]) if far is None else far
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
                scale = max(abs(before), np.abs(new[h]).max() / f32(127))
                by = scale if scale > 0 else f32(1)
                if old and scale != before:
                    cells[i, h, :old] = np.rint(np.minimum(cells[i, h, :old].astype(f32) * (before / by), f32(127)))
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


# ---- rotation by position ----------------------------------------------------------------------------------------------

def angles(positions, freqs, sections):
    """[..., L, pairs] of positions [..., axes, L]."""
    axis = np.repeat(np.arange(len(sections)), sections)
    return np.swapaxes(np.asarray(positions, np.float64)[..., axis, :], -1, -2) * np.asarray(freqs, np.float64)


def _pairs(pairs, interleaved):
    at = np.arange(pairs)
    return (2 * at, 2 * at + 1) if interleaved else (at, at + pairs)


def turn(x, a, interleaved, back=False):
    """x [..., L, D] turned by the angles a [..., L, pairs], and sum of the magnitudes that each channel is made of."""
    c, s = np.cos(a), -np.sin(a) if back else np.sin(a)
    lo, hi = _pairs(a.shape[-1], interleaved)
    z, size = x.copy(), np.abs(x)
    z[..., lo], z[..., hi] = x[..., lo] * c - x[..., hi] * s, x[..., hi] * c + x[..., lo] * s
    size[..., lo] = size[..., hi] = np.abs(x[..., lo]) + np.abs(x[..., hi])
    return z, size


def rotary(x, positions, freqs, sections, weight=None, eps=1e-6, interleaved=False, dz=None, u=0.0, tiny=0.0):
    """x [B, heads, L, D]; positions [axes, L] or [B, axes, L] -> (results, bounds): z and, with dz, dx and dw.

    Held in fp32: the mean of D <= 128 squares in a chain of at most 20 sums (10 2^-24 of its root), the root and its reciprocal (2^-22), three products (3 2^-24); a cosine by 2^-22 (its
    angle in turns, below a half, rounded to fp32; the function's own last digit), the products and their sum (2 2^-24).  In all below 2^-19 of the channels of a pair.  Backward: the
    same, the mean of products, and their difference: 2^-18 of the magnitudes that come in.  dw: a chain of at most 400 sums."""
    e = 2.0 ** -19
    a = angles(positions, freqs, sections)
    a = a if a.ndim == 2 else a[:, None]
    D = x.shape[-1]
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps) if weight is not None else 1.0
    w = 1.0 if weight is None else weight
    z, size = turn(x * r * w, a, interleaved)
    res, bound = {"z": z}, {"z": u * np.abs(z) + e * size + tiny / 2}
    if dz is not None:
        dy, size = turn(dz, a, interleaved, back=True)
        if weight is None:
            res["dx"], off = dy, e * size
        else:
            g, xr = w * dy, x * r
            res["dx"] = r * (g - xr * (g * xr).mean(-1, keepdims=True))
            size = size * np.abs(w)
            off = 2 * e * r * (size + np.abs(xr) * (size * np.abs(xr)).mean(-1, keepdims=True))
            res["dw"] = (dy * xr).sum((0, 1, 2))
            bound["dw"] = u * np.abs(res["dw"]) + (2 * e + 400 * 2.0 ** -24) * (size / np.abs(w) * np.abs(xr)).sum((0, 1, 2)) + tiny / 2
        bound["dx"] = u * np.abs(res["dx"]) + off + tiny / 2
    return res, bound


# ---- a tree of drafted tokens ------------------------------------------------------------------------------------------

def depths(parents):
    """Nodes above each node; -1: no node."""
    out = []
    for i, p in enumerate(parents):
        out.append(0 if p == -1 else out[p] + 1 if 0 <= p < i and out[p] >= 0 else -1)
    return out


def tree(q, k, v, parents, there, L, window=None):
    """What the nodes of one sequence see of its L tokens and of themselves: see [n, L + n] and far.  there: bool [L], tokens whose page is one."""
    n, depth = len(parents), depths(parents)
    see = np.zeros((n, L + n), dtype=bool)
    for i in range(n):
        if depth[i] >= 0:
            see[i, :L] = there
            at = i
            while at >= 0:
                see[i, L + at] = True
                at = parents[at]
    stands = L + np.array(depth)
    far = stands[:, None] - np.concatenate([np.arange(L), stands])[None]
    return see & (far < (window or L + n + 1)), np.maximum(far, 0)


def _probabilities(logits, temperature):
    x = np.where(np.isnan(logits), -INF, np.minimum(logits, np.finfo(np.float32).max))
    if x.max() == -INF:
        return np.zeros_like(x)
    if not temperature > 0:
        p = np.zeros_like(x)
        p[x.argmax()] = 1
        return p
    p = np.zeros_like(x)
    some = x > -INF
    p[some] = np.exp((x[some] - x.max()) / temperature)
    return p / p.sum()


def _drawn(p, u):
    """-1: p gives none."""
    sums = np.cumsum(p)
    some = np.flatnonzero(p > 0)
    if len(some) == 0:
        return -1
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    passed = some[sums[some] > u * sums[-1]]
    return int(passed[0] if len(passed) else some[-1])


def verify(logits, tokens, uniforms, parents=None, draft=None, temperature=1.0):
    """One sequence: logits [n, V], tokens [n], uniforms [n] (with draft [n - 1, V]: [n + 1]) -> (path, next)."""
    n, V = logits.shape
    number = lambda u: min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    if draft is None:
        node, path = 0, [0]
        while True:
            token = _drawn(_probabilities(logits[node], temperature), uniforms[node])
            child = [c for c in range(node + 1, n) if (c - 1 if parents is None else parents[c]) == node and tokens[c] == token and token >= 0]
            if not child:
                return path, token
            node = child[0]
            path.append(node)
    for i in range(n):
        p, path = _probabilities(logits[i], temperature), list(range(i + 1))
        if i == n - 1 or not 0 <= tokens[i + 1] < V:
            return path, _drawn(p, uniforms[n])
        if not temperature > 0:
            if p[tokens[i + 1]] != 1:
                return path, _drawn(p, 0.0)
            continue
        q = _probabilities(draft[i], temperature)
        if not number(uniforms[i]) * q[tokens[i + 1]] < p[tokens[i + 1]]:
            rest = np.maximum(p - q, 0)
            return path, _drawn(rest if rest.sum() > 0 else p, uniforms[n])
