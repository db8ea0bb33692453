"""Positions, drafts and their check: what the operators are timed on, their plain form in torch, and their definition in 64 bits.

Four operators of ``paper_2204_07143_amd.functional``, which a decoder with drafted tokens runs one after the other:

* ``seq_rotary``: queries and keys [B, heads, L, D] (or maps [B, heads, H, W, D]), each head's vector divided by its root mean square and times a
  weight, then rotated by its token's position; forward and backward.  Pair p of a vector (channels p and p + R / 2, or 2 p and 2 p + 1) turns by
  ``positions[axis of p] * freqs[p]``: sections say how many pairs each axis (time, height, width) has.  Channels from R on are not rotated.
* ``seq_cache_append`` with a rotation: new keys, normed and rotated on the way, and values into a cache of pages held in 8 bits.
* ``seq_cache_tree_attention``: attention of a tree of drafted tokens over a cache: a node sees the cache, its ancestors and itself, and stands at the
  cache's length plus its depth.
* ``seq_verify``: which of the drafted tokens the target's probabilities accept, from given random numbers, and the token behind them.
"""
from __future__ import annotations

import math
import random

import torch

own = False   # True: run() calls the library's operators; False: their plain form

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_EPS = 1e-6


def _rotary(name, op, B, heads, kv, L, D, dtype, sections, base=10000.0, start=0, norm=True, interleaved=False, rows=True, width=0):
    """op: "rotate" (one call) or "rotate_train" (forward and backward).  sections: pairs of each axis, "16,24,24"; one axis counts tokens from `start`, two are the rows and
    columns of a map of `width` columns, three frames, rows and columns of a video.  rows: as a projection leaves them, [B, L, heads, D]; else maps [B, heads, H, W, D]."""
    return {"name": name, "op": op, "B": B, "heads": heads, "kv": kv, "L": L, "D": D, "dtype": dtype, "sections": sections, "base": base, "start": start, "norm": norm,
            "interleaved": interleaved, "rows": rows, "width": width}


def _append(name, B, kv, n, longest, D, page, dtype, rotated, norm=True, interleaved=False, scattered=False):
    """scattered: the tokens kept are some of those given, the accepted path of a tree."""
    return {"name": name, "op": "append", "B": B, "kv": kv, "n": n, "longest": longest, "D": D, "page": page, "dtype": dtype, "rotated": rotated, "norm": norm,
            "interleaved": interleaved, "scattered": scattered}


def _tree(name, B, heads, kv, n, longest, D, page, dtype, window=0, cap=0.0, slopes=False):
    return {"name": name, "op": "tree", "B": B, "heads": heads, "kv": kv, "n": n, "longest": longest, "D": D, "page": page, "dtype": dtype, "window": window, "cap": cap,
            "slopes": slopes}


def _verify(name, op, B, n, V, dtype, greedy=0):
    """op: "verify_tree" (a tree of tokens) or "verify_drafts" (a line of tokens and the distributions they were drawn from).  greedy: one sequence in so many takes the largest logit
    (0: none)."""
    return {"name": name, "op": op, "B": B, "n": n, "V": V, "dtype": dtype, "greedy": greedy}


def listed():
    return [
        # one token each of a few sequences, between projection and cache: latency
        _rotary("rotate_tokens_bf16", "rotate", 8, 32, 8, 1, 128, "bf16", "64", start=5000),
        # a decoder's layer in training on video: frames, rows, columns
        _rotary("rotate_train_video_bf16", "rotate_train", 2, 16, 4, 8192, 128, "bf16", "16,24,24", width=32),
        # queries and keys of 56 x 56 maps before neighbourhood attention, two axes, neighbouring channels paired
        _rotary("rotate_train_maps_f16", "rotate_train", 64, 2, 2, 3136, 32, "f16", "8,8", base=100.0, interleaved=True, rows=False, width=56),
        # full precision, half of the channels rotated, far positions, a length that nothing divides
        _rotary("rotate_train_far_f32", "rotate_train", 3, 6, 2, 3137, 64, "f32", "16", base=500000.0, start=1000000, norm=False),
        # a batch of prompts into the cache, rotated on the way
        _append("append_rotated_prompts_bf16", 8, 8, 1000, 700, 128, 64, "bf16", 128),
        # one token for each of many sequences: latency
        _append("append_rotated_token_f16", 64, 4, 1, 1000, 64, 16, "f16", 64, interleaved=True),
        # a few nodes over one sequence: latency
        _tree("tree_one_f16", 1, 8, 2, 7, 1000, 64, 16, "f16"),
        # a batch of long sequences, wide trees
        _tree("tree_batch_bf16", 16, 32, 8, 48, 8000, 128, 64, "bf16"),
        # window, capped scores and distance bias, sizes that no tile divides
        _tree("tree_window_capped_bf16", 5, 12, 4, 27, 6000, 128, 32, "bf16", window=2048, cap=30.0, slopes=True),
        # one sequence's drafts: latency
        _verify("verify_drafts_one_f16", "verify_drafts", 1, 6, 32000, "f16"),
        # the trees of a batch, a large vocabulary
        _verify("verify_tree_bf16", "verify_tree", 16, 48, 131072, "bf16", greedy=5),
        # drafts of many sequences in full precision, rows that no vector divides
        _verify("verify_drafts_f32", "verify_drafts", 24, 8, 50021, "f32", greedy=7),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_ROTATED = 2 * 20 * 8192 * 128    # elements of queries and keys
_MOST_CACHED = 16 * 8 * 8000 * 128     # elements of the keys that the sequences hold
_MOST_PRODUCTS = 16 * 32 * 48 * 8000 * 128 // 2
_MOST_LOGITS = 16 * 48 * 131072


def draw(rng):
    D, kv, group = rng.choice([32, 64, 64, 128, 128]), rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 1, 2, 3, 4, 8])
    op = rng.choice(["rotate", "rotate_train", "rotate_train", "append", "append", "tree", "tree", "tree", "verify_tree", "verify_drafts", "verify_drafts"])
    if op in ("rotate", "rotate_train"):
        dtype, axes = rng.choice(["bf16", "bf16", "f16", "f16", "f32"]), rng.choice([1, 1, 2, 3])
        pairs = rng.choice([x for x in (8, 16, 32, 48, 64) if 2 * x <= D and x >= D // 4])
        cuts = [0] + sorted(rng.sample(range(1, pairs), axes - 1)) + [pairs]
        L, most = _log_uniform(rng, 1, 16384), _MOST_ROTATED // (2 if dtype == "f32" else 1) // (kv * (group + 1) * D)
        L = min(L, most)
        B = _log_uniform(rng, 1, max(1, min(64, most // L)))
        case = _rotary("", op, B, kv * group, kv, L, D, dtype, ",".join(str(b - a) for a, b in zip(cuts, cuts[1:])), rng.choice([100.0, 10000.0, 500000.0]),
                       rng.choice([0, 0, 7, _log_uniform(rng, 10, 2000000)]), rng.random() < 0.6, rng.random() < 0.4, rng.random() < 0.6, max(1, int(L ** 0.5)))
    elif op == "append":
        n, longest, page = rng.choice([1, _log_uniform(rng, 2, 1500)]), _log_uniform(rng, 24, 16000), rng.choice([16, 32, 64, 128])
        scattered = rng.random() < 0.3
        B = _log_uniform(rng, 1, max(1, min(96, 8 * 8 * 1000 * 128 // (kv * D * n), _MOST_CACHED // (kv * D * (longest + n)))))
        case = _append("", B, kv, n, longest, D, page, rng.choice(["f16", "bf16"]), D if rng.random() < 0.6 else D // 2, rng.random() < 0.6, rng.random() < 0.4, scattered)
    elif op == "tree":
        n, longest, page = rng.choice([_log_uniform(rng, 1, 64), rng.randint(2, 64)]), _log_uniform(rng, 24, 16000), rng.choice([16, 32, 64, 128])
        B = _log_uniform(rng, 1, max(1, min(64, _MOST_CACHED // (kv * D * (longest + n)), _MOST_PRODUCTS // (kv * group * n * (longest + n) * D))))
        case = _tree("", B, kv * group, kv, n, longest, D, page, rng.choice(["f16", "bf16"]), _log_uniform(rng, 16, longest) if rng.random() < 0.3 else 0,
                     rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.3)
    else:
        dtype, V, n = rng.choice(["bf16", "bf16", "f16", "f32"]), _log_uniform(rng, 100, 160000), rng.randint(1, 10) if op == "verify_drafts" else rng.randint(2, 64)
        B = _log_uniform(rng, 1, max(1, min(64, _MOST_LOGITS // 3 // (n * V))))
        case = _verify("", op, B, n, V, dtype, rng.choice([0, 0, 3]))
    del case["name"]
    return case


# ---- what the seed does not change: lengths, trees, positions ---------------------------------------------------------

def _rng(case):
    return random.Random(",".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name"))


def _lengths(case):
    rng = _rng(case)
    lengths = [max(1, int(case["longest"] * rng.uniform(0.125, 1.0))) for _ in range(case["B"])]
    lengths[0] = case["longest"]
    return lengths


def _parents(case):
    """Of every node of every sequence; node 0 is the token that the draft follows.  The last nodes of some sequences are none (-2)."""
    rng, n = _rng(case), case["n"]
    trees = []
    for b in range(case["B"]):
        nodes = n if b == 0 else rng.randint(max(1, 3 * n // 4), n)
        trees.append([-1] + [rng.randint(max(0, (i - 1) // 2 - 1), i - 1) for i in range(1, nodes)] + [-2] * (n - nodes))
    return trees


def _depths(parents):
    """Nodes above each node of one tree; -1: not a node."""
    depth = []
    for i, p in enumerate(parents):
        depth.append(0 if p == -1 else -1 if not 0 <= p < i or depth[p] < 0 else depth[p] + 1)
    return depth


def _sections(case):
    return [int(x) for x in case["sections"].split(",")]


def _positions(case):
    """[axes, L]"""
    at, width, start = torch.arange(case["L"], dtype=torch.int32), case["width"], case["start"]
    axes = len(_sections(case))
    if axes == 1:
        return (at + start)[None]
    if axes == 2:
        return torch.stack([at // width + start, at % width])
    frame = width * max(1, width // 2)
    return torch.stack([at // frame + start, at % frame // width, at % width])


def _freqs(sections, base):
    """A ladder of its own for each axis, as a user hands them in: fp32."""
    return torch.tensor([base ** (-i / x) for x in sections for i in range(x)], dtype=torch.float32)


# ---- inputs -----------------------------------------------------------------------------------------------------

def prepare(case, seed):
    """Activations of unit variance, as a projection leaves them; weights near one; caches as appends leave them, in pages that lie scattered; logits with a few
    tokens far above the others, drafts that mostly agree with them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    def heads_of(count, L):   # [B, L, heads, D] of a projection
        return normal(case["B"], L, count, case["D"]).to(dt).transpose(1, 2)

    state = {"op": case["op"], "dtype": dt}
    if case["op"] in ("rotate", "rotate_train"):
        train = case["op"] == "rotate_train"
        B, L, D, sections = case["B"], case["L"], case["D"], _sections(case)
        if case["rows"]:
            make = lambda count: heads_of(count, L)
        else:
            width = case["width"] if L % case["width"] == 0 else 1
            make = lambda count: normal(B, count, L // width, width, D).to(dt)
        weight = lambda: (1 + 0.1 * normal(D)).to(dt).requires_grad_(train) if case["norm"] else None
        q, k = make(case["heads"]), make(case["kv"])
        positions = _positions(case).cuda()
        state.update(q=q.requires_grad_(train), k=k.requires_grad_(train), q_weight=weight(), k_weight=weight(), positions=positions if case["rows"] else positions.reshape(-1, *q.shape[2:4]),
                     freqs=_freqs(sections, case["base"]).cuda(), sections=tuple(sections), interleaved=case["interleaved"])
        if train:
            state.update(dq=make(case["heads"]), dk=make(case["kv"]))
        return state
    if case["op"] in ("verify_tree", "verify_drafts"):
        return _prepare_verify(case, g, normal, state)
    lengths, page, kv, n, D = _lengths(case), case["page"], case["kv"], case["n"], case["D"]
    held = [x + (n if case["op"] == "append" else 0) for x in lengths]
    width = -(-max(held) // page)
    pages = sum(-(-x // page) for x in held) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).tolist()
    table, at = [], 0
    for x in held:
        used = -(-x // page)
        table.append(order[at:at + used] + [0] * (width - used))
        at += used
    # a page's values: normal, and its scale what the largest of them makes it (about three standard deviations)
    cells = lambda: normal(pages, kv, page, D).mul_(40.0).round_().clamp_(-127, 127).to(torch.int8)
    scales = lambda: torch.rand((pages, kv), generator=g, device="cuda").mul_(0.01).add_(0.02)
    state.update(k_pages=cells(), v_pages=cells(), k_scales=scales(), v_scales=scales(), table=torch.tensor(table, dtype=torch.int32, device="cuda"),
                 lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    if case["op"] == "append":
        given = 2 * n if case["scattered"] else n
        rows = None
        if case["scattered"]:
            rows = torch.rand((case["B"], given), generator=g, device="cuda").argsort(1)[:, :n].sort(1).values.to(torch.int32)
        # read back: the last page's worth of positions for a token, a little more than what was written for a prompt
        state.update(k=heads_of(kv, given), v=heads_of(kv, given), rows=rows, weight=(1 + 0.1 * normal(D)).to(dt) if case["norm"] else None,
                     freqs=_freqs([case["rotated"] // 2], 10000.0).cuda(), interleaved=case["interleaved"], n=n, read=n + page - 1,
                     after=torch.tensor(held, dtype=torch.int32, device="cuda"), first=torch.tensor([x - n - page + 1 for x in held], dtype=torch.int32, device="cuda"))
        return state
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / case["heads"]) for h in range(case["heads"])], device="cuda") if case["slopes"] else None
    state.update(q=heads_of(case["heads"], n), k=heads_of(kv, n), v=heads_of(kv, n), parents=torch.tensor(_parents(case), dtype=torch.int32, device="cuda"), slopes=slopes,
                 window=case["window"] or None, cap=case["cap"] or None)
    return state


def _prepare_verify(case, g, normal, state):
    B, n, V, dt = case["B"], case["n"], case["V"], state["dtype"]

    def logits(rows):
        x = normal(B, rows, V).mul_(2.0)
        likely = torch.randint(V, (B, rows, 8), generator=g, device="cuda")
        return x.scatter_(2, likely, torch.rand((B, rows, 8), generator=g, device="cuda") * 6 + 10)

    rng = _rng(case)
    temperatures = [0.0 if case["greedy"] and b % case["greedy"] == case["greedy"] - 1 else rng.uniform(0.7, 1.3) for b in range(B)]
    state.update(temperatures=torch.tensor(temperatures, dtype=torch.float32, device="cuda"), parents=None, draft=None)
    target = logits(n)
    if case["op"] == "verify_drafts":
        # the draft's logits: the target's, off by something; its tokens drawn from them
        draft = (target[:, :n - 1] + normal(B, n - 1, V) * 0.7).to(dt)
        gumbel = -torch.log(-torch.log(torch.rand(draft.shape, generator=g, device="cuda").clamp_(1e-12, 1 - 1e-7)))
        drawn = (draft.float() / state["temperatures"][:, None, None].clamp(min=1e-3) + gumbel).argmax(-1) if n > 1 else torch.zeros((B, 0), dtype=torch.long, device="cuda")
        state.update(draft=draft, tokens=torch.cat([drawn.new_zeros(B, 1), drawn], 1).to(torch.int32), uniforms=torch.rand((B, n + 1), generator=g, device="cuda"))
    else:
        # a node's children: the likeliest tokens of a draft that is near the target
        trees = _parents(case)
        ranks = [[sum(p == t[i] for p in t[:i]) for i in range(n)] for t in trees]
        best = torch.stack([(x + normal(n, V) * 0.5).topk(min(V, n), -1).indices for x in target])
        parents, rank = torch.tensor(trees, device="cuda"), torch.tensor(ranks, device="cuda")
        tokens = best[torch.arange(B, device="cuda")[:, None], parents.clamp(min=0), rank.clamp(max=best.shape[2] - 1)]
        state.update(parents=parents.to(torch.int32), tokens=tokens.to(torch.int32), uniforms=torch.rand((B, n), generator=g, device="cuda"))
    state["logits"] = target.to(dt)
    return state


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2204_07143_amd import functional as F

    if s["op"] in ("rotate", "rotate_train"):
        how = dict(sections=s["sections"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=_EPS, interleaved=s["interleaved"])
        if s["op"] == "rotate":
            with torch.no_grad():
                return F.seq_rotary(s["q"], s["k"], s["positions"], s["freqs"], **how)
        q, k = F.seq_rotary(s["q"], s["k"], s["positions"], s["freqs"], **how)
        leaves = [s[x] for x in ("q", "k", "q_weight", "k_weight") if s[x] is not None]
        return (q.detach(), k.detach(), *torch.autograd.grad((q, k), leaves, (s["dq"], s["dk"])))
    if s["op"] in ("verify_tree", "verify_drafts"):
        return F.seq_verify(s["logits"], s["tokens"], s["uniforms"], parents=s["parents"], draft=s["draft"], temperatures=s["temperatures"])
    cache = F.SeqCache(s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"])
    if s["op"] == "append":
        F.seq_cache_append(cache, s["k"], s["v"], s["table"], s["lengths"], rows=s["rows"], freqs=s["freqs"], weight=s["weight"], eps=_EPS, interleaved=s["interleaved"])
        return F.seq_cache_gather(cache, s["table"], s["after"], s["first"], s["read"], dtype=s["dtype"])
    return F.seq_cache_tree_attention(s["q"], s["k"], s["v"], s["parents"], cache, s["table"], s["lengths"], window=s["window"], softcap=s["cap"], slopes=s["slopes"])


def _run_plain(s):
    if s["op"] in ("rotate", "rotate_train"):
        return _plain_rotary(s)
    if s["op"] == "verify_tree":
        return _plain_verify_tree(s)
    if s["op"] == "verify_drafts":
        return _plain_verify_drafts(s)
    if s["op"] == "tree":
        return _plain_tree(s)
    return _plain_append(s)


def _cos_sin(positions, freqs, sections):
    """[..., L, pairs] fp32, the angles in 64 bits.  positions [..., axes, L]."""
    axis = torch.cat([torch.full((x,), a, device=freqs.device) for a, x in enumerate(sections)])
    angle = positions.double().transpose(-1, -2)[..., axis] * freqs.double()
    return angle.cos().float(), angle.sin().float()


def _turn(y, cos, sin, interleaved):
    """y [..., L, D] rotated, cos and sin [..., L, pairs]."""
    pairs = cos.shape[-1]
    a, b = (y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2]) if interleaved else (y[..., :pairs], y[..., pairs:2 * pairs])
    za, zb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([za, zb], -1).flatten(-2) if interleaved else torch.cat([za, zb], -1)
    return torch.cat([turned, y[..., 2 * pairs:]], -1)


def _norm(x):
    return torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS)


def _plain_rotary(s):
    flat = lambda x: x.flatten(2, 3) if x.dim() == 5 else x
    cos, sin = _cos_sin(s["positions"].flatten(1), s["freqs"], s["sections"])
    outs, grads, weight_grads = [], [], []
    for name in ("q", "k"):
        x, weight = s[name].detach(), s[name + "_weight"]
        shape, x = x.shape, flat(x).float()
        r = None if weight is None else _norm(x)
        y = x if weight is None else x * r * weight.detach().float()
        outs.append(_turn(y, cos, sin, s["interleaved"]).to(s["dtype"]).reshape(shape))
        if s["op"] == "rotate_train":
            dy = _turn(flat(s["d" + name]).float(), cos, -sin, s["interleaved"])
            if weight is None:
                grads.append(dy.to(s["dtype"]).reshape(shape))
            else:
                gy = dy * weight.detach().float()
                grads.append((r * gy - x * r.pow(3) * (gy * x).mean(-1, keepdim=True)).to(s["dtype"]).reshape(shape))
                weight_grads.append((dy * x * r).sum((0, 1, 2)).to(s["dtype"]))
    return (*outs, *grads, *weight_grads)


def _plain_append(s):
    k, v, n = s["k"].float(), s["v"].float(), s["n"]
    if s["rows"] is not None:
        at = s["rows"].long()[:, None, :, None].expand(-1, k.shape[1], -1, k.shape[3])
        k, v = k.gather(2, at), v.gather(2, at)
    if s["weight"] is not None:
        k = k * _norm(k) * s["weight"].float()
    cos, sin = _cos_sin((s["lengths"][:, None] + torch.arange(n, device=k.device))[:, None], s["freqs"], [s["freqs"].numel()])
    k = _turn(k, cos[:, None], sin[:, None], s["interleaved"])
    read = lambda pages, scales: _plain_read(pages, scales, s["table"], s["after"], s["first"], s["read"]).to(s["dtype"])
    return read(*_plain_store(s, s["k_pages"], s["k_scales"], k)), read(*_plain_store(s, s["v_pages"], s["v_scales"], v))


def _plain_store(s, pages, scales, x):
    """Writes x [B, kv, n, D] behind the sequences' tokens; a page's scale grows with its largest value, and what it held is rounded again."""
    B, kv, n, D = x.shape
    page, table, lengths = pages.shape[2], s["table"].long(), s["lengths"].long()
    touched = (lengths // page)[:, None] + torch.arange((n + page - 2) // page + 1, device=x.device)            # [B, T]
    live = (touched * page < (lengths + n)[:, None])
    ids = torch.gather(table, 1, touched.clamp(max=table.shape[1] - 1))
    token = touched[:, :, None] * page + torch.arange(page, device=x.device) - lengths[:, None, None]          # [B, T, page]: which new token
    is_new, is_old = (token >= 0) & (token < n), token < 0
    new = x.transpose(1, 2)[torch.arange(B, device=x.device)[:, None, None], token.clamp(0, n - 1)]            # [B, T, page, kv, D]
    new = new.transpose(2, 3) * is_new[:, :, None, :, None]
    before = torch.where(is_old.any(-1, keepdim=True), scales[ids], torch.zeros_like(scales[ids]))             # [B, T, kv]
    scale = torch.maximum(before, new.abs().amax((-1, -2)) / 127)
    by = torch.where(scale > 0, scale, torch.ones_like(scale))[..., None, None]
    held = pages[ids]
    again = torch.round(held.float() * (before[..., None, None] / by))
    cells = torch.where(is_new[:, :, None, :, None], torch.round(new / by).clamp(-127, 127), torch.where(is_old[:, :, None, :, None], again, held.float()))
    pages[ids[live]] = cells[live].to(torch.int8)
    scales[ids[live]] = scale[live]
    return pages, scales


def _plain_read(pages, scales, table, lengths, first, n):
    """[B, kv, n, D] in fp32: the values at positions first .. first + n - 1, zero where the sequence has none."""
    page, at = pages.shape[2], first.long()[:, None] + torch.arange(n, device=pages.device)
    inside = (at >= 0) & (at < lengths[:, None])
    at = at.clamp(0, table.shape[1] * page - 1)
    ids = torch.gather(table.long(), 1, at // page)
    x = pages[ids, :, at % page].float() * scales[ids][..., None]      # [B, n, kv, D]
    return (x * inside[:, :, None, None]).transpose(1, 2)


def _plain_above(parents):
    """bool [B, n, n]: j is i or one of its ancestors, of nodes that are some."""
    B, n = parents.shape
    at = torch.arange(n, device=parents.device)
    above = torch.zeros((B, n, n), dtype=torch.bool, device=parents.device)
    for i in range(n):
        p = parents[:, i]
        inner = (p >= 0) & (p < i)
        mine = above[torch.arange(B, device=parents.device), p.clamp(0, n - 1).long()]
        there = (p == -1) | (inner & mine.any(-1))
        above[:, i] = ((mine & inner[:, None]) | (at == i)) & there[:, None]
    return above


def _plain_tree(s):
    q, lengths = s["q"].float(), s["lengths"]
    B, heads, n, D = q.shape
    kv, L = s["k_pages"].shape[1], s["table"].shape[1] * s["k_pages"].shape[2]
    nothing = torch.zeros_like(lengths)
    k, v = (torch.cat([_plain_read(s[x + "_pages"], s[x + "_scales"], s["table"], lengths, nothing, L), s[x].float()], 2) for x in ("k", "v"))
    above = _plain_above(s["parents"])                                   # [B, n, n]
    stands = lengths[:, None] + above.sum(-1) - 1                        # [B, n]
    key_at = torch.cat([torch.arange(L, device=q.device).expand(B, L), stands], 1)
    distance = stands[:, :, None] - key_at[:, None]
    there = above.any(-1)
    visible = torch.cat([(torch.arange(L, device=q.device) < lengths[:, None])[:, None] & there[:, :, None], above], 2)
    if s["window"] is not None:
        visible = visible & (distance < s["window"])
    # the heads of a group read the same keys: they are rows of one product
    rows = lambda x: x.reshape(B, kv, heads // kv * n, x.shape[-1])
    spread = lambda x: x.expand(B, heads, n, L + n).reshape(B, kv, heads // kv * n, L + n)
    raw = torch.matmul(rows(q.contiguous()) * D ** -0.5, k.transpose(-1, -2).contiguous())
    if s["cap"] is not None:
        raw = torch.tanh(raw / s["cap"]) * s["cap"]
    if s["slopes"] is not None:
        raw = raw - spread(s["slopes"][:, None, None] * distance[:, None].float())
    raw = raw.masked_fill(~spread(visible[:, None]), float("-inf"))
    m = raw.amax(-1, keepdim=True)
    p = raw.sub_(torch.where(m == float("-inf"), torch.zeros_like(m), m)).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total == 0, torch.ones_like(total), total))
    return torch.matmul(p, v.contiguous()).reshape(B, heads, n, D).to(s["dtype"])


def _first(mask):
    """The lowest place that is true in each row, the row's length where none is."""
    at = torch.arange(mask.shape[-1], device=mask.device)
    return torch.where(mask, at, torch.full_like(at, mask.shape[-1])).amin(-1)


def _plain_weights(logits, temperatures):
    """Probabilities in 64 bits, [B, rows, V]: the answers are whole numbers, and sums of a long row decide them."""
    x = logits.double() / torch.where(temperatures > 0, temperatures, torch.ones_like(temperatures)).double()[:, None, None]
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    return x.div_(x.sum(-1, keepdim=True))


def _plain_drawn(weights, u):
    """The lowest token up to which the weights [..., V] sum to more than the share u of their total."""
    sums = weights.cumsum(-1)
    return (sums <= u.double()[..., None] * sums[..., -1:]).sum(-1).clamp(max=weights.shape[-1] - 1)


def _largest(logits):
    return _first(logits == logits.amax(-1, keepdim=True))


def _plain_verify_tree(s):
    B, n, V = s["logits"].shape
    at = torch.arange(B, device=s["logits"].device)
    greedy = ~(s["temperatures"] > 0)
    drawn = torch.where(greedy[:, None], _largest(s["logits"]), _plain_drawn(_plain_weights(s["logits"], s["temperatures"]), s["uniforms"]))   # [B, n]
    node, going = torch.zeros_like(at), torch.ones_like(greedy)
    path, counts = torch.full((B, n), -1, dtype=torch.int32, device=at.device), torch.zeros_like(at)
    for step in range(n):
        path[:, step] = torch.where(going, node, -torch.ones_like(node)).to(torch.int32)
        counts += going
        child = (s["parents"] == node[:, None]) & (s["tokens"] == drawn[at, node][:, None]) & (torch.arange(n, device=at.device) > node[:, None])
        going = going & child.any(-1)
        node = torch.where(going, _first(child), node)
    return path, counts.to(torch.int32), drawn[at, node].to(torch.int32)


def _plain_verify_drafts(s):
    B, n, V = s["logits"].shape
    at, greedy = torch.arange(B, device=s["logits"].device), ~(s["temperatures"] > 0)
    p, largest = _plain_weights(s["logits"], s["temperatures"]), _largest(s["logits"])
    tokens = s["tokens"][:, 1:].long()
    if n > 1:
        q = _plain_weights(s["draft"], s["temperatures"])
        pick = lambda x: x.gather(2, tokens[..., None])[..., 0]
        taken = torch.where(greedy[:, None], largest[:, :n - 1] == tokens, s["uniforms"][:, :n - 1].double() * pick(q) < pick(p[:, :n - 1]))
        accepted = taken.int().cumprod(1).sum(1)                          # [B]
    else:
        q, accepted = p[:, :0], torch.zeros_like(at)
    row = p[at, accepted]
    if n > 1:
        rest = (row - q[at, accepted.clamp(max=n - 2)]).clamp_(min=0)
        row = torch.where(((accepted < n - 1) & (rest.sum(-1) > 0))[:, None], rest, row)
    following = torch.where(greedy, largest[at, accepted], _plain_drawn(row, s["uniforms"][:, n]))
    step = torch.arange(n, device=at.device).expand(B, n)
    path = torch.where(step <= accepted[:, None], step, -torch.ones_like(step))
    return path.to(torch.int32), (accepted + 1).to(torch.int32), following.to(torch.int32)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("rotate", "rotate_train"):
        return _exact_rotary(case, s)
    if case["op"] in ("verify_tree", "verify_drafts"):
        return _exact_verify(case, s)
    if case["op"] == "tree":
        return _exact_tree(case, s)
    return _exact_append(case, s)


def _exact_rotated(x, angles, weight, interleaved):
    """x [..., L, D] in 64 bits, angles [L, pairs] or [..., L, pairs]: pairs as complex numbers."""
    if weight is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + _EPS).sqrt() * weight
    pairs = angles.shape[-1]
    turned, rest = x[..., :2 * pairs], x[..., 2 * pairs:]
    turned = turned.unflatten(-1, (pairs, 2) if interleaved else (2, pairs))
    z = torch.complex(*turned.unbind(-1 if interleaved else -2)) * torch.polar(torch.ones_like(angles), angles)
    turned = torch.stack([z.real, z.imag], -1 if interleaved else -2).flatten(-2)
    return torch.cat([turned, rest], -1)


def _exact_angles(positions, freqs, sections):
    parts, at = [], 0
    for axis, x in enumerate(sections):
        parts.append(positions[axis].double()[:, None] * freqs[at:at + x].double()[None])
        at += x
    return torch.cat(parts, 1)


def _exact_rotary(case, s):
    angles = _exact_angles(s["positions"].reshape(len(s["sections"]), -1), s["freqs"], s["sections"])
    outs, grads, weight_grads = [], [], []
    for name in ("q", "k"):
        x = s[name].detach().double().requires_grad_(case["op"] == "rotate_train")
        weight = None if s[name + "_weight"] is None else s[name + "_weight"].detach().double().requires_grad_(case["op"] == "rotate_train")
        z = _exact_rotated(x.flatten(2, 3) if x.dim() == 5 else x, angles, weight, case["interleaved"]).reshape(x.shape)
        outs.append(z.detach())
        if case["op"] == "rotate_train":
            got = torch.autograd.grad(z, [x] if weight is None else [x, weight], s["d" + name].double())
            grads.append(got[0])
            weight_grads += got[1:]
    return (*outs, *grads, *weight_grads)


def _exact_append(case, s):
    """Page by page: what a page holds, its scale, and both again with the new tokens."""
    page, n, table, lengths = case["page"], case["n"], s["table"].tolist(), s["lengths"].tolist()
    results = []
    for which in ("k", "v"):
        cells, scales = s[which + "_pages"].double(), s[which + "_scales"].double()
        rows = []
        for b, L in enumerate(lengths):
            x = s[which][b].double()                                      # [kv, given, D]
            if s["rows"] is not None:
                x = x[:, s["rows"][b].long()]
            if which == "k":
                angles = _exact_angles([torch.arange(L, L + n, device="cuda")], s["freqs"], [s["freqs"].numel()])
                x = _exact_rotated(x, angles, None if s["weight"] is None else s["weight"].double(), case["interleaved"])
            for p in range(L // page, (L + n - 1) // page + 1):
                lo, hi, i = max(L, p * page), min(L + n, (p + 1) * page), table[b][p]
                new, old = x[:, lo - L:hi - L], lo - p * page
                most = new.abs().amax((1, 2)) / 127
                scale = torch.maximum(scales[i], most) if old else most
                if old:
                    cells[i, :, :old] = torch.round(cells[i, :, :old] * (scales[i] / scale)[:, None, None])
                cells[i, :, old:hi - p * page] = torch.round(new / scale.clamp(min=1e-300)[:, None, None])
                scales[i] = scale
            at = list(range(max(L + n - s["read"], 0), L + n))
            ids, slot = torch.tensor([table[b][a // page] for a in at], device="cuda"), torch.tensor([a % page for a in at], device="cuda")
            got = (cells[ids, :, slot] * scales[ids][..., None]).transpose(0, 1)
            rows.append(torch.cat([got.new_zeros((case["kv"], s["read"] - len(at), case["D"])), got], 1))
        results.append(torch.stack(rows))
    return tuple(results)


def _exact_tree(case, s):
    """One sequence and head at a time."""
    B, heads, n, D = s["q"].shape
    group, out = heads // case["kv"], torch.zeros((B, heads, n, D), dtype=torch.float64, device="cuda")
    page, table, scale = case["page"], s["table"].tolist(), D ** -0.5
    for b, (L, parents) in enumerate(zip(s["lengths"].tolist(), s["parents"].tolist())):
        depth = _depths(parents)
        see = torch.zeros((n, L + n), dtype=torch.bool)
        for i in range(n):
            if depth[i] >= 0:
                see[i, :L] = True
                at = i
                while at >= 0:
                    see[i, L + at] = True
                    at = parents[at]
        stands = torch.tensor([L + d for d in depth], device="cuda")
        far = (stands[:, None] - torch.cat([torch.arange(L, device="cuda"), stands])[None]).double()
        see = see.cuda() & (far < (case["window"] or L + n + 1))
        ids = torch.tensor(table[b][:-(-L // page)], device="cuda")
        held = [torch.cat([(s[x + "_pages"][ids].double() * s[x + "_scales"][ids].double()[..., None, None]).transpose(0, 1).flatten(1, 2)[:, :L], s[x][b].double()], 1) for x in ("k", "v")]
        for h in range(heads):
            score = s["q"][b, h].double() @ held[0][h // group].T * scale
            if case["cap"]:
                score = case["cap"] * torch.tanh(score / case["cap"])
            if s["slopes"] is not None:
                score = score - float(s["slopes"][h]) * far
            weight = torch.softmax(score.where(see, score.new_tensor(-math.inf)), 1)
            out[b, h] = weight.where(see.any(1, keepdim=True), weight.new_zeros(())) @ held[1][h // group]
    return out


def _exact_row(logits, temperature):
    return torch.softmax(logits.double() / temperature, 0)


def _exact_choice(weights, u):
    sums = torch.cumsum(weights, 0)
    return min(int(torch.searchsorted(sums, sums[-1:] * u, right=True)), weights.numel() - 1)


def _exact_verify(case, s):
    """One sequence at a time, from node to node."""
    n, paths, counts, following = case["n"], [], [], []
    host = {x: s[x].tolist() for x in ("tokens", "uniforms", "temperatures")}
    trees = [list(range(-1, n - 1))] * case["B"] if s["parents"] is None else s["parents"].tolist()
    for b, parents in enumerate(trees):
        T, tokens, u = host["temperatures"][b], host["tokens"][b], host["uniforms"][b]
        T = float(torch.tensor(T, dtype=torch.float32))
        path = [0]
        while True:
            node = path[-1]
            children = [c for c in range(node + 1, n) if parents[c] == node]
            if T <= 0:
                token = int((s["logits"][b, node] == s["logits"][b, node].max()).nonzero()[0])
                match = [c for c in children if tokens[c] == token]
            elif s["draft"] is None:
                token = _exact_choice(_exact_row(s["logits"][b, node], T), u[node])
                match = [c for c in children if tokens[c] == token]
            else:
                p = _exact_row(s["logits"][b, node], T)
                match = []
                if children:
                    q, x = _exact_row(s["draft"][b, node], T), tokens[children[0]]
                    if u[node] * float(q[x]) < float(p[x]):
                        match = children
                    else:
                        rest = (p - q).clamp(min=0)
                        p = rest if float(rest.sum()) > 0 else p
                if not match:
                    token = _exact_choice(p, u[n])
            if not match:
                break
            path.append(match[0])
        paths.append(path + [-1] * (n - len(path)))
        counts.append(len(path))
        following.append(token)
    return tuple(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (paths, counts, following))


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    B, e = case["B"], 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("rotate", "rotate_train"):
        # in and out; upstream gradients, and gradients; norm and rotation a few operations an element
        elements, train = B * (case["heads"] + case["kv"]) * case["L"] * case["D"], case["op"] == "rotate_train"
        return {"bytes": (4 if train else 2) * elements * e + 4 * len(_sections(case)) * case["L"], "flops": (20 if train else 7) * elements}
    if case["op"] in ("verify_tree", "verify_drafts"):
        rows = case["n"] + (case["n"] - 1 if case["op"] == "verify_drafts" else 0)
        return {"bytes": B * rows * case["V"] * e + 12 * B * case["n"], "flops": 2 * B * rows * case["V"]}
    lengths, n, page, kv, D = _lengths(case), case["n"], case["page"], case["kv"], case["D"]
    if case["op"] == "append":
        # the new tokens read, and written in 8 bits; the old ones of their first pages read and written; then read back
        old = sum(L % page for L in lengths)
        back = sum(min(n + page - 1, L + n) for L in lengths)
        return {"bytes": 2 * kv * D * (B * n * (e + 1) + 2 * old + back + B * (n + page - 1) * e), "flops": 10 * kv * D * B * n + 4 * kv * D * (B * n + old + back)}
    read = pairs = nodes = 0
    for L, parents in zip(lengths, _parents(case)):
        depth, window = _depths(parents), case["window"] or max(lengths) + n + 1
        read += min(L, window - 1)
        pairs += sum(min(L, max(0, window - 1 - d)) + min(d + 1, window) for d in depth if d >= 0)
        nodes += sum(d >= 0 for d in depth)
    return {"bytes": 2 * kv * D * (read + nodes * e) + 2 * case["heads"] * D * nodes * e, "flops": 4 * D * case["heads"] * pairs}
