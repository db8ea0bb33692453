"""Attention over token sequences: what it is timed on, its plain form in torch, and its definition in 64 bits.

Four operators of ``paper_2204_07143_amd.functional``:

* ``seq_attention``: softmax attention of queries [B, heads, Lq, D] over keys and values [B, kv_heads, Lk, D], forward and
  backward.  Query i stands at position i + Lk - Lq; its score with key j is ``cap * tanh(scale <q, k> / cap)`` (no cap:
  ``scale <q, k>``) less ``slope * |distance|``; it sees the keys of its own document that the causal order and the window
  allow, and every key of its document that is marked as prefix.
* ``seq_cache_append``: new keys and values into a cache of pages held in 8 bits, one scale for each page and head.
* ``seq_cache_gather``: the values that such a cache holds for a range of positions, in 16 bits.
* ``seq_cache_attention``: attention of each sequence's newest tokens over its cache.
"""
from __future__ import annotations

import math
import random

import torch

own = False   # True: run() calls the library's operators; False: their plain form

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _attention(name, op, B, heads, kv, Lq, Lk, D, dtype, causal=True, window=0, cap=0.0, slopes=False, docs=0, prefix=False, rows=True):
    """op: "infer" (one call) or "train" (forward and backward).  rows: q, k, v as a projection leaves them, [B, L, heads, D].
    docs: documents packed into each batch item (0: no document mask), the last tokens being padding."""
    return {"name": name, "op": op, "B": B, "heads": heads, "kv": kv, "Lq": Lq, "Lk": Lk, "D": D, "dtype": dtype, "causal": causal, "window": window, "cap": cap,
            "slopes": slopes, "docs": docs, "prefix": prefix, "rows": rows}


def _cache(name, op, B, heads, kv, n, longest, D, page, dtype, window=0, cap=0.0, slopes=False):
    """op: "append" (and what the cache then holds there), "gather" or "decode".  n: new tokens, or positions read; the
    sequences' lengths lie between an eighth of `longest` and `longest`."""
    return {"name": name, "op": op, "B": B, "heads": heads, "kv": kv, "n": n, "longest": longest, "D": D, "page": page, "dtype": dtype, "window": window, "cap": cap,
            "slopes": slopes}


def listed():
    return [
        # the tokens of one 14 x 14 map as a sequence, every token seeing every other: a call whose time is latency
        _attention("infer_one_map_f16", "infer", 1, 8, 8, 196, 196, 32, "f16", causal=False, cap=30.0, rows=False),
        # a decoder's layer in training: grouped heads, causal, capped scores
        _attention("train_capped_causal_bf16", "train", 4, 16, 4, 2048, 2048, 128, "bf16", cap=50.0),
        # the same on long rows of packed documents, with a bias that falls with the distance
        _attention("train_packed_documents_bf16", "train", 1, 16, 8, 8192, 8192, 128, "bf16", slopes=True, docs=9),
        # prompts read in both directions, answers in one: prefix mask, a window, sizes that no tile divides
        _attention("train_prefix_window_f16", "train", 3, 6, 2, 1571, 1571, 64, "f16", window=400, cap=30.0, docs=2, prefix=True),
        # full precision: the tokens of a 56 x 56 map as a sequence
        _attention("train_sequence_f32", "train", 2, 4, 4, 3136, 3136, 32, "f32", slopes=True),
        # the last chunk of a long prompt over all that came before it
        _attention("infer_prompt_chunk_bf16", "infer", 1, 32, 8, 1024, 8192, 128, "bf16", window=4096, cap=50.0),
        # a batch of prompts into the cache, behind what it holds already, and read back
        _cache("append_prompts_bf16", "append", 8, 8, 8, 1000, 700, 128, 64, "bf16"),
        # one token for each of many sequences: latency
        _cache("append_token_f16", "append", 64, 4, 4, 1, 1000, 64, 16, "f16"),
        # a long cache read back for a prompt's next chunk
        _cache("gather_long_f16", "gather", 4, 8, 8, 8192, 8192, 128, 32, "f16"),
        # one sequence's next token: latency
        _cache("decode_one_f16", "decode", 1, 8, 2, 1, 1000, 64, 16, "f16"),
        # the next token of a batch of long sequences, capped scores: the cache streams through once
        _cache("decode_batch_bf16", "decode", 64, 32, 8, 1, 16000, 128, 64, "bf16", cap=50.0),
        # a few drafted tokens a sequence, checked at once: distance bias and window
        _cache("decode_draft_bf16", "decode", 16, 16, 2, 5, 6000, 128, 32, "bf16", window=2048, slopes=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_SCORES = 16 * 8192 * 8192 // 2        # (query, key) pairs of all heads in a drawn case
_MOST_PRODUCTS = _MOST_SCORES * 128
_MOST_CACHED = 64 * 8 * 16000 * 128 // 3    # elements of the keys that the sequences hold


def draw(rng):
    D, kv, group = rng.choice([32, 64, 64, 128, 128]), rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 1, 2, 3, 4, 8])
    cap = rng.choice([0.0, 0.0, 20.0, 30.0, 50.0])
    slopes = rng.random() < 0.35
    if rng.random() < 0.55:
        op = rng.choice(["infer", "train", "train"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f16", "f32"])
        Lk = _log_uniform(rng, 16, 8192)
        Lq = _log_uniform(rng, 1, Lk) if rng.random() < 0.25 else Lk
        causal = rng.random() < 0.75
        window = _log_uniform(rng, 8, Lk) if rng.random() < 0.3 else 0
        docs = rng.randint(1, 1 + min(12, Lk // 16)) if rng.random() < 0.4 else 0
        prefix = causal and rng.random() < 0.3
        most = _MOST_PRODUCTS // (2 if dtype == "f32" else 1)
        while kv * group * Lq * Lk > _MOST_SCORES or kv * group * Lq * Lk * D > most or kv * group > 32:
            kv, group, Lq = max(1, kv // 2), (group if kv > 1 else max(1, group // 2)), (Lq if kv * group > 1 else max(1, Lq // 2))
        B = _log_uniform(rng, 1, max(1, min(16, _MOST_SCORES // (kv * group * Lq * Lk), most // (kv * group * Lq * Lk * D))))
        case = _attention("", op, B, kv * group, kv, Lq, Lk, D, dtype, causal, window, cap, slopes, docs, prefix, rng.random() < 0.7)
    else:
        op = rng.choice(["append", "gather", "decode", "decode", "decode"])
        dtype, page, longest = rng.choice(["f16", "bf16"]), rng.choice([16, 32, 64, 128]), _log_uniform(rng, 24, 16000)
        n = {"append": lambda: rng.choice([1, _log_uniform(rng, 2, 1500)]), "gather": lambda: _log_uniform(rng, 1, longest),
             "decode": lambda: rng.choice([1, 1, 1, rng.randint(2, 8)])}[op]()
        window = _log_uniform(rng, 16, longest) if op == "decode" and rng.random() < 0.3 else 0
        B = _log_uniform(rng, 1, max(1, min(96, _MOST_CACHED // (kv * D * (longest + n)))))
        case = _cache("", op, B, kv * group, kv, n, longest, D, page, dtype, window, cap if op == "decode" else 0.0, slopes and op == "decode")
    del case["name"]
    return case


# ---- what the seed does not change: documents, prefixes, lengths ----------------------------------------------------

def _rng(case):
    return random.Random(",".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name"))


def _layout(case):
    """Document of every position (-1: padding) and whether it is marked as prefix: lists [B][Lk] or None."""
    rng, L = _rng(case), case["Lk"]
    documents, prefix = [], []
    for _ in range(case["B"]):
        docs = max(1, case["docs"])
        padding = rng.randint(0, L // 20) if case["docs"] else 0
        cuts = [0] + sorted(rng.randint(1, max(1, L - padding)) for _ in range(docs - 1)) + [L - padding]
        ids, marks = [], []
        for d, (a, b) in enumerate(zip(cuts, cuts[1:])):
            ids += [d] * (b - a)
            head = rng.randint(0, b - a)
            marks += [True] * head + [False] * (b - a - head)
        documents.append(ids + [-1] * padding)
        prefix.append(marks + [False] * padding)
    return (documents if case["docs"] else None), (prefix if case["prefix"] else None)


def _lengths(case):
    """Tokens of each sequence: those before an append, those the cache holds otherwise (the newest included)."""
    rng = _rng(case)
    lengths = [max(1, int(case["longest"] * rng.uniform(0.125, 1.0))) for _ in range(case["B"])]
    lengths[0] = case["longest"]
    return [max(x, case["n"]) for x in lengths] if case["op"] == "decode" else lengths


def _slopes(case):
    heads = case["heads"]
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


# ---- inputs -----------------------------------------------------------------------------------------------------

def prepare(case, seed):
    """Activations of unit variance, as a normalisation and a projection leave them; caches as appends leave them, in
    pages that lie scattered."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, B, D = _TYPES[case["dtype"]], case["B"], case["D"]
    slopes = torch.tensor(_slopes(case), device="cuda") if case["slopes"] else None

    def normal(heads, L, rows):
        shape = (B, L, heads, D) if rows else (B, heads, L, D)
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)
        return x.transpose(1, 2) if rows else x

    state = {"op": case["op"], "slopes": slopes, "cap": case["cap"] or None, "window": case["window"] or None, "dtype": dt}
    if case["op"] in ("infer", "train"):
        documents, prefix = _layout(case)
        train, rows = case["op"] == "train", case["rows"]
        q, k, v = normal(case["heads"], case["Lq"], rows), normal(case["kv"], case["Lk"], rows), normal(case["kv"], case["Lk"], rows)
        state.update(q=q.requires_grad_(train), k=k.requires_grad_(train), v=v.requires_grad_(train), causal=case["causal"],
                     documents=None if documents is None else torch.tensor(documents, dtype=torch.int32, device="cuda"),
                     prefix=None if prefix is None else torch.tensor(prefix, device="cuda"),
                     dout=normal(case["heads"], case["Lq"], rows) if train else None)
        return state
    lengths, page, kv, n = _lengths(case), case["page"], case["kv"], case["n"]
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
    cells = lambda: torch.randn((pages, kv, page, D), generator=g, device="cuda", dtype=torch.float32).mul_(40.0).round_().clamp_(-127, 127).to(torch.int8)
    scales = lambda: torch.rand((pages, kv), generator=g, device="cuda").mul_(0.01).add_(0.02)
    state.update(k_pages=cells(), v_pages=cells(), k_scales=scales(), v_scales=scales(), table=torch.tensor(table, dtype=torch.int32, device="cuda"),
                 lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), n=n)
    if case["op"] == "append":
        # read back: the last page's worth of positions for a token, a little more than what was written for a prompt
        state.update(k=normal(kv, n, True), v=normal(kv, n, True), after=torch.tensor(held, dtype=torch.int32, device="cuda"), read=n + page - 1,
                     first=torch.tensor([x - n - page + 1 for x in held], dtype=torch.int32, device="cuda"))
    elif case["op"] == "gather":
        state.update(first=torch.tensor([max(0, x - n) for x in lengths], dtype=torch.int32, device="cuda"))
    else:
        state.update(q=normal(case["heads"], n, True))
    return state


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2204_07143_amd import functional as F

    if s["op"] in ("infer", "train"):
        mask = dict(causal=s["causal"], window=s["window"], softcap=s["cap"], slopes=s["slopes"], documents=s["documents"], prefix=s["prefix"])
        if s["op"] == "infer":
            with torch.no_grad():
                return F.seq_attention(s["q"], s["k"], s["v"], **mask)
        out = F.seq_attention(s["q"], s["k"], s["v"], **mask)
        return (out.detach(), *torch.autograd.grad(out, (s["q"], s["k"], s["v"]), s["dout"]))
    cache = F.SeqCache(s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"])
    if s["op"] == "append":
        F.seq_cache_append(cache, s["k"], s["v"], s["table"], s["lengths"])
        return F.seq_cache_gather(cache, s["table"], s["after"], s["first"], s["read"], dtype=s["dtype"])
    if s["op"] == "gather":
        return F.seq_cache_gather(cache, s["table"], s["lengths"], s["first"], s["n"], dtype=s["dtype"])
    return F.seq_cache_attention(s["q"], cache, s["table"], s["lengths"], window=s["window"], softcap=s["cap"], slopes=s["slopes"])


def _run_plain(s):
    if s["op"] in ("infer", "train"):
        return _plain_attention(s)
    if s["op"] == "append":
        for_k = _plain_append(s, s["k_pages"], s["k_scales"], s["k"])
        for_v = _plain_append(s, s["v_pages"], s["v_scales"], s["v"])
        return (_plain_read(*for_k, s["table"], s["after"], s["first"], s["read"]).to(s["dtype"]),
                _plain_read(*for_v, s["table"], s["after"], s["first"], s["read"]).to(s["dtype"]))
    if s["op"] == "gather":
        return (_plain_read(s["k_pages"], s["k_scales"], s["table"], s["lengths"], s["first"], s["n"]).to(s["dtype"]),
                _plain_read(s["v_pages"], s["v_scales"], s["table"], s["lengths"], s["first"], s["n"]).to(s["dtype"]))
    return _plain_decode(s)


def _scores(q, k, distance, visible, cap, slopes):
    """fp32 scores and, where they are capped, the tanh.  distance: query's position less key's."""
    s = torch.matmul(q * (q.shape[-1] ** -0.5), k.transpose(-1, -2).contiguous())
    t = None
    if cap is not None:
        t = torch.tanh(s.div_(cap))
        s = t * cap
    if slopes is not None:
        s = s.sub_(slopes[:, None, None] * distance.abs())
    return s.masked_fill_(~visible, float("-inf")), t


def _softmax(s):
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), torch.zeros_like(m), m)   # a row that sees nothing
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    return p.div_(torch.where(total == 0, torch.ones_like(total), total))


def _plain_attention(s):
    q, k, v = (s[x].detach().float() for x in ("q", "k", "v"))
    B, heads, Lq, D = q.shape
    kv, Lk = k.shape[1], k.shape[2]
    k, v = (x.repeat_interleave(heads // kv, 1) for x in (k, v))
    at, key = torch.arange(Lk - Lq, Lk, device=q.device)[:, None], torch.arange(Lk, device=q.device)[None]
    distance = at - key
    visible = (distance >= 0) if s["causal"] else torch.ones_like(distance, dtype=torch.bool)
    if s["window"] is not None:
        visible = visible & (distance.abs() < s["window"])
    visible = visible[None]
    if s["prefix"] is not None:
        visible = visible | s["prefix"][:, None, :]
    if s["documents"] is not None:
        ids = s["documents"]
        mine = torch.where(at[:, 0] >= 0, ids[:, at[:, 0].clamp(min=0)], torch.full_like(ids[:, :1], -1))
        visible = visible & (mine[:, :, None] == ids[:, None, :]) & (ids[:, None, :] >= 0)
    p, t = _scores(q, k, distance.float(), visible[:, None], s["cap"], s["slopes"])
    p = _softmax(p)
    out = torch.matmul(p, v).to(s["dtype"])
    if s["op"] == "infer":
        return out
    dout = s["dout"].float()
    ds = torch.matmul(dout, v.transpose(-1, -2).contiguous())
    ds = ds.sub_((p * ds).sum(-1, keepdim=True)).mul_(p)
    if t is not None:
        ds = ds.mul_(1 - t.square_())
    scale = D ** -0.5
    dq = torch.matmul(ds, k).mul_(scale)
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q).mul_(scale)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), dout)
    shared = lambda x: x.reshape(B, kv, heads // kv, Lk, D).sum(2).to(s["dtype"])
    return out, dq.to(s["dtype"]), shared(dk), shared(dv)


def _plain_append(s, pages, scales, x):
    """Writes x [B, kv, n, D] behind the sequences' tokens; a page's scale grows with its largest value, and what it held is rounded again."""
    B, kv, n, D = x.shape
    page, table, lengths = pages.shape[2], s["table"].long(), s["lengths"].long()
    touched = (lengths // page)[:, None] + torch.arange((n + page - 2) // page + 1, device=x.device)            # [B, T]
    live = (touched * page < (lengths + n)[:, None])
    ids = torch.gather(table, 1, touched.clamp(max=table.shape[1] - 1))
    token = touched[:, :, None] * page + torch.arange(page, device=x.device) - lengths[:, None, None]          # [B, T, page]: which new token
    is_new, is_old = (token >= 0) & (token < n), token < 0
    new = x.float().transpose(1, 2)[torch.arange(B, device=x.device)[:, None, None], token.clamp(0, n - 1)]    # [B, T, page, kv, D]
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


def _plain_decode(s):
    q, lengths = s["q"].float(), s["lengths"]
    B, heads, n, D = q.shape
    kv, L = s["k_pages"].shape[1], s["table"].shape[1] * s["k_pages"].shape[2]
    nothing = torch.zeros_like(lengths)
    k, v = (_plain_read(s[x + "_pages"], s[x + "_scales"], s["table"], lengths, nothing, L).contiguous() for x in ("k", "v"))
    at = lengths[:, None, None] - n + torch.arange(n, device=q.device)[:, None]
    distance = (at - torch.arange(L, device=q.device))[:, None]        # [B, 1, n, L]
    visible = (distance >= 0) if s["window"] is None else (distance >= 0) & (distance < s["window"])
    # the heads of a group read the same keys: they are rows of one product
    rows = lambda x: x.reshape(B, kv, heads // kv * n, x.shape[-1])
    spread = lambda x: x.expand(B, heads, n, L).reshape(B, kv, heads // kv * n, L)
    raw = torch.matmul(rows(q.contiguous()) * D ** -0.5, k.transpose(-1, -2).contiguous())
    if s["cap"] is not None:
        raw = torch.tanh(raw / s["cap"]) * s["cap"]
    if s["slopes"] is not None:
        raw = raw - spread(s["slopes"][:, None, None] * distance.float())
    p = _softmax(raw.masked_fill(~spread(visible), float("-inf")))
    return torch.matmul(p, v).reshape(B, heads, n, D).to(s["dtype"])


# ---- the definition in 64 bits, one batch item and head at a time ---------------------------------------------------

def _exact_head(q, k, v, dout, see, far, cap, slope):
    scale = q.shape[-1] ** -0.5
    raw = (q @ k.T) * scale
    score = raw if cap is None else cap * torch.tanh(raw / cap)
    if slope is not None:
        score = score - slope * far
    weight = torch.softmax(score.where(see, score.new_tensor(-math.inf)), 1)
    weight = weight.where(see.any(1, keepdim=True), weight.new_zeros(()))   # a row that sees nothing gives zero
    out = weight @ v
    if dout is None:
        return out, None, None, None
    slopes_at = weight * (dout @ v.T - (dout * out).sum(1, keepdim=True))
    if cap is not None:
        slopes_at = slopes_at * torch.cosh(raw / cap).pow(-2)
    return out, slopes_at @ k * scale, slopes_at.T @ q * scale, weight.T @ dout


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("infer", "train"):
        return _exact_attention(case, s)
    if case["op"] == "append":
        return _exact_append(case, s)
    held = [s["lengths"].tolist(), s["table"].tolist()]
    if case["op"] == "gather":
        read = [_exact_positions(case, s, b, x) for b, x in enumerate(s["first"].tolist())]
        return tuple(torch.stack([_exact_values(s, which, held, b, at) for b, at in enumerate(read)]) for which in ("k", "v"))
    out, n, group = [], case["n"], case["heads"] // case["kv"]
    for b, L in enumerate(held[0]):
        k, v = (_exact_values(s, which, held, b, list(range(L))) for which in ("k", "v"))
        far = torch.arange(L - n, L, device="cuda")[:, None] - torch.arange(L, device="cuda")[None]
        see = (far >= 0) & (far < (case["window"] or L + 1))
        for h in range(case["heads"]):
            out.append(_exact_head(s["q"][b, h].double(), k[h // group], v[h // group], None, see, far.double(), s["cap"], float(s["slopes"][h]) if case["slopes"] else None)[0])
    return torch.stack(out).reshape(case["B"], case["heads"], n, case["D"])


def _exact_attention(case, s):
    q, k, v = (s[x].detach().double() for x in ("q", "k", "v"))
    dout = None if s["dout"] is None else s["dout"].double()
    group, Lq, Lk = case["heads"] // case["kv"], case["Lq"], case["Lk"]
    out, dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    far = (torch.arange(Lq, device="cuda") + (Lk - Lq))[:, None] - torch.arange(Lk, device="cuda")
    for b in range(case["B"]):
        see = far >= 0 if case["causal"] else far == far
        if case["window"]:
            see = see & (far < case["window"]) & (far > -case["window"])
        if s["prefix"] is not None:
            see = see | s["prefix"][b]
        if s["documents"] is not None:
            ids = s["documents"][b]
            see = see & (ids[Lk - Lq:, None] == ids) & (ids >= 0)
        for h in range(case["heads"]):
            got = _exact_head(q[b, h], k[b, h // group], v[b, h // group], None if dout is None else dout[b, h], see, far.abs().double(), s["cap"],
                              float(s["slopes"][h]) if case["slopes"] else None)
            out[b, h] = got[0]
            if dout is not None:
                dq[b, h] = got[1]
                dk[b, h // group] += got[2]
                dv[b, h // group] += got[3]
    return out if dout is None else (out, dq, dk, dv)


def _exact_positions(case, s, b, first):
    return list(range(first, first + s.get("read", case["n"])))


def _exact_values(s, which, held, b, at):
    lengths, table = held
    page = s[which + "_pages"].shape[2]
    inside = torch.tensor([0 <= x < lengths[b] for x in at], device="cuda")
    at = [min(max(x, 0), lengths[b] - 1) for x in at]
    ids = torch.tensor([table[b][x // page] for x in at], device="cuda")
    slot = torch.tensor([x % page for x in at], device="cuda")
    x = s[which + "_pages"][ids, :, slot].double() * s[which + "_scales"][ids].double()[..., None]
    return (x * inside[:, None, None]).transpose(0, 1)


def _exact_append(case, s):
    """Page by page: what a page holds, its scale, and both again with the new tokens."""
    page, n, table, lengths = case["page"], case["n"], s["table"].tolist(), s["lengths"].tolist()
    results = []
    for which in ("k", "v"):
        cells, scales, x = s[which + "_pages"].double(), s[which + "_scales"].double(), s[which].double()
        rows = []
        for b, L in enumerate(lengths):
            for p in range(L // page, (L + n - 1) // page + 1):
                lo, hi, i = max(L, p * page), min(L + n, (p + 1) * page), table[b][p]
                new, old = x[b, :, lo - L:hi - L], lo - p * page
                most = new.abs().amax((1, 2)) / 127
                scale = torch.maximum(scales[i], most) if old else most
                if old:
                    cells[i, :, :old] = torch.round(cells[i, :, :old] * (scales[i] / scale)[:, None, None])
                cells[i, :, old:hi - p * page] = torch.round(new / scale.clamp(min=1e-300)[:, None, None])
                scales[i] = scale
            first = L + n - s["read"]
            at = list(range(max(first, 0), L + n))
            ids, slot = torch.tensor([table[b][a // page] for a in at], device="cuda"), torch.tensor([a % page for a in at], device="cuda")
            got = (cells[ids, :, slot] * scales[ids][..., None]).transpose(0, 1)
            rows.append(torch.cat([got.new_zeros((case["kv"], s["read"] - len(at), case["D"])), got], 1))
        results.append(torch.stack(rows))
    return tuple(results)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def _pairs(case):
    """(query, key) pairs of one head that are not masked, over the batch."""
    documents, prefix = _layout(case)
    total, Lq, Lk = 0, case["Lq"], case["Lk"]
    window = case["window"] or Lk + Lq
    key = torch.arange(Lk)
    for b in range(case["B"]):
        ids = None if documents is None else torch.tensor(documents[b])
        marks = None if prefix is None else torch.tensor(prefix[b])
        for lo in range(Lk - Lq, Lk, 512):
            at = torch.arange(lo, min(lo + 512, Lk))[:, None]
            see = (at - key < window) & (key - at < window)
            if case["causal"]:
                see &= key <= at
            if marks is not None:
                see |= marks
            if ids is not None:
                see &= (ids[at] == ids) & (ids >= 0)
            total += int(see.sum())
    return total


def work(case):
    B, heads, kv, D = case["B"], case["heads"], case["kv"], case["D"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("infer", "train"):
        # q and the output (and dout and dq), k and v (and their gradients); two products forward, four backward
        train = case["op"] == "train"
        nq, nk = B * heads * case["Lq"] * D, B * kv * case["Lk"] * D
        marks = B * case["Lk"] * ((4 if case["docs"] else 0) + (1 if case["prefix"] else 0))
        return {"bytes": (4 if train else 2) * (nq + nk) * e + marks, "flops": (12 if train else 4) * D * heads * _pairs(case)}
    lengths, n, page = _lengths(case), case["n"], case["page"]
    if case["op"] == "append":
        # the new tokens read, and written in 8 bits; the old ones of their first pages read and written; then read back
        old = sum(L % page for L in lengths)
        back = sum(min(n + page - 1, L + n) for L in lengths)
        return {"bytes": 2 * kv * D * (B * n * (e + 1) + 2 * old + back + B * (n + page - 1) * e), "flops": 4 * kv * D * (B * n + old + back)}
    if case["op"] == "gather":
        read = sum(min(n, L) for L in lengths)
        return {"bytes": 2 * kv * D * (read + B * n * e), "flops": 2 * kv * D * read}
    window = case["window"] or max(lengths)
    read = sum(min(L, window + n - 1) for L in lengths)
    pairs = sum(min(L - n + i + 1, window) for L in lengths for i in range(n))
    return {"bytes": 2 * kv * D * read + 2 * B * heads * n * D * e, "flops": 4 * D * heads * pairs}
