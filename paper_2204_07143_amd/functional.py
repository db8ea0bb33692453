"""Differentiable wrappers around the C-ABI calls (``torch.autograd.Function``), for drop-in use.

The paper's extension exposes two differentiable functions, QK+RPB and AV, with the softmax
between them left to the framework (arXiv 2204.07143, Appendix A, "Implementation notes");
``na2d_qk_rpb`` and ``na2d_av`` below are that split.  ``na2d`` is the whole operator (Eq. 2-4)
through the fused forward and the fused backward, which keep the attention tensor out of memory.

Only argument marshalling and buffer allocation happen here: every gradient comes from the
library's kernels.  ``na2d``, ``na1d``, ``na2d_unfused`` and the attention over sequences (``seq_*``) do it in native code (``na2d_torch.so``, from
``csrc/host/torch_ops.cpp``): a call on small tensors takes longer in the interpreter than on the GPU.  The functions below
serve ``na2d_qk_rpb``, ``na2d_av`` and ``na2d_softmax``, and whatever the native code hands back: invalid arguments (the
binding's errors), functorch transforms, forward-mode differentiation, tracing, tensors that are not plain ones.  Tensors are ``[B, heads, H, W, D]`` (q, k, v, out), ``[B, heads, H, W, k*k]``
(logits / attention weights) and ``[heads, 2k-1, 2k-1]`` (bias), contiguous, on the GPU; the
library is loaded on first use and a missing library raises.
"""
from __future__ import annotations

import importlib.machinery
import importlib.util
import os
from typing import NamedTuple

import torch

from . import binding as na

_NATIVE_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "na2d_torch.so")
_native_module = None


def _native():
    """The native operators, loaded on first use.  Raises if they or the library have not been built."""
    global _native_module
    if _native_module is None:
        na.load()
        if not os.path.exists(_NATIVE_PATH):
            raise FileNotFoundError(f"{_NATIVE_PATH} is missing: build it with `python -m paper_2204_07143_amd.build`")
        loader = importlib.machinery.ExtensionFileLoader("na2d_torch", _NATIVE_PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("na2d_torch", loader))
        loader.exec_module(module)
        _native_module = module
    return _native_module


def _dense(t: torch.Tensor) -> torch.Tensor:
    """``t`` as it lies in memory: contiguous, and a negated view written out."""
    return t.resolve_neg().contiguous()


def _workspace(x: torch.Tensor, kernel_size: int, kind: int) -> torch.Tensor:
    B, heads, H, W, D = x.shape
    p = na.problem(B, heads, H, W, D, kernel_size, x.dtype)
    return torch.empty(max(16, na.na2d_workspace_bytes(p, kind)), dtype=torch.uint8, device=x.device)


def _bias_grad(d_rpb_f32, rpb):
    return None if d_rpb_f32 is None else d_rpb_f32.to(rpb.dtype)


class _NA2DQKRPB(torch.autograd.Function):
    """logits = scale * <q, k over the neighbourhood> + bias (Eq. 2)."""

    @staticmethod
    def forward(ctx, q, k, rpb, kernel_size, scale):
        q, k = _dense(q), _dense(k)
        rpb_c = None if rpb is None else _dense(rpb)
        logits = torch.empty((*q.shape[:4], kernel_size * kernel_size), dtype=q.dtype, device=q.device)
        na.na2d_qk_rpb(q, k, rpb_c, scale, kernel_size, logits)
        ctx.save_for_backward(q, k)
        ctx.kernel_size, ctx.scale, ctx.has_rpb = kernel_size, scale, rpb is not None
        ctx.rpb_dtype = None if rpb is None else rpb.dtype
        return logits

    @staticmethod
    def backward(ctx, dlogits):
        q, k = ctx.saved_tensors
        ks, scale = ctx.kernel_size, ctx.scale
        dlogits = _dense(dlogits)
        dq, dk, d_rpb = None, None, None
        if ctx.needs_input_grad[0]:
            dq = na.na2d_qk_bwd_q(dlogits, k, scale, ks, torch.empty_like(q))
        if ctx.needs_input_grad[1]:
            dk = na.na2d_qk_bwd_k(dlogits, q, scale, ks, torch.empty_like(k))
        if ctx.has_rpb and ctx.needs_input_grad[2]:
            d32 = torch.empty((q.shape[1], 2 * ks - 1, 2 * ks - 1), dtype=torch.float32, device=q.device)
            na.na2d_qk_bwd_rpb(dlogits, ks, q, d32, _workspace(q, ks, na.WS_QK_BWD_RPB))
            d_rpb = d32.to(ctx.rpb_dtype)
        return dq, dk, d_rpb, None, None


class _NA2DAV(torch.autograd.Function):
    """out = attention weights times the neighbourhood's values (Eq. 3-4)."""

    @staticmethod
    def forward(ctx, attn, v, kernel_size):
        attn, v = _dense(attn), _dense(v)
        out = na.na2d_av(attn, v, kernel_size, torch.empty_like(v))
        ctx.save_for_backward(attn, v)
        ctx.kernel_size = kernel_size
        return out

    @staticmethod
    def backward(ctx, dout):
        attn, v = ctx.saved_tensors
        ks = ctx.kernel_size
        dout = _dense(dout)
        dattn, dv = None, None
        if ctx.needs_input_grad[0]:
            dattn = na.na2d_av_bwd_p(dout, v, ks, torch.empty_like(attn))
        if ctx.needs_input_grad[1]:
            dv = na.na2d_av_bwd_v(attn, dout, ks, torch.empty_like(v))
        return dattn, dv, None


class _NA2D(torch.autograd.Function):
    """The whole operator: softmax(scale * QK + bias) V over each query's neighbourhood."""

    @staticmethod
    def forward(ctx, q, k, v, rpb, kernel_size, scale):
        q, k, v = _dense(q), _dense(k), _dense(v)
        rpb_c = None if rpb is None else _dense(rpb)
        out = torch.empty_like(q)
        lse = torch.empty(q.shape[:4], dtype=torch.float32, device=q.device)
        na.na2d_fused_fwd(q, k, v, rpb_c, scale, kernel_size, out, lse)
        ctx.save_for_backward(q, k, v, lse) if rpb_c is None else ctx.save_for_backward(q, k, v, lse, rpb_c)
        ctx.kernel_size, ctx.scale, ctx.has_rpb = kernel_size, scale, rpb is not None
        return out

    @staticmethod
    def backward(ctx, dout):
        if ctx.has_rpb:
            q, k, v, lse, rpb = ctx.saved_tensors
        else:
            (q, k, v, lse), rpb = ctx.saved_tensors, None
        ks = ctx.kernel_size
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        want_bias = ctx.has_rpb and ctx.needs_input_grad[3]
        d32 = torch.empty((q.shape[1], 2 * ks - 1, 2 * ks - 1), dtype=torch.float32, device=q.device) if want_bias else None
        direct = na.na2d_direct_bwd_workspace_bytes(na.problem(*q.shape, ks, q.dtype))   # 0: not for this problem
        if direct:
            na.na2d_direct_bwd(q, k, v, rpb, ctx.scale, lse, _dense(dout), ks, dq, dk, dv, d32,
                               torch.empty(direct, dtype=torch.uint8, device=q.device))
        else:
            na.na2d_fused_bwd(q, k, v, rpb, ctx.scale, lse, _dense(dout), ks, dq, dk, dv, d32,
                              _workspace(q, ks, na.WS_FUSED_BWD))
        return dq, dk, dv, (d32.to(rpb.dtype) if want_bias else None), None, None


class _NA1D(torch.autograd.Function):
    """The 1D operator on [B, heads, L, D] tensors (bias [heads, 2k-1]): fused forward, fused backward."""

    @staticmethod
    def forward(ctx, q, k, v, rpb, kernel_size, scale):
        q, k, v = _dense(q), _dense(k), _dense(v)
        rpb_c = None if rpb is None else _dense(rpb)
        out = torch.empty_like(q)
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
        na.na1d_fused_fwd(q, k, v, rpb_c, scale, kernel_size, out, lse)
        ctx.save_for_backward(q, k, v, lse) if rpb_c is None else ctx.save_for_backward(q, k, v, lse, rpb_c)
        ctx.kernel_size, ctx.scale, ctx.has_rpb = kernel_size, scale, rpb is not None
        return out

    @staticmethod
    def backward(ctx, dout):
        if ctx.has_rpb:
            q, k, v, lse, rpb = ctx.saved_tensors
        else:
            (q, k, v, lse), rpb = ctx.saved_tensors, None
        ks = ctx.kernel_size
        B, heads, L, D = q.shape
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        want_bias = ctx.has_rpb and ctx.needs_input_grad[3]
        d32 = torch.empty((heads, 2 * ks - 1), dtype=torch.float32, device=q.device) if want_bias else None
        ws = torch.empty(max(16, na.na1d_fused_bwd_workspace_bytes(na.problem_1d(B, heads, L, D, ks, q.dtype))),
                         dtype=torch.uint8, device=q.device)
        na.na1d_fused_bwd(q, k, v, rpb, ctx.scale, lse, _dense(dout), ks, dq, dk, dv, d32, ws)
        return dq, dk, dv, (d32.to(rpb.dtype) if want_bias else None), None, None


class _NA2DSoftmax(torch.autograd.Function):
    """attn = softmax(logits) over the k*k axis (Eq. 4), forward and backward by the library's kernels."""

    @staticmethod
    def forward(ctx, logits, like, kernel_size):
        logits = _dense(logits)
        attn = na.na2d_softmax(logits, kernel_size, like, torch.empty_like(logits))
        ctx.save_for_backward(attn)
        ctx.kernel_size, ctx.like_shape = kernel_size, like.shape
        return attn

    @staticmethod
    def backward(ctx, dattn):
        (attn,) = ctx.saved_tensors
        like = torch.empty(ctx.like_shape, dtype=attn.dtype, device="meta")   # shape and dtype only
        ds = na.na2d_softmax_bwd(attn, _dense(dattn), ctx.kernel_size, like, torch.empty_like(attn))
        return ds, None, None


def _scale_of(q, scale):
    return float(q.shape[-1]) ** -0.5 if scale is None else float(scale)


def na2d_qk_rpb(q, k, rpb, kernel_size: int, scale: float | None = None):
    """Neighbourhood logits ``[B, heads, H, W, k*k]``; differentiable in q, k and rpb (rpb may be None)."""
    return _NA2DQKRPB.apply(q, k, rpb, int(kernel_size), _scale_of(q, scale))


def na2d_av(attn, v, kernel_size: int):
    """Weighted sum of the neighbourhood's values ``[B, heads, H, W, D]``; differentiable in attn and v."""
    return _NA2DAV.apply(attn, v, int(kernel_size))


def na2d(q, k, v, rpb=None, kernel_size: int = 7, scale: float | None = None):
    """2D neighbourhood attention, fused; differentiable in q, k, v and rpb."""
    out = _native().na2d(q, k, v, rpb, int(kernel_size), None if scale is None else float(scale))
    return out if out is not None else _NA2D.apply(q, k, v, rpb, int(kernel_size), _scale_of(q, scale))


def na1d(q, k, v, rpb=None, kernel_size: int = 7, scale: float | None = None):
    """1D neighbourhood attention ([B, heads, L, D]), fused; differentiable in q, k, v and rpb."""
    out = _native().na1d(q, k, v, rpb, int(kernel_size), None if scale is None else float(scale))
    return out if out is not None else _NA1D.apply(q, k, v, rpb, int(kernel_size), _scale_of(q, scale))


def na2d_softmax(logits, like, kernel_size: int):
    """Softmax over the k*k axis of neighbourhood logits; ``like`` is any [B, heads, H, W, D] tensor of the
    problem (its shape and dtype describe it to the library).  Differentiable in logits."""
    return _NA2DSoftmax.apply(logits, like, int(kernel_size))


def na2d_unfused(q, k, v, rpb=None, kernel_size: int = 7, scale: float | None = None):
    """The same operator as the paper composes it: QK+RPB, softmax, AV; every step, forward and backward, is a
    library kernel."""
    out = _native().na2d_unfused(q, k, v, rpb, int(kernel_size), None if scale is None else float(scale))
    if out is not None:
        return out
    logits = na2d_qk_rpb(q, k, rpb, kernel_size, scale)
    return na2d_av(na2d_softmax(logits, q, kernel_size), v, kernel_size)


# ---- attention over sequences -----------------------------------------------------------------------------------------

def _rows(t: torch.Tensor) -> torch.Tensor:
    """``t`` as the library reads it: any strides of whole 16 bytes but for the last dimension's; a copy where it has others."""
    t = t.resolve_neg()
    step = 16 // t.element_size()
    fits = (t.shape[-1] == 1 or t.stride(-1) == 1) and t.data_ptr() % 16 == 0
    fits = fits and all(n == 1 or s % step == 0 for n, s in zip(t.shape[:-1], t.stride()[:-1]))
    fits = fits and ((t.shape[-2] - 1) * t.stride(-2) + t.shape[-1]) * t.element_size() < 1 << 31
    return t if fits else t.clone(memory_format=torch.contiguous_format)


def _like(t: torch.Tensor) -> torch.Tensor:
    """An empty tensor in ``t``'s order of dimensions, with the last one innermost."""
    out = torch.empty_like(t)
    return out if out.stride(-1) == 1 and _rows(out) is out else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _scratch(size: int, like: torch.Tensor):
    return torch.empty(size, dtype=torch.uint8, device=like.device) if size else None


class _OnceOnly(torch.autograd.Function):
    """Gradients as they are, tied to what they depend on by a node that raises: no second derivative, and none that is silently zero."""

    @staticmethod
    def forward(ctx, count, *tensors):
        return tuple(t.view_as(t) for t in tensors[:count])

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("seq_attention has no second derivative")


class _SeqAttention(torch.autograd.Function):
    """Softmax attention over a sequence (include/seq.h)."""

    @staticmethod
    def forward(ctx, q, k, v, slopes, documents, prefix, settings):
        q, k, v = _rows(q), _rows(k), _rows(v)
        out = _like(q)
        ctx.settings, ctx.empty = settings, 0 in q.shape or 0 in k.shape
        train = any(ctx.needs_input_grad)
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if train else None
        rest = torch.empty_like(out) if train and q.element_size() == 2 else None
        if ctx.empty:
            out.zero_()
        else:
            marked = documents is not None or prefix is not None
            ws = _scratch(na.seq_attention_workspace_bytes(na.seq_problem(q, k, v=v, out=out, **settings), marked), q)
            na.seq_attention_fwd(q, k, v, slopes, documents, prefix, out, lse, rest, ws, **settings)
        if train:
            ctx.save_for_backward(q, k, v, out, lse, rest, slopes, documents, prefix)
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v = ctx.saved_tensors[:3]
        with torch.no_grad():
            grads = _SeqAttention.gradients(ctx, dout)
        if torch.is_grad_enabled():
            grads = _OnceOnly.apply(3, *grads, q, k, v, dout)
        return (*grads, None, None, None, None)

    @staticmethod
    def gradients(ctx, dout):
        q, k, v, out, lse, rest, slopes, documents, prefix = ctx.saved_tensors
        dq, dk, dv = _like(q), _like(k), _like(v)
        if ctx.empty:
            return dq.zero_(), dk.zero_(), dv.zero_()
        dout = _rows(dout)
        p = na.seq_problem(q, k, v=v, out=out, dout=dout, dq=dq, dk=dk, dv=dv, **ctx.settings)
        ws = _scratch(na.seq_attention_workspace_bytes(p, documents is not None or prefix is not None, True), q)
        na.seq_attention_bwd(q, k, v, slopes, documents, prefix, out, lse, rest, dout, dq, dk, dv, ws, **ctx.settings)
        return dq, dk, dv


def _settings(q, window, softcap, scale, slopes) -> dict:
    if window is not None and (int(window) != window or not 1 <= window <= 1 << 30):
        raise ValueError(f"window must be a whole number of at least 1, or None, got {window}")
    if softcap is not None and not 0 < softcap < float("inf"):
        raise ValueError(f"softcap must be positive and finite, or None, got {softcap}")
    if slopes is not None and slopes.requires_grad:
        raise ValueError("slopes are constants: they have no gradient")
    return dict(window=0 if window is None else int(window), softcap=0.0 if softcap is None else float(softcap), scale=_scale_of(q, scale))


def _heads_of(q, k, v):
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("expected [B, heads, L, D] tensors")
    B, heads, _, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != D:
        raise ValueError(f"keys {tuple(k.shape)} and values {tuple(v.shape)} do not fit queries {tuple(q.shape)}")
    if k.shape[1] == 0 or heads % k.shape[1]:
        raise ValueError(f"{heads} query heads cannot share {k.shape[1]} key heads")


def seq_attention(q, k, v, *, causal: bool = False, window: int | None = None, softcap: float | None = None, slopes=None, documents=None, prefix=None,
                  scale: float | None = None):
    """Softmax attention of ``q`` [B, heads, Lq, D] over ``k``, ``v`` [B, kv_heads, Lk, D]; differentiable in q, k and v.

    Query i stands at position i + Lk - Lq.  It sees the keys less than ``window`` away, none behind it if ``causal``, and wherever they stand those marked in
    ``prefix`` (bool [B, Lk]); of all these only the keys of its own document (``documents``, int32 [B, Lk], Lq <= Lk; a
    negative one marks padding, which sees and is seen by nobody).  A score is ``softcap * tanh(scale <q, k> / softcap)`` (None: ``scale <q, k>``)
    less ``slopes[head] * |distance|`` (fp32 [heads]).  ``scale`` is D ** -0.5 unless given.  D is 32, 64 or 128; f32, f16, bf16.  The
    tensors may be strided views ([B, L, heads, D] transposed); others than of whole 16-byte rows are copied.  A call that is differentiated keeps q, k, v, out and
    its log-sum-exp for the backward pass, and in 16 bit a second tensor of out's size: what out's rounding took.
    """
    out = _native().seq_attention(q, k, v, causal, window, softcap, slopes, documents, prefix, scale)
    if out is not None:
        return out
    _heads_of(q, k, v)
    settings = dict(causal=bool(causal), **_settings(q, window, softcap, scale, slopes))
    return _SeqAttention.apply(q, k, v, slopes, documents, prefix, settings)


class SeqCache(NamedTuple):
    """Keys and values in 8 bits: pages int8 [pages, kv_heads, page, D] and a scale for each page and head, fp32 [pages, kv_heads]; a value is
    the integer times the scale.  Which page holds what is the caller's: a table, int32 [B, width], gives each sequence's pages in order."""
    k_pages: torch.Tensor
    v_pages: torch.Tensor
    k_scales: torch.Tensor
    v_scales: torch.Tensor

    @classmethod
    def empty(cls, pages: int, kv_heads: int, page: int, head_dim: int, device="cuda") -> "SeqCache":
        cells = (torch.zeros((pages, kv_heads, page, head_dim), dtype=torch.int8, device=device) for _ in range(2))
        return cls(*cells, *(torch.zeros((pages, kv_heads), dtype=torch.float32, device=device) for _ in range(2)))


def seq_cache_append(cache: SeqCache, k, v, table, lengths, counts=None) -> None:
    """Puts ``k``, ``v`` [B, kv_heads, n, D] behind the ``lengths`` (int32 [B]) tokens of each sequence, the first ``counts[b]`` of the n where ``counts``
    (int32 [B]) is given.  A page's scale grows with its largest value; what it held is then rounded again.  ``lengths`` stays as it is.  No page may be
    appended to twice in one call; a page number that is none is passed over."""
    if _native().seq_cache_append(*cache, k, v, table, lengths, counts):
        return
    if k.dim() != 4 or v.dim() != 4:
        raise ValueError("expected [B, heads, L, D] tensors")
    if 0 not in k.shape:
        with torch.no_grad():
            na.seq_cache_append(_rows(k), _rows(v), table, lengths, counts, *cache)


def seq_cache_gather(cache: SeqCache, table, lengths, first, n: int, dtype=torch.bfloat16):
    """The keys and values, [B, kv_heads, n, D] each, that the cache holds at positions ``first[b]`` (int32 [B]) .. + n - 1; 0 where a sequence has no token."""
    out = _native().seq_cache_gather(*cache, table, lengths, first, n, dtype)
    if out is not None:
        return out
    B, (_, kv_heads, _, D) = table.shape[0], cache.k_pages.shape
    k, v = (torch.empty((B, kv_heads, n, D), dtype=dtype, device=cache.k_pages.device) for _ in range(2))
    return (k, v) if k.numel() == 0 else na.seq_cache_gather(*cache, table, lengths, first, k, v)


def seq_cache_attention(q, cache: SeqCache, table, lengths, *, window: int | None = None, softcap: float | None = None, slopes=None, scale: float | None = None):
    """Attention of each sequence's last n tokens, ``q`` [B, heads, n, D] in f16 or bf16, over its cache, which holds their keys and values already:
    ``lengths`` counts them.  The work is laid out for sequences as long as ``table`` is wide: hand in the columns in use.  In causal order; scores as ``seq_attention`` has them.  Not differentiable."""
    out = _native().seq_cache_attention(q, *cache, table, lengths, window, softcap, slopes, scale)
    if out is not None:
        return out
    if q.dim() != 4:
        raise ValueError("expected [B, heads, L, D] tensors")
    settings = _settings(q, window, softcap, scale, slopes)
    with torch.no_grad():
        q = _rows(q)
        out = _like(q)
        if q.numel() == 0:
            return out
        p = na.seq_cache_problem(q, cache.k_pages, table, heads=q.shape[1], out=out, **settings)
        return na.seq_cache_attention(q, *cache, table, lengths, slopes, out, _scratch(na.seq_cache_attention_workspace_bytes(p), q), **settings)
