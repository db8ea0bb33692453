"""Thin Python binding of the C-ABI library ``libna2d.so`` (see ``include/na2d.h``).

Argument marshalling only: every function takes torch tensors that already live on the GPU
(PyTorch is used for device memory and streams, nothing else), checks dtype / shape /
contiguity, passes raw device pointers and the current HIP stream through ctypes and raises
``Na2dError`` on a non-zero status.  There is no fallback: if the library has not been built
(``python -m paper_2204_07143_amd.build``) loading raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libna2d.so")

DTYPE_CODES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
WS_QK_BWD_RPB, WS_BWD, WS_FUSED_BWD = 0, 1, 2

EXPORTS = (
    "na2d_qk_rpb", "na2d_softmax", "na2d_av", "na2d_fused_fwd", "na2d_av_bwd_p", "na2d_av_bwd_v",
    "na2d_softmax_bwd", "na2d_qk_bwd_q", "na2d_qk_bwd_k", "na2d_qk_bwd_rpb", "na2d_qk_bwd_rpb_noalloc", "na2d_bwd", "na2d_fused_bwd",
    "na2d_fused_bwd_is_fused", "na2d_direct_bwd", "na2d_direct_bwd_workspace_bytes",
    "na2d_workspace_bytes", "na2d_debug_indices", "na2d_host_axis_tables", "na2d_validate_problem",
    "na2d_strerror", "na2d_version",
)


EXPORTS_1D = (
    "na1d_validate_problem", "na1d_qk_rpb", "na1d_softmax", "na1d_av", "na1d_fused_fwd", "na1d_av_bwd_p", "na1d_av_bwd_v",
    "na1d_softmax_bwd", "na1d_qk_bwd_q", "na1d_qk_bwd_k", "na1d_qk_bwd_rpb", "na1d_workspace_bytes",
    "na1d_fused_bwd", "na1d_fused_bwd_workspace_bytes",
)


EXPORTS_SEQ = (
    "seq_validate_problem", "seq_attention_workspace_bytes", "seq_attention_fwd", "seq_attention_bwd", "seq_cache_validate", "seq_cache_append",
    "seq_cache_gather", "seq_cache_attention", "seq_cache_attention_workspace_bytes",
    "seq_rotary_validate", "seq_rotary_fwd", "seq_rotary_bwd", "seq_rotary_bwd_workspace_bytes", "seq_cache_append_rows",
    "seq_cache_tree_attention", "seq_cache_tree_attention_workspace_bytes", "seq_verify_validate", "seq_verify", "seq_verify_workspace_bytes",
)
SEQ_CACHE_APPEND, SEQ_CACHE_GATHER, SEQ_CACHE_ATTENTION = 0, 1, 2


class Na2dError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"na2d status {status}: {message}")
        self.status = status


class Na2dProblem(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "heads", "H", "W", "D", "k", "dtype")]


class Na1dProblem(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "heads", "L", "D", "k", "dtype")]


class SeqStrides(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("batch", "head", "row")]


class SeqProblem(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "heads", "kv_heads", "Lq", "Lk", "D", "dtype", "causal", "window")]
                + [(n, ctypes.c_float) for n in ("scale", "softcap")]
                + [(n, SeqStrides) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")])


class SeqCacheProblem(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "heads", "kv_heads", "D", "page", "pages", "table_width", "dtype", "n", "window")]
                + [(n, ctypes.c_float) for n in ("scale", "softcap")] + [(n, SeqStrides) for n in ("q", "out")])


class SeqRotation(ctypes.Structure):
    _fields_ = [("pairs", ctypes.c_int32), ("axes", ctypes.c_int32), ("sections", ctypes.c_int32 * 4), ("interleaved", ctypes.c_int32), ("weight_dtype", ctypes.c_int32),
                ("eps", ctypes.c_float)]


class SeqRotaryProblem(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "heads", "kv_heads", "L", "D", "dtype")] + [("rotation", SeqRotation), ("shared", ctypes.c_int32)]
                + [(n, SeqStrides) for n in ("q", "k", "q_out", "k_out", "dq", "dk")])


class SeqVerifyProblem(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "n", "V", "dtype", "drafted")] + [(n, ctypes.c_int64) for n in ("batch", "row", "draft_batch", "draft_row")]


_lib = None


def load(path: str | None = None) -> ctypes.CDLL:
    """Load libna2d.so (once). Raises if it has not been built.  ``path`` (first call only) names another build of
    the same library, e.g. the benchmark's memory-only measurement build."""
    global _lib
    if _lib is None:
        lib_path = LIB_PATH if path is None else path
        if not os.path.exists(lib_path):
            raise FileNotFoundError(
                f"{lib_path} is missing: build it with `python -m paper_2204_07143_amd.build` "
                "(there is no CPU or PyTorch fallback)")
        lib = ctypes.CDLL(lib_path)
        vp, pp, f = ctypes.c_void_p, ctypes.POINTER(Na2dProblem), ctypes.c_float
        sigs = {
            "na2d_qk_rpb": [pp, vp, vp, vp, f, vp, vp],
            "na2d_softmax": [pp, vp, vp, vp],
            "na2d_av": [pp, vp, vp, vp, vp],
            "na2d_fused_fwd": [pp, vp, vp, vp, vp, f, vp, vp, vp],
            "na2d_av_bwd_p": [pp, vp, vp, vp, vp],
            "na2d_av_bwd_v": [pp, vp, vp, vp, vp],
            "na2d_softmax_bwd": [pp, vp, vp, vp, vp],
            "na2d_qk_bwd_q": [pp, vp, vp, f, vp, vp],
            "na2d_qk_bwd_k": [pp, vp, vp, f, vp, vp],
            "na2d_qk_bwd_rpb": [pp, vp, vp, vp, ctypes.c_size_t, vp],
            "na2d_qk_bwd_rpb_noalloc": [pp, vp, vp, vp],
            "na2d_bwd": [pp, vp, vp, vp, vp, vp, f, vp, vp, vp, vp, vp, ctypes.c_size_t, vp],
            "na2d_fused_bwd": [pp, vp, vp, vp, vp, f, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp],
            "na2d_direct_bwd": [pp, vp, vp, vp, vp, f, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp],
            "na2d_debug_indices": [pp, vp, vp, vp],
            "na2d_host_axis_tables": [ctypes.c_int32, ctypes.c_int32, vp, vp, vp],
            "na2d_validate_problem": [pp],
            "na2d_fused_bwd_is_fused": [pp],
        }
        for name, argtypes in sigs.items():
            fn = getattr(lib, name)
            fn.argtypes = argtypes
            fn.restype = ctypes.c_int
        p1 = ctypes.POINTER(Na1dProblem)
        sigs_1d = {
            "na1d_validate_problem": [p1],
            "na1d_qk_rpb": [p1, vp, vp, vp, f, vp, vp],
            "na1d_softmax": [p1, vp, vp, vp],
            "na1d_av": [p1, vp, vp, vp, vp],
            "na1d_fused_fwd": [p1, vp, vp, vp, vp, f, vp, vp, vp],
            "na1d_av_bwd_p": [p1, vp, vp, vp, vp],
            "na1d_av_bwd_v": [p1, vp, vp, vp, vp],
            "na1d_softmax_bwd": [p1, vp, vp, vp, vp],
            "na1d_qk_bwd_q": [p1, vp, vp, f, vp, vp],
            "na1d_qk_bwd_k": [p1, vp, vp, f, vp, vp],
            "na1d_qk_bwd_rpb": [p1, vp, vp, vp, ctypes.c_size_t, vp],
            "na1d_fused_bwd": [p1, vp, vp, vp, vp, f, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp],
        }
        for name, argtypes in sigs_1d.items():
            fn = getattr(lib, name)
            fn.argtypes = argtypes
            fn.restype = ctypes.c_int
        ps, pc, pr, pv, size = (*(ctypes.POINTER(t) for t in (SeqProblem, SeqCacheProblem, SeqRotaryProblem, SeqVerifyProblem)), ctypes.c_size_t)
        sigs_seq = {
            "seq_validate_problem": [ps, ctypes.c_int],
            "seq_attention_fwd": [ps] + [vp] * 10 + [size, vp],
            "seq_attention_bwd": [ps] + [vp] * 14 + [size, vp],
            "seq_cache_validate": [pc, ctypes.c_int],
            "seq_cache_append": [pc] + [vp] * 10,
            "seq_cache_gather": [pc] + [vp] * 10,
            "seq_cache_attention": [pc] + [vp] * 10 + [size, vp],
            "seq_cache_append_rows": [pc, ctypes.POINTER(SeqRotation), ctypes.c_int32] + [vp] * 4 + [ctypes.c_int] + [vp] * 10,
            "seq_cache_tree_attention": [pc, ctypes.POINTER(SeqStrides), ctypes.POINTER(SeqStrides)] + [vp] * 13 + [size, vp],
            "seq_verify_validate": [pv],
            "seq_verify": [pv] + [vp] * 10 + [size, vp],
            "seq_rotary_validate": [pr, ctypes.c_int],
            "seq_rotary_fwd": [pr] + [vp] * 9,
            "seq_rotary_bwd": [pr] + [vp] * 13 + [size, vp],
        }
        for name, argtypes in sigs_seq.items():
            fn = getattr(lib, name)
            fn.argtypes = argtypes
            fn.restype = ctypes.c_int
        lib.seq_attention_workspace_bytes.argtypes = [ps, ctypes.c_int, ctypes.c_int]
        lib.seq_attention_workspace_bytes.restype = size
        for name, problem in (("seq_rotary_bwd", pr), ("seq_cache_tree_attention", pc), ("seq_verify", pv)):
            fn = getattr(lib, name + "_workspace_bytes")
            fn.argtypes, fn.restype = [problem], size
        lib.seq_cache_attention_workspace_bytes.argtypes = [pc]
        lib.seq_cache_attention_workspace_bytes.restype = size
        lib.na1d_workspace_bytes.argtypes = [p1]
        lib.na1d_workspace_bytes.restype = ctypes.c_size_t
        lib.na1d_fused_bwd_workspace_bytes.argtypes = [p1]
        lib.na1d_fused_bwd_workspace_bytes.restype = ctypes.c_size_t
        lib.na2d_workspace_bytes.argtypes = [pp, ctypes.c_int]
        lib.na2d_workspace_bytes.restype = ctypes.c_size_t
        lib.na2d_direct_bwd_workspace_bytes.argtypes = [pp]
        lib.na2d_direct_bwd_workspace_bytes.restype = ctypes.c_size_t
        lib.na2d_strerror.argtypes = [ctypes.c_int]
        lib.na2d_strerror.restype = ctypes.c_char_p
        lib.na2d_version.restype = ctypes.c_int
        _lib = lib
    return _lib


def strerror(status: int) -> str:
    return load().na2d_strerror(int(status)).decode()


def _check(status: int) -> None:
    if status != 0:
        raise Na2dError(status, strerror(status))


def problem(B: int, heads: int, H: int, W: int, D: int, k: int, dtype) -> Na2dProblem:
    code = DTYPE_CODES[dtype] if dtype in DTYPE_CODES else int(dtype)
    return Na2dProblem(B, heads, H, W, D, k, code)


def _problem_of(x: torch.Tensor, k: int) -> Na2dProblem:
    if x.dim() != 5:
        raise ValueError("expected a [B, heads, H, W, D] tensor")
    B, heads, H, W, D = x.shape
    return problem(B, heads, H, W, D, k, x.dtype)


def _ptr(t, dtype=None, shape=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("na2d takes GPU tensors only")
    if not t.is_contiguous():
        raise ValueError("na2d takes contiguous tensors only")
    if t.is_neg():
        raise ValueError("na2d does not take negated views")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _attn_shape(x: torch.Tensor, k: int):
    return (*x.shape[:4], k * k)


def _rpb_shape(x: torch.Tensor, k: int):
    return (x.shape[1], 2 * k - 1, 2 * k - 1)


# ---- the C ABI, one Python function per export, same names ---------------------------------

def na2d_qk_rpb(q, k_, rpb, scale: float, kernel: int, logits):
    p = _problem_of(q, kernel)
    _check(load().na2d_qk_rpb(ctypes.byref(p), _ptr(q), _ptr(k_, q.dtype, q.shape),
                              _ptr(rpb, q.dtype, _rpb_shape(q, kernel)) if rpb is not None else None,
                              scale, _ptr(logits, q.dtype, _attn_shape(q, kernel)), _stream()))
    return logits


def na2d_softmax(logits, kernel: int, like, out):
    p = _problem_of(like, kernel)
    _check(load().na2d_softmax(ctypes.byref(p), _ptr(logits, like.dtype, _attn_shape(like, kernel)),
                               _ptr(out, like.dtype, _attn_shape(like, kernel)), _stream()))
    return out


def na2d_av(attn, v, kernel: int, out):
    p = _problem_of(v, kernel)
    _check(load().na2d_av(ctypes.byref(p), _ptr(attn, v.dtype, _attn_shape(v, kernel)), _ptr(v),
                          _ptr(out, v.dtype, v.shape), _stream()))
    return out


def na2d_fused_fwd(q, k_, v, rpb, scale: float, kernel: int, out, lse=None):
    p = _problem_of(q, kernel)
    _check(load().na2d_fused_fwd(ctypes.byref(p), _ptr(q), _ptr(k_, q.dtype, q.shape), _ptr(v, q.dtype, q.shape),
                                 _ptr(rpb, q.dtype, _rpb_shape(q, kernel)) if rpb is not None else None, scale,
                                 _ptr(out, q.dtype, q.shape),
                                 _ptr(lse, torch.float32, q.shape[:4]) if lse is not None else None, _stream()))
    return out


def na2d_av_bwd_p(dout, v, kernel: int, dp):
    p = _problem_of(v, kernel)
    _check(load().na2d_av_bwd_p(ctypes.byref(p), _ptr(dout, v.dtype, v.shape), _ptr(v),
                                _ptr(dp, v.dtype, _attn_shape(v, kernel)), _stream()))
    return dp


def na2d_av_bwd_v(attn, dout, kernel: int, dv):
    p = _problem_of(dout, kernel)
    _check(load().na2d_av_bwd_v(ctypes.byref(p), _ptr(attn, dout.dtype, _attn_shape(dout, kernel)), _ptr(dout),
                                _ptr(dv, dout.dtype, dout.shape), _stream()))
    return dv


def na2d_softmax_bwd(attn, dp, kernel: int, like, ds):
    p = _problem_of(like, kernel)
    shape = _attn_shape(like, kernel)
    _check(load().na2d_softmax_bwd(ctypes.byref(p), _ptr(attn, like.dtype, shape), _ptr(dp, like.dtype, shape),
                                   _ptr(ds, like.dtype, shape), _stream()))
    return ds


def na2d_qk_bwd_q(ds, k_, scale: float, kernel: int, dq):
    p = _problem_of(k_, kernel)
    _check(load().na2d_qk_bwd_q(ctypes.byref(p), _ptr(ds, k_.dtype, _attn_shape(k_, kernel)), _ptr(k_), scale,
                                _ptr(dq, k_.dtype, k_.shape), _stream()))
    return dq


def na2d_qk_bwd_k(ds, q, scale: float, kernel: int, dk):
    p = _problem_of(q, kernel)
    _check(load().na2d_qk_bwd_k(ctypes.byref(p), _ptr(ds, q.dtype, _attn_shape(q, kernel)), _ptr(q), scale,
                                _ptr(dk, q.dtype, q.shape), _stream()))
    return dk


def na2d_workspace_bytes(p: Na2dProblem, kind: int) -> int:
    return int(load().na2d_workspace_bytes(ctypes.byref(p), int(kind)))


def na2d_qk_bwd_rpb(ds, kernel: int, like, d_rpb, workspace):
    p = _problem_of(like, kernel)
    _check(load().na2d_qk_bwd_rpb(ctypes.byref(p), _ptr(ds, like.dtype, _attn_shape(like, kernel)),
                                  _ptr(d_rpb, torch.float32, _rpb_shape(like, kernel)), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream()))
    return d_rpb


NOALLOC_SCRATCH_BYTES = 4 << 20   # NA2D_NOALLOC_SCRATCH_BYTES of na2d.h


def na2d_qk_bwd_rpb_noalloc(ds, kernel: int, like, d_rpb):
    """na2d_qk_bwd_rpb with the partials in the library's own device array: no workspace argument."""
    p = _problem_of(like, kernel)
    _check(load().na2d_qk_bwd_rpb_noalloc(ctypes.byref(p), _ptr(ds, like.dtype, _attn_shape(like, kernel)),
                                          _ptr(d_rpb, torch.float32, _rpb_shape(like, kernel)), _stream()))
    return d_rpb


def na2d_bwd(q, k_, v, attn, dout, scale: float, kernel: int, dq, dk, dv, d_rpb, workspace):
    p = _problem_of(q, kernel)
    _check(load().na2d_bwd(ctypes.byref(p), _ptr(q), _ptr(k_, q.dtype, q.shape), _ptr(v, q.dtype, q.shape),
                           _ptr(attn, q.dtype, _attn_shape(q, kernel)), _ptr(dout, q.dtype, q.shape), scale,
                           _ptr(dq, q.dtype, q.shape), _ptr(dk, q.dtype, q.shape), _ptr(dv, q.dtype, q.shape),
                           _ptr(d_rpb, torch.float32, _rpb_shape(q, kernel)) if d_rpb is not None else None,
                           _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))
    return dq, dk, dv, d_rpb


def na2d_fused_bwd(q, k_, v, rpb, scale: float, lse, dout, kernel: int, dq, dk, dv, d_rpb, workspace):
    p = _problem_of(q, kernel)
    _check(load().na2d_fused_bwd(ctypes.byref(p), _ptr(q), _ptr(k_, q.dtype, q.shape), _ptr(v, q.dtype, q.shape),
                                 _ptr(rpb, q.dtype, _rpb_shape(q, kernel)) if rpb is not None else None, scale,
                                 _ptr(lse, torch.float32, q.shape[:4]), _ptr(dout, q.dtype, q.shape),
                                 _ptr(dq, q.dtype, q.shape), _ptr(dk, q.dtype, q.shape), _ptr(dv, q.dtype, q.shape),
                                 _ptr(d_rpb, torch.float32, _rpb_shape(q, kernel)) if d_rpb is not None else None,
                                 _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))
    return dq, dk, dv, d_rpb


def na2d_direct_bwd_workspace_bytes(p: Na2dProblem) -> int:
    """Bytes na2d_direct_bwd needs; 0 where it does not take the problem."""
    return int(load().na2d_direct_bwd_workspace_bytes(ctypes.byref(p)))


def na2d_direct_bwd(q, k_, v, rpb, scale: float, lse, dout, kernel: int, dq, dk, dv, d_rpb, workspace):
    p = _problem_of(q, kernel)
    _check(load().na2d_direct_bwd(ctypes.byref(p), _ptr(q), _ptr(k_, q.dtype, q.shape), _ptr(v, q.dtype, q.shape),
                                 _ptr(rpb, q.dtype, _rpb_shape(q, kernel)) if rpb is not None else None, scale,
                                 _ptr(lse, torch.float32, q.shape[:4]), _ptr(dout, q.dtype, q.shape),
                                 _ptr(dq, q.dtype, q.shape), _ptr(dk, q.dtype, q.shape), _ptr(dv, q.dtype, q.shape),
                                 _ptr(d_rpb, torch.float32, _rpb_shape(q, kernel)) if d_rpb is not None else None,
                                 _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))
    return dq, dk, dv, d_rpb


def na2d_fused_bwd_is_fused(p: Na2dProblem) -> int:
    return int(load().na2d_fused_bwd_is_fused(ctypes.byref(p)))


def na2d_debug_indices(H: int, W: int, kernel: int, key_index, rpb_index):
    p = problem(1, 1, H, W, 32, kernel, torch.float32)
    shape = (H, W, kernel * kernel)
    _check(load().na2d_debug_indices(ctypes.byref(p),
                                     _ptr(key_index, torch.int32, shape) if key_index is not None else None,
                                     _ptr(rpb_index, torch.int32, shape) if rpb_index is not None else None,
                                     _stream()))
    return key_index, rpb_index


def na2d_host_axis_tables(L: int, kernel: int):
    """(start, qs, qe) int32 numpy arrays of length L, computed on the host by the library."""
    import numpy as np
    start, qs, qe = (np.empty(L, dtype=np.int32) for _ in range(3))
    _check(load().na2d_host_axis_tables(L, kernel, start.ctypes.data, qs.ctypes.data, qe.ctypes.data))
    return start, qs, qe


def na2d_validate_problem(p: Na2dProblem) -> int:
    return int(load().na2d_validate_problem(ctypes.byref(p)))


def na2d_version() -> int:
    return int(load().na2d_version())


# ---- 1D entry points (include/na1d.h): tensors are [B, heads, L, D], [B, heads, L, k], [heads, 2k-1] ----------

def problem_1d(B: int, heads: int, L: int, D: int, k: int, dtype) -> Na1dProblem:
    code = DTYPE_CODES[dtype] if dtype in DTYPE_CODES else int(dtype)
    return Na1dProblem(B, heads, L, D, k, code)


def _p1(x: torch.Tensor, k: int) -> Na1dProblem:
    if x.dim() != 4:
        raise ValueError("expected a [B, heads, L, D] tensor")
    B, heads, L, D = x.shape
    return problem_1d(B, heads, L, D, k, x.dtype)


def _attn1(x, k):
    return (*x.shape[:3], k)


def _rpb1(x, k):
    return (x.shape[1], 2 * k - 1)


def na1d_validate_problem(p: Na1dProblem) -> int:
    return int(load().na1d_validate_problem(ctypes.byref(p)))


def na1d_qk_rpb(q, k_, rpb, scale: float, kernel: int, logits):
    p = _p1(q, kernel)
    _check(load().na1d_qk_rpb(ctypes.byref(p), _ptr(q), _ptr(k_, q.dtype, q.shape),
                              _ptr(rpb, q.dtype, _rpb1(q, kernel)) if rpb is not None else None, scale,
                              _ptr(logits, q.dtype, _attn1(q, kernel)), _stream()))
    return logits


def na1d_softmax(logits, kernel: int, like, out):
    p = _p1(like, kernel)
    _check(load().na1d_softmax(ctypes.byref(p), _ptr(logits, like.dtype, _attn1(like, kernel)),
                               _ptr(out, like.dtype, _attn1(like, kernel)), _stream()))
    return out


def na1d_av(attn, v, kernel: int, out):
    p = _p1(v, kernel)
    _check(load().na1d_av(ctypes.byref(p), _ptr(attn, v.dtype, _attn1(v, kernel)), _ptr(v), _ptr(out, v.dtype, v.shape),
                          _stream()))
    return out


def na1d_fused_fwd(q, k_, v, rpb, scale: float, kernel: int, out, lse=None):
    p = _p1(q, kernel)
    _check(load().na1d_fused_fwd(ctypes.byref(p), _ptr(q), _ptr(k_, q.dtype, q.shape), _ptr(v, q.dtype, q.shape),
                                 _ptr(rpb, q.dtype, _rpb1(q, kernel)) if rpb is not None else None, scale,
                                 _ptr(out, q.dtype, q.shape),
                                 _ptr(lse, torch.float32, q.shape[:3]) if lse is not None else None, _stream()))
    return out


def na1d_av_bwd_p(dout, v, kernel: int, dp):
    p = _p1(v, kernel)
    _check(load().na1d_av_bwd_p(ctypes.byref(p), _ptr(dout, v.dtype, v.shape), _ptr(v), _ptr(dp, v.dtype, _attn1(v, kernel)),
                                _stream()))
    return dp


def na1d_av_bwd_v(attn, dout, kernel: int, dv):
    p = _p1(dout, kernel)
    _check(load().na1d_av_bwd_v(ctypes.byref(p), _ptr(attn, dout.dtype, _attn1(dout, kernel)), _ptr(dout),
                                _ptr(dv, dout.dtype, dout.shape), _stream()))
    return dv


def na1d_softmax_bwd(attn, dp, kernel: int, like, ds):
    p = _p1(like, kernel)
    shape = _attn1(like, kernel)
    _check(load().na1d_softmax_bwd(ctypes.byref(p), _ptr(attn, like.dtype, shape), _ptr(dp, like.dtype, shape),
                                   _ptr(ds, like.dtype, shape), _stream()))
    return ds


def na1d_qk_bwd_q(ds, k_, scale: float, kernel: int, dq):
    p = _p1(k_, kernel)
    _check(load().na1d_qk_bwd_q(ctypes.byref(p), _ptr(ds, k_.dtype, _attn1(k_, kernel)), _ptr(k_), scale,
                                _ptr(dq, k_.dtype, k_.shape), _stream()))
    return dq


def na1d_qk_bwd_k(ds, q, scale: float, kernel: int, dk):
    p = _p1(q, kernel)
    _check(load().na1d_qk_bwd_k(ctypes.byref(p), _ptr(ds, q.dtype, _attn1(q, kernel)), _ptr(q), scale,
                                _ptr(dk, q.dtype, q.shape), _stream()))
    return dk


def na1d_workspace_bytes(p: Na1dProblem) -> int:
    return int(load().na1d_workspace_bytes(ctypes.byref(p)))


def na1d_qk_bwd_rpb(ds, kernel: int, like, d_rpb, workspace):
    p = _p1(like, kernel)
    _check(load().na1d_qk_bwd_rpb(ctypes.byref(p), _ptr(ds, like.dtype, _attn1(like, kernel)),
                                  _ptr(d_rpb, torch.float32, _rpb1(like, kernel)), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream()))
    return d_rpb


def na1d_fused_bwd_workspace_bytes(p: Na1dProblem) -> int:
    return int(load().na1d_fused_bwd_workspace_bytes(ctypes.byref(p)))


def na1d_fused_bwd(q, k_, v, rpb, scale: float, lse, dout, kernel: int, dq, dk, dv, d_rpb, workspace):
    p = _p1(q, kernel)
    _check(load().na1d_fused_bwd(ctypes.byref(p), _ptr(q), _ptr(k_, q.dtype, q.shape), _ptr(v, q.dtype, q.shape),
                                 _ptr(rpb, q.dtype, _rpb1(q, kernel)) if rpb is not None else None, scale,
                                 _ptr(lse, torch.float32, q.shape[:3]), _ptr(dout, q.dtype, q.shape),
                                 _ptr(dq, q.dtype, q.shape), _ptr(dk, q.dtype, q.shape), _ptr(dv, q.dtype, q.shape),
                                 _ptr(d_rpb, torch.float32, _rpb1(q, kernel)) if d_rpb is not None else None,
                                 _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))
    return dq, dk, dv, d_rpb


# ---- attention over sequences and its cache (include/seq.h) ---------------------------------------------------------------
# q, out: [B, heads, Lq, D]; k, v: [B, kv_heads, Lk, D], with strides of their own but for the last dimension's.

def _strided(t, of, shape, dtype=None):
    """Checks of a tensor that may have strides, and its pointer."""
    if not t.is_cuda:
        raise ValueError("na2d takes GPU tensors only")
    if t.device != of.device:
        raise ValueError(f"expected a tensor on {of.device}, got one on {t.device}")
    if t.is_neg():
        raise ValueError("na2d does not take negated views")
    if t.dtype != (of.dtype if dtype is None else dtype):
        raise ValueError(f"expected dtype {of.dtype if dtype is None else dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.stride(-1) != 1 and t.shape[-1] != 1:
        raise ValueError("the elements of a row must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _dense(t, of, shape, dtype):
    if t is None:
        return None
    p = _strided(t, of, shape, dtype)
    if not t.is_contiguous():
        raise ValueError("na2d takes contiguous tensors only")
    return p


def _seq_strides(t) -> SeqStrides:
    return SeqStrides(*(0 if n == 1 else s for n, s in zip(t.shape[:3], t.stride()[:3])))


def _seq_stream(t):
    return ctypes.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)


def seq_problem(q, k_, *, causal: bool, window: int, softcap: float, scale: float, **strided) -> SeqProblem:
    """strided: the tensors by name (v, out and, backward, dout, dq, dk, dv)."""
    if q.dim() != 4 or k_.dim() != 4:
        raise ValueError("expected [B, heads, L, D] tensors")
    (B, heads, Lq, D), (_, kv_heads, Lk, _) = q.shape, k_.shape
    code = DTYPE_CODES.get(q.dtype, -1)
    p = SeqProblem(B, heads, kv_heads, Lq, Lk, D, code, int(causal), int(window), scale, softcap)
    for name, t in dict(q=q, k=k_, **strided).items():
        setattr(p, name, _seq_strides(t))
    return p


def seq_validate_problem(p: SeqProblem, backward: bool = False) -> int:
    return int(load().seq_validate_problem(ctypes.byref(p), int(backward)))


def seq_attention_workspace_bytes(p: SeqProblem, marked: bool, backward: bool = False) -> int:
    return int(load().seq_attention_workspace_bytes(ctypes.byref(p), int(marked), int(backward)))


def _seq_inputs(q, k_, v, slopes, documents, prefix):
    B, heads, Lq, D = q.shape
    kv_shape = (B, k_.shape[1], k_.shape[2], D)
    return (_strided(q, q, q.shape), _strided(k_, q, kv_shape), _strided(v, q, kv_shape), _dense(slopes, q, (heads,), torch.float32),
            _dense(documents, q, (B, k_.shape[2]), torch.int32), _dense(prefix, q, (B, k_.shape[2]), torch.bool))


def _bytes(workspace):
    return (None, 0) if workspace is None else (ctypes.c_void_p(workspace.data_ptr()), workspace.numel() * workspace.element_size())


def _rest(rest, out):
    if rest is None:
        return None
    if rest.stride() != out.stride():
        raise ValueError("rest has out's strides")
    return _strided(rest, out, out.shape)


def seq_attention_fwd(q, k_, v, slopes, documents, prefix, out, lse=None, rest=None, workspace=None, *, causal=False, window=0, softcap=0.0, scale=1.0):
    p = seq_problem(q, k_, causal=causal, window=window, softcap=softcap, scale=scale, v=v, out=out)
    inputs = _seq_inputs(q, k_, v, slopes, documents, prefix)
    with torch.cuda.device(q.device):
        _check(load().seq_attention_fwd(ctypes.byref(p), *inputs, _strided(out, q, q.shape), _dense(lse, q, q.shape[:3], torch.float32), _rest(rest, out),
                                        *_bytes(workspace), _seq_stream(q)))
    return out


def seq_attention_bwd(q, k_, v, slopes, documents, prefix, out, lse, rest, dout, dq, dk, dv, workspace, *, causal=False, window=0, softcap=0.0, scale=1.0):
    p = seq_problem(q, k_, causal=causal, window=window, softcap=softcap, scale=scale, v=v, out=out, dout=dout, dq=dq, dk=dk, dv=dv)
    inputs = _seq_inputs(q, k_, v, slopes, documents, prefix)
    with torch.cuda.device(q.device):
        _check(load().seq_attention_bwd(ctypes.byref(p), *inputs, _strided(out, q, q.shape), _dense(lse, q, q.shape[:3], torch.float32), _rest(rest, out), _strided(dout, q, q.shape),
                                        _strided(dq, q, q.shape), _strided(dk, q, k_.shape), _strided(dv, q, k_.shape), *_bytes(workspace), _seq_stream(q)))
    return dq, dk, dv


def seq_rotation(dtype, *, sections, weights=(), eps=1e-6, interleaved=False) -> SeqRotation:
    """sections: pairs of each axis; none for no rotation.  weights: those that are given have one type."""
    kinds = {w.dtype for w in weights if w is not None}
    if len(kinds) > 1:
        raise ValueError(f"weights of one dtype are expected, got {sorted(map(str, kinds))}")
    if len(sections) > 4:
        raise ValueError(f"at most 4 axes, got {len(sections)}")
    return SeqRotation(sum(sections), len(sections), (ctypes.c_int32 * 4)(*sections), int(interleaved), DTYPE_CODES.get(next(iter(kinds), dtype), -1), eps)


def seq_rotary_problem(q, k_, positions, rotation: SeqRotation, **strided) -> SeqRotaryProblem:
    """q: [B, heads, L, D]; k_: [B, kv_heads, L, D] or None; strided: other tensors by name (q_out, k_out, dq, dk)."""
    if q.dim() != 4 or (k_ is not None and k_.dim() != 4):
        raise ValueError("expected [B, heads, L, D] tensors")
    B, heads, L, D = q.shape
    p = SeqRotaryProblem(B, heads, 0 if k_ is None else k_.shape[1], L, D, DTYPE_CODES.get(q.dtype, -1), rotation, int(positions.dim() == 2))
    for name, t in dict(q=q, k=k_, **strided).items():
        if t is not None:
            setattr(p, name, _seq_strides(t))
    return p


def seq_rotary_validate(p: SeqRotaryProblem, backward: bool = False) -> int:
    return int(load().seq_rotary_validate(ctypes.byref(p), int(backward)))


def seq_rotary_bwd_workspace_bytes(p: SeqRotaryProblem) -> int:
    return int(load().seq_rotary_bwd_workspace_bytes(ctypes.byref(p)))


def _axis_positions(positions, of, B, axes, L):
    return _dense(positions, of, (axes, L) if positions.dim() == 2 else (B, axes, L), torch.int32)


def _rotary_inputs(q, k_, positions, freqs, q_weight, k_weight, rotation):
    B, _, L, D = q.shape
    weight = lambda w: None if w is None else _dense(w, q, (D,), w.dtype)
    return (_strided(q, q, q.shape), None if k_ is None else _strided(k_, q, (B, k_.shape[1], L, D)), _axis_positions(positions, q, B, rotation.axes, L),
            _dense(freqs, q, (rotation.pairs,), torch.float32), weight(q_weight), weight(k_weight))


def seq_rotary_fwd(q, k_, positions, freqs, q_weight, k_weight, q_out, k_out, *, sections, eps=1e-6, interleaved=False):
    rotation = seq_rotation(q.dtype, sections=sections, weights=(q_weight, k_weight), eps=eps, interleaved=interleaved)
    p = seq_rotary_problem(q, k_, positions, rotation, q_out=q_out, k_out=k_out)
    inputs = _rotary_inputs(q, k_, positions, freqs, q_weight, k_weight, rotation)
    with torch.cuda.device(q.device):
        _check(load().seq_rotary_fwd(ctypes.byref(p), *inputs, _strided(q_out, q, q.shape), None if k_ is None else _strided(k_out, q, k_.shape), _seq_stream(q)))
    return q_out, k_out


def seq_rotary_bwd(q, k_, positions, freqs, q_weight, k_weight, dq_out, dk_out, dq, dk, dq_weight, dk_weight, workspace=None, *, sections, eps=1e-6, interleaved=False):
    """q, k_: as in the forward pass (only their form counts where there is no weight)."""
    rotation = seq_rotation(q.dtype, sections=sections, weights=(q_weight, k_weight), eps=eps, interleaved=interleaved)
    p = seq_rotary_problem(q, k_, positions, rotation, q_out=dq_out, k_out=dk_out, dq=dq, dk=dk)
    inputs = _rotary_inputs(q, k_, positions, freqs, q_weight, k_weight, rotation)
    side = lambda t: None if k_ is None else _strided(t, q, k_.shape)
    grad = lambda t, w: None if w is None else _dense(t, q, w.shape, w.dtype)
    with torch.cuda.device(q.device):
        _check(load().seq_rotary_bwd(ctypes.byref(p), *inputs, _strided(dq_out, q, q.shape), side(dk_out), _strided(dq, q, q.shape), side(dk), grad(dq_weight, q_weight),
                                     grad(dk_weight, k_weight), *_bytes(workspace), _seq_stream(q)))
    return dq, dk, dq_weight, dk_weight


def seq_cache_problem(rows, k_pages, table, *, heads=None, window=0, softcap=0.0, scale=1.0, out=None) -> SeqCacheProblem:
    """rows: [B, heads or kv_heads, n, D]; out: the call's other tensor of that form."""
    if rows.dim() != 4 or k_pages.dim() != 4 or table.dim() != 2:
        raise ValueError("expected [B, heads, n, D] rows, [pages, kv_heads, page, D] pages and a [B, width] table")
    (B, _, n, D), (pages, kv_heads, page, _) = rows.shape, k_pages.shape
    p = SeqCacheProblem(B, kv_heads if heads is None else heads, kv_heads, D, page, pages, table.shape[1], DTYPE_CODES.get(rows.dtype, -1), n, int(window), scale, softcap)
    p.q, p.out = _seq_strides(rows), _seq_strides(rows if out is None else out)
    return p


def seq_cache_validate(p: SeqCacheProblem, call: int) -> int:
    """call: SEQ_CACHE_APPEND, SEQ_CACHE_GATHER or SEQ_CACHE_ATTENTION."""
    return int(load().seq_cache_validate(ctypes.byref(p), call))


def _cache_inputs(rows, k_pages, v_pages, k_scales, v_scales):
    pages, kv_heads, page, _ = k_pages.shape
    shape = (pages, kv_heads, page, rows.shape[3])
    return (_dense(k_pages, rows, shape, torch.int8), _dense(v_pages, rows, shape, torch.int8), _dense(k_scales, rows, shape[:2], torch.float32),
            _dense(v_scales, rows, shape[:2], torch.float32))


def seq_cache_append(k_, v, table, lengths, counts, k_pages, v_pages, k_scales, v_scales):
    p = seq_cache_problem(k_, k_pages, table, out=v)
    B, shape = k_.shape[0], (k_.shape[0], k_pages.shape[1], *k_.shape[2:])
    cache = _cache_inputs(k_, k_pages, v_pages, k_scales, v_scales)
    with torch.cuda.device(k_.device):
        _check(load().seq_cache_append(ctypes.byref(p), _strided(k_, k_, shape), _strided(v, k_, shape), _dense(table, k_, (B, table.shape[1]), torch.int32),
                                       _dense(lengths, k_, (B,), torch.int32), _dense(counts, k_, (B,), torch.int32), *cache, _seq_stream(k_)))


def seq_cache_append_rows(k_, v, table, lengths, counts, k_pages, v_pages, k_scales, v_scales, *, rows=None, positions=None, freqs=None, weight=None, sections=(), eps=1e-6,
                          interleaved=False):
    """k_, v: the given rows [B, kv_heads, given, D]; rows: int32 [B, n] or None."""
    p = seq_cache_problem(k_, k_pages, table, out=v)
    B, given, shape = k_.shape[0], k_.shape[2], (k_.shape[0], k_pages.shape[1], *k_.shape[2:])
    if rows is not None:
        if rows.dim() != 2:
            raise ValueError("expected rows [B, n]")
        p.n = rows.shape[1]
    rotation = seq_rotation(k_.dtype, sections=sections, weights=(weight,), eps=eps, interleaved=interleaved)
    cache = _cache_inputs(k_, k_pages, v_pages, k_scales, v_scales)
    int32 = lambda t, s: _dense(t, k_, s, torch.int32)
    with torch.cuda.device(k_.device):
        _check(load().seq_cache_append_rows(
            ctypes.byref(p), ctypes.byref(rotation), given, _strided(k_, k_, shape), _strided(v, k_, shape), int32(rows, None if rows is None else (B, rows.shape[1])),
            None if positions is None else _axis_positions(positions, k_, B, rotation.axes, given), int(positions is not None and positions.dim() == 2),
            _dense(freqs, k_, (rotation.pairs,), torch.float32), None if weight is None else _dense(weight, k_, (k_.shape[3],), weight.dtype),
            int32(table, (B, table.shape[1])), int32(lengths, (B,)), int32(counts, (B,)), *cache, _seq_stream(k_)))


def seq_cache_gather(k_pages, v_pages, k_scales, v_scales, table, lengths, first, k_, v):
    p = seq_cache_problem(k_, k_pages, table, out=v)
    B, shape = k_.shape[0], (k_.shape[0], k_pages.shape[1], *k_.shape[2:])
    cache = _cache_inputs(k_, k_pages, v_pages, k_scales, v_scales)
    with torch.cuda.device(k_.device):
        _check(load().seq_cache_gather(ctypes.byref(p), *cache, _dense(table, k_, (B, table.shape[1]), torch.int32), _dense(lengths, k_, (B,), torch.int32),
                                       _dense(first, k_, (B,), torch.int32), _strided(k_, k_, shape), _strided(v, k_, shape), _seq_stream(k_)))
    return k_, v


def seq_cache_attention_workspace_bytes(p: SeqCacheProblem) -> int:
    return int(load().seq_cache_attention_workspace_bytes(ctypes.byref(p)))


def seq_cache_attention(q, k_pages, v_pages, k_scales, v_scales, table, lengths, slopes, out, workspace=None, *, window=0, softcap=0.0, scale=1.0):
    p = seq_cache_problem(q, k_pages, table, heads=q.shape[1], window=window, softcap=softcap, scale=scale, out=out)
    B = q.shape[0]
    cache = _cache_inputs(q, k_pages, v_pages, k_scales, v_scales)
    with torch.cuda.device(q.device):
        _check(load().seq_cache_attention(ctypes.byref(p), _strided(q, q, q.shape), *cache, _dense(table, q, (B, table.shape[1]), torch.int32),
                                          _dense(lengths, q, (B,), torch.int32), _dense(slopes, q, (q.shape[1],), torch.float32), _strided(out, q, q.shape),
                                          *_bytes(workspace), _seq_stream(q)))
    return out


def seq_cache_tree_attention_workspace_bytes(p: SeqCacheProblem) -> int:
    return int(load().seq_cache_tree_attention_workspace_bytes(ctypes.byref(p)))


def seq_cache_tree_attention(q, k_, v, parents, k_pages, v_pages, k_scales, v_scales, table, lengths, slopes, out, workspace, *, window=0, softcap=0.0, scale=1.0):
    p = seq_cache_problem(q, k_pages, table, heads=q.shape[1], window=window, softcap=softcap, scale=scale, out=out)
    B, _, n, D = q.shape
    shape, cache = (B, k_pages.shape[1], n, D), _cache_inputs(q, k_pages, v_pages, k_scales, v_scales)
    inputs = (_strided(q, q, q.shape), _strided(k_, q, shape), _strided(v, q, shape), _dense(parents, q, (B, n), torch.int32))
    ks, vs = _seq_strides(k_), _seq_strides(v)
    with torch.cuda.device(q.device):
        _check(load().seq_cache_tree_attention(ctypes.byref(p), ctypes.byref(ks), ctypes.byref(vs), *inputs, *cache, _dense(table, q, (B, table.shape[1]), torch.int32),
                                               _dense(lengths, q, (B,), torch.int32), _dense(slopes, q, (q.shape[1],), torch.float32), _strided(out, q, q.shape), *_bytes(workspace),
                                               _seq_stream(q)))
    return out


def seq_verify_problem(logits, draft=None) -> SeqVerifyProblem:
    if logits.dim() != 3 or (draft is not None and draft.dim() != 3):
        raise ValueError("expected [B, n, V] logits and [B, n - 1, V] logits of a draft")
    B, n, V = logits.shape
    p = SeqVerifyProblem(B, n, V, DTYPE_CODES.get(logits.dtype, -1), int(draft is not None), *_row_strides(logits))
    if draft is not None:
        p.draft_batch, p.draft_row = _row_strides(draft)
    return p


def _row_strides(t):
    return tuple(0 if n <= 1 else s for n, s in zip(t.shape[:2], t.stride()[:2]))


def seq_verify_validate(p: SeqVerifyProblem) -> int:
    return int(load().seq_verify_validate(ctypes.byref(p)))


def seq_verify_workspace_bytes(p: SeqVerifyProblem) -> int:
    return int(load().seq_verify_workspace_bytes(ctypes.byref(p)))


def seq_verify(logits, draft, tokens, parents, uniforms, temperatures, path, counts, next_, workspace):
    p = seq_verify_problem(logits, draft)
    B, n, V = logits.shape
    int32 = lambda t, shape: _dense(t, logits, shape, torch.int32)
    f32 = lambda t, shape: _dense(t, logits, shape, torch.float32)
    inputs = (_strided(logits, logits, logits.shape), None if draft is None else _strided(draft, logits, (B, n - 1, V)), int32(tokens, (B, n)), int32(parents, (B, n)),
              f32(uniforms, (B, n if draft is None else n + 1)), f32(temperatures, (B,)))
    with torch.cuda.device(logits.device):
        _check(load().seq_verify(ctypes.byref(p), *inputs, int32(path, (B, n)), int32(counts, (B,)), int32(next_, (B,)), *_bytes(workspace), _seq_stream(logits)))
    return path, counts, next_
