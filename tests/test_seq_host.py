"""Refusals of the attention over sequences and of its cache, before any GPU call (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2204_07143_amd import binding as na
from paper_2204_07143_amd import functional as F

from test_host_abi import declared_symbols


def test_library_exports_every_declared_symbol():
    lib, names = na.load(), declared_symbols("seq.h", "seq_")
    assert sorted(na.EXPORTS_SEQ) == names and all(hasattr(lib, n) for n in names)


def P(B=2, heads=4, kv=2, Lq=100, Lk=100, D=64, dtype=1, causal=1, window=0, scale=0.125, cap=0.0, **strides):
    p = na.SeqProblem(B, heads, kv, Lq, Lk, D, dtype, causal, window, scale, cap)
    for n in ("q", "out", "dout", "dq"):
        setattr(p, n, strides.get(n, na.SeqStrides(heads * Lq * D, Lq * D, D)))
    for n in ("k", "v", "dk", "dv"):
        setattr(p, n, strides.get(n, na.SeqStrides(kv * Lk * D, Lk * D, D)))
    return p


@pytest.mark.parametrize("problem,code", [
    (P(), 0), (P(Lq=1, Lk=1 << 24, kv=1, heads=1, B=1, D=32), 0), (P(window=5, cap=30.0), 0), (P(scale=-1.0), 0), (P(q=na.SeqStrides(0, 0, 64)), 0),
    (P(dtype=3), -2), (P(dtype=-1), -2), (P(D=16), -5), (P(D=96), -5),
    (P(B=0), -6), (P(heads=3), -6), (P(kv=0), -6), (P(Lq=0), -6), (P(Lk=-1), -6), (P(Lk=(1 << 24) + 1), -6), (P(causal=2), -6), (P(window=-1), -6), (P(window=(1 << 30) + 1), -6),
    (P(scale=float("nan")), -6), (P(scale=float("inf")), -6), (P(cap=-1.0), -6), (P(cap=float("nan")), -6), (P(cap=float("inf")), -6), (P(cap=5000.0), -6), (P(cap=5000.0, dtype=0), 0), (P(cap=1e-7), -6),
    (P(q=na.SeqStrides(6400, 6400, -64)), -6), (P(q=na.SeqStrides(6400, 6400, 1 << 26)), -6), (P(k=na.SeqStrides(6400, 6400, 68)), -7), (P(v=na.SeqStrides(6401, 6400, 64)), -7),
    (P(B=1 << 20, heads=1 << 12, kv=1, Lq=1 << 10), -6),
])
def test_problems(problem, code):
    assert na.seq_validate_problem(problem) == code
    assert (na.seq_attention_workspace_bytes(problem, True, True) == 0) == (code != 0)


def test_backward_strides_count_only_there():
    p = P(dk=na.SeqStrides(6400, 6400, 65))
    assert na.seq_validate_problem(p) == 0 and na.seq_validate_problem(p, True) == -7


def test_attention_arguments():
    lib, p = na.load(), P()
    at = lambda n: ctypes.c_void_p(4096 + 16 * n)
    fwd = lambda p, q=at(1), k=at(2), v=at(3), slopes=None, docs=None, prefix=None, out=at(4), lse=None, rest=None, ws=None, n=0: lib.seq_attention_fwd(
        ctypes.byref(p), q, k, v, slopes, docs, prefix, out, lse, rest, ws, n, None)
    assert lib.seq_attention_fwd(None, *[at(1)] * 10, 0, None) == -1
    assert fwd(p, q=None) == -1 and fwd(p, out=None) == -1
    assert fwd(p, v=ctypes.c_void_p(4100)) == -7 and fwd(p, slopes=ctypes.c_void_p(4098)) == -7 and fwd(p, lse=ctypes.c_void_p(4098)) == -7
    assert fwd(p, out=at(2)) == -10
    assert fwd(p, docs=at(9)) == -8 and fwd(p, prefix=at(9), ws=at(10), n=16) == -8 and fwd(p, docs=at(9), ws=ctypes.c_void_p(4100), n=1 << 20) == -8
    assert fwd(P(Lq=101), docs=at(9), ws=at(10), n=1 << 20) == -6   # documents need a position for every query
    bwd = lambda p, **x: lib.seq_attention_bwd(ctypes.byref(p), *({n: at(i + 1) for i, n in enumerate(("q", "k", "v", "slopes", "docs", "prefix", "out", "lse", "rest", "dout", "dq", "dk", "dv"))}
                                                                   | {"slopes": None, "docs": None, "prefix": None} | x).values(), None, 0, None)
    assert fwd(p, rest=at(4)) == -10 and fwd(p, rest=at(1)) == -10 and fwd(P(dtype=0), rest=at(5)) == -2
    assert bwd(p) == -8 and bwd(p, rest=at(11)) == -10 and bwd(p, dout=None) == -1 and bwd(p, lse=None) == -1 and bwd(p, dq=at(1)) == -10 and bwd(p, dk=at(13)) == -10


def C(B=2, heads=4, kv=2, D=64, page=16, pages=8, width=4, dtype=1, n=1, window=0, scale=0.1, cap=0.0, rows=None):
    p = na.SeqCacheProblem(B, heads, kv, D, page, pages, width, dtype, n, window, scale, cap)
    p.q = p.out = na.SeqStrides(heads * n * D, n * D, D) if rows is None else rows
    return p


@pytest.mark.parametrize("problem,codes", [   # append, gather, attention
    (C(), (0, 0, 0)), (C(dtype=0), (0, 0, -2)), (C(dtype=5), (-2, -2, -2)), (C(D=48), (-5,) * 3), (C(page=48), (-6,) * 3), (C(page=8), (-6,) * 3), (C(pages=0), (-6,) * 3),
    (C(width=0), (-6,) * 3), (C(width=1 << 27, page=16), (-6,) * 3), (C(n=0), (-6,) * 3), (C(heads=5), (-6,) * 3), (C(window=-2), (-6,) * 3), (C(cap=-1.0), (-6,) * 3),
    (C(rows=na.SeqStrides(256, 64, 60)), (-7,) * 3), (C(rows=na.SeqStrides(-256, 64, 64)), (-6,) * 3),
])
def test_cache_problems(problem, codes):
    assert tuple(na.seq_cache_validate(problem, call) for call in range(3)) == codes
    assert na.seq_cache_validate(problem, 3) == -6


def test_cache_arguments():
    lib, p = na.load(), C(B=1, width=1024, pages=1024)
    at = [ctypes.c_void_p(4096 + 16 * n) for n in range(12)]
    assert na.seq_cache_attention_workspace_bytes(p) > 0   # a single long sequence is split
    assert lib.seq_cache_attention(ctypes.byref(p), *at[:7], None, at[8], None, 0, None) == -8
    assert lib.seq_cache_attention(ctypes.byref(p), *at[:7], None, at[0], at[9], 1 << 30, None) == -10
    assert lib.seq_cache_attention(ctypes.byref(p), None, *at[1:7], None, at[8], None, 0, None) == -1
    assert lib.seq_cache_append(ctypes.byref(p), at[0], at[1], None, at[3], None, *at[4:8], None) == -1
    assert lib.seq_cache_append(ctypes.byref(p), at[0], at[1], at[2], at[3], None, at[4], at[4], at[6], at[7], None) == -10
    assert lib.seq_cache_append(ctypes.byref(p), at[0], ctypes.c_void_p(4100), *at[2:4], None, *at[4:8], None) == -7
    assert lib.seq_cache_gather(ctypes.byref(p), *at[:7], at[8], at[8], None) == -10
    assert lib.seq_cache_gather(ctypes.byref(p), *at[:6], None, at[8], at[9], None) == -1


@pytest.mark.parametrize("strides,ok", [   # batch, head, row of [2, 4, 100, 64]
    ((25600, 6400, 64), True), ((25600, 64, 256), True), ((6400, 12800, 64), True), ((64, 128, 512), True), ((51200, 6400, 64), True),
    ((0, 6400, 64), False), ((25600, 0, 64), False), ((25600, 6400, 0), False), ((25600, 6400, 32), False), ((25600, 6392, 64), False), ((6400, 6400, 64), False), ((25600, 64, 248), False),
    ((19200, 6400, 64), False),
])
def test_rows_of_outputs_do_not_overlap(strides, ok):
    code = 0 if ok else -10
    for name in ("q", "k", "v", "dout"):
        assert na.seq_validate_problem(P(kv=4, **{name: na.SeqStrides(*strides)}), True) == 0
    for name in ("out", "dq", "dk", "dv"):
        assert na.seq_validate_problem(P(kv=4, **{name: na.SeqStrides(*strides)}), True) == code
    rows = na.SeqStrides(*strides)
    assert tuple(na.seq_cache_validate(C(kv=4, n=100, rows=rows), call) for call in range(3)) == (0, code, code)


def test_strides_of_one_row_do_not_count():
    zero = na.SeqStrides(0, 0, 0)
    assert na.seq_validate_problem(P(B=1, heads=1, kv=1, Lq=1, Lk=1, **{n: zero for n in ("out", "dq", "dk", "dv")}), True) == 0
    assert na.seq_validate_problem(P(out=na.SeqStrides(1 << 45, 1 << 45, 64), B=1, heads=1, kv=1)) == 0
    assert na.seq_validate_problem(P(q=na.SeqStrides(1 << 45, 64, 64), B=1 << 20)) == -6   # no such address


def test_python_arguments():
    x = lambda *s, **k: torch.zeros(s, **k)
    q, kv = x(2, 4, 10, 32), x(2, 2, 10, 32)
    for bad in (dict(window=0), dict(window=2.5), dict(softcap=0.0), dict(softcap=float("inf")), dict(slopes=x(4, requires_grad=True))):
        with pytest.raises(ValueError):
            F.seq_attention(q, kv, kv, **bad)
    for args in ((q[0], kv, kv), (q, kv, kv[:, :1]), (q, x(2, 3, 10, 32), x(2, 3, 10, 32)), (q, x(1, 2, 10, 32), x(1, 2, 10, 32)), (q, x(2, 2, 10, 64), x(2, 2, 10, 64)), (q, x(2, 0, 10, 32), x(2, 0, 10, 32))):
        with pytest.raises(ValueError):
            F.seq_attention(*args)
    with pytest.raises(ValueError, match="GPU tensors only"):
        F.seq_attention(q, kv, kv)
    cache = F.SeqCache.empty(2, 2, 16, 32, device="cpu")
    table, lengths = torch.zeros((2, 1), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: F.seq_cache_append(cache, kv, kv, table, lengths), lambda: F.seq_cache_gather(cache, table, lengths, lengths, 3),
                 lambda: F.seq_cache_attention(q.half(), cache, table, lengths)):
        with pytest.raises(ValueError, match="GPU tensors only"):
            call()


def test_planes_whose_size_passes_64_bits():
    """2^22 rows 2^42 elements apart are 2^64 elements: refused, not taken for none."""
    rows, far = (1 << 22) + 1, na.SeqStrides(0, 0, 1 << 42)
    for name in ("q", "out", "dout", "dq"):
        assert na.seq_validate_problem(P(B=1, heads=1, kv=1, Lq=rows, Lk=rows, **{name: far}), True) == -6
    for name in ("k", "v", "dk", "dv"):
        assert na.seq_validate_problem(P(B=1, heads=1, kv=1, Lk=rows, **{name: far}), True) == -6
    for last in (1 << 24, (1 << 24) - 1):
        assert na.seq_validate_problem(P(B=1, heads=1, kv=1, Lq=last, q=na.SeqStrides(0, 0, 1 << 45))) == -6
    assert tuple(na.seq_cache_validate(C(B=1, heads=1, kv=1, n=rows, rows=far), call) for call in range(3)) == (-6, -6, -6)
    # the largest plane there is
    assert na.seq_validate_problem(P(B=1, heads=1, kv=1, Lq=(1 << 24) - 1, Lk=64, D=64, q=na.SeqStrides(0, 0, 64), out=na.SeqStrides(0, 0, 64))) == 0
    assert na.seq_validate_problem(P(B=1, heads=1, kv=1, Lq=1 << 24, Lk=64, D=64, q=na.SeqStrides(0, 0, 64), out=na.SeqStrides(0, 0, 64))) == -6


@pytest.mark.parametrize("scale,cap,code", [(2.35e38, 0.0, 0), (2.4e38, 0.0, -6), (-2.4e38, 0.0, -6), (2e34, 1e-4, -6), (1e34, 1e-4, 0), (3e38, 50.0, 0), (-1e33, 2.0 ** -20, -6)])
def test_scales_that_pass_fp32_on_the_way_to_base_2(scale, cap, code):
    assert na.seq_validate_problem(P(scale=scale, cap=cap)) == code
    assert tuple(na.seq_cache_validate(C(scale=scale, cap=cap), call) for call in range(3)) == (code,) * 3


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_as_many_tiles_as_a_launch_holds(dtype):
    """2^24 - 1 workgroups of 256: of queries and of keys each, in either pass; fp16's backward pass forms the keys' sizes beside the queries'."""
    most = (1 << 24) - 1
    for B, heads, L, code in ((most, 1, 64, 0), (1 << 12, 1 << 12, 64, -6), ((1 << 24) - 2, 1, 1, 0), (1 << 23, 1, 65, -6)):
        p = P(B=B, heads=heads, kv=heads, Lq=L, Lk=L, D=32, dtype=dtype, **{n: na.SeqStrides(heads * L * 32, L * 32, 32) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")})
        assert na.seq_validate_problem(p) == code, (B, heads, L)
        assert na.seq_validate_problem(p, True) == (-6 if dtype == 1 and B == most else code), (B, heads, L)
