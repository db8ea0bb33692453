"""Refusals of the rotation by position and of the append that rotates, before any GPU call (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2204_07143_amd import binding as na
from paper_2204_07143_amd import functional as F


def R(pairs=16, sections=(16,), interleaved=0, weight_dtype=1, eps=1e-6, axes=None):
    return na.SeqRotation(pairs, len(sections) if axes is None else axes, (ctypes.c_int32 * 4)(*sections), interleaved, weight_dtype, eps)


def P(B=2, heads=4, kv=2, L=10, D=64, dtype=1, rotation=None, shared=1, **strides):
    p = na.SeqRotaryProblem(B, heads, kv, L, D, dtype, R() if rotation is None else rotation, shared)
    for n in ("q", "q_out", "dq"):
        setattr(p, n, strides.get(n, na.SeqStrides(heads * L * D, L * D, D)))
    for n in ("k", "k_out", "dk"):
        setattr(p, n, strides.get(n, na.SeqStrides(kv * L * D, L * D, D)))
    return p


@pytest.mark.parametrize("problem,code", [
    (P(), 0), (P(kv=0), 0), (P(kv=3), 0), (P(D=16, rotation=R(8, (3, 5))), 0), (P(rotation=R(32, (8, 8, 8, 8), 1)), 0), (P(q=na.SeqStrides(0, 0, 0)), 0), (P(rotation=R(weight_dtype=7)), 0),
    (P(dtype=4), -2), (P(D=48), -5), (P(D=256), -5), (P(B=0), -6), (P(heads=0), -6), (P(kv=-1), -6), (P(L=0), -6), (P(B=1 << 16, L=1 << 15), -6), (P(shared=2), -6),
    (P(rotation=R(40, (40,))), -6), (P(rotation=R(0, ())), -6), (P(rotation=R(12, (12,))), -6), (P(rotation=R(-8, (-8,))), -6), (P(rotation=R(16, (8, 4))), -6), (P(rotation=R(16, (16, 0))), -6),
    (P(rotation=R(16, (24, -8))), -6), (P(rotation=R(axes=0)), -6), (P(rotation=R(axes=5)), -6), (P(rotation=R(interleaved=2)), -6),
    (P(q_out=na.SeqStrides(0, 640, 64)), -10), (P(k=na.SeqStrides(1280, 640, 60)), -7), (P(q=na.SeqStrides(-640, 640, 64)), -6), (P(k_out=na.SeqStrides(1280, 640, 32)), -10),
])
def test_problems(problem, code):
    assert na.seq_rotary_validate(problem) == code
    if code not in (0, -10):   # (rows of q_out and k_out are read in the backward pass, and may overlap)
        assert na.seq_rotary_bwd_workspace_bytes(problem) == 0


def test_backward_strides_count_only_there():
    assert na.seq_rotary_validate(P(dq=na.SeqStrides(0, 640, 64))) == 0 and na.seq_rotary_validate(P(dq=na.SeqStrides(0, 640, 64)), True) == -10
    assert na.seq_rotary_validate(P(q_out=na.SeqStrides(0, 0, 0)), True) == 0   # an upstream gradient may be broadcast
    assert na.seq_rotary_validate(P(kv=0, dk=na.SeqStrides(0, 0, 1)), True) == 0


def test_arguments():
    lib, at = na.load(), lambda n: ctypes.c_void_p(4096 + 16 * n)
    names = ("q", "k", "positions", "freqs", "qw", "kw", "q_out", "k_out")
    fwd = lambda p=P(), **x: lib.seq_rotary_fwd(ctypes.byref(p), *({n: at(i) for i, n in enumerate(names)} | x).values(), None)
    assert lib.seq_rotary_fwd(None, *[at(1)] * 8, None) == -1
    for name in ("q", "k", "positions", "freqs", "q_out", "k_out"):
        assert fwd(**{name: None}) == -1
    assert fwd(q=ctypes.c_void_p(4100)) == -7 and fwd(freqs=ctypes.c_void_p(4098)) == -7 and fwd(qw=ctypes.c_void_p(4097)) == -7
    assert fwd(q_out=at(0)) == -10 and fwd(q_out=at(7)) == -10 and fwd(k_out=at(0)) == -10
    assert fwd(P(kv=0)) == -6 and fwd(P(kv=0), k=None, k_out=None) == -6   # a weight of keys that are not there
    for bad, code in ((R(weight_dtype=2), -2), (R(eps=0.0), -6), (R(eps=float("nan")), -6), (R(eps=float("inf")), -6), (R(eps=-1.0), -6)):
        assert fwd(P(rotation=bad)) == code
    names_b = ("q", "k", "positions", "freqs", "qw", "kw", "dq_out", "dk_out", "dq", "dk", "dqw", "dkw")
    bwd = lambda p=P(), ws=None, n=0, **x: lib.seq_rotary_bwd(ctypes.byref(p), *({m: at(i) for i, m in enumerate(names_b)} | x).values(), ws, n, None)
    need = na.seq_rotary_bwd_workspace_bytes(P())
    assert need > 0 and bwd() == -8 and bwd(ws=at(20), n=need - 1) == -8 and bwd(ws=ctypes.c_void_p(4100), n=need) == -8
    for name in ("q", "k", "dqw", "dkw", "dq", "dk", "dq_out", "dk_out"):
        assert bwd(**{name: None}) == -1
    assert bwd(dq=at(6)) == -10 and bwd(dk=at(8)) == -10 and bwd(dqw=at(4)) == -10 and bwd(dkw=at(10)) == -10


def C(n=4, given=4, **x):
    p = na.SeqCacheProblem(*({"B": 2, "heads": 2, "kv": 2, "D": 64, "page": 16, "pages": 8, "width": 4, "dtype": 1, "n": n, "window": 0, "scale": 1.0, "cap": 0.0} | x).values())
    p.q = p.out = na.SeqStrides(2 * given * 64, given * 64, 64)
    return p


def test_append_arguments():
    lib, at = na.load(), lambda n: ctypes.c_void_p(4096 + 16 * n)
    names = ("k", "v", "rows", "positions", "shared", "freqs", "weight", "table", "lengths", "counts", "kp", "vp", "ks", "vs")

    def call(p=C(), r=R(), given=4, **x):
        values = {n: at(i) for i, n in enumerate(names)} | {"shared": 1} | x
        return lib.seq_cache_append_rows(ctypes.byref(p), None if r is None else ctypes.byref(r), given, *values.values(), None)
    for name in ("k", "v", "freqs", "table", "lengths", "kp", "vp", "ks", "vs"):
        assert call(**{name: None}) == -1
    assert call(given=0) == -6 and call(given=3, rows=None) == -6 and call(shared=2) == -6 and call(C(n=0)) == -6 and call(C(D=48)) == -5 and call(C(page=48)) == -6 and call(C(dtype=9)) == -2
    assert call(r=None) == -1   # a weight, without how
    assert call(r=R(16, (8, 8)), positions=None) == -6 and call(r=R(40, (40,))) == -6 and call(r=R(eps=0.0)) == -6 and call(r=R(weight_dtype=0), weight=ctypes.c_void_p(4098)) == -7
    assert call(rows=ctypes.c_void_p(4097)) == -7 and call(vp=at(10)) == -10


def test_python_arguments():
    x = lambda *s, **k: torch.zeros(s, **k)
    q, k, positions, freqs = x(2, 4, 10, 32), x(2, 2, 10, 32), torch.zeros((1, 10), dtype=torch.int32), torch.ones(16)
    for bad in (dict(sections=(8, 4)), dict(sections=()), dict(sections=(16, 0)), dict(sections=(4, 4, 4, 2, 2))):
        with pytest.raises(ValueError):
            F.seq_rotary(q, k, positions, freqs, **bad)
    for args in ((q[0], k, positions, freqs), (q, k[:, :, :5], positions, freqs), (q, x(1, 2, 10, 32), positions, freqs), (q, k, positions[0], freqs), (q, k, positions, freqs.requires_grad_())):
        with pytest.raises(ValueError):
            F.seq_rotary(*args)
    freqs = freqs.detach()
    with pytest.raises(ValueError, match="not given"):
        F.seq_rotary(q, None, positions, freqs, k_weight=x(32))
    with pytest.raises(ValueError, match="one dtype"):
        F.seq_rotary(q, k, positions, freqs, q_weight=x(32), k_weight=x(32, dtype=torch.half))
    with pytest.raises(ValueError, match="GPU tensors only"):
        F.seq_rotary(q, k, positions, freqs)
    cache = F.SeqCache.empty(2, 2, 16, 32, device="cpu")
    table, lengths = torch.zeros((2, 1), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="freqs are missing"):
        F.seq_cache_append(cache, k, k, table, lengths, positions=positions)
    with pytest.raises(ValueError, match="freqs are missing"):
        F.seq_cache_append(cache, k, k, table, lengths, weight=x(32), sections=(16,))
    with pytest.raises(ValueError):
        F.seq_cache_append(cache, k, k, table, lengths, rows=lengths)
    for more in (dict(rows=table), dict(freqs=freqs), dict(weight=x(32))):
        with pytest.raises(ValueError, match="GPU tensors only"):
            F.seq_cache_append(cache, k, k, table, lengths, **more)
