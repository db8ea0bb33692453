"""Refusals of the attention of drafted trees and of their verification, before any GPU call (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2204_07143_amd import binding as na
from paper_2204_07143_amd import functional as F

from test_seq_host import C


def S(*s):
    return ctypes.byref(na.SeqStrides(*s))


@pytest.mark.parametrize("problem,ok", [(C(), True), (C(n=64), True), (C(n=65), False), (C(dtype=0), False), (C(n=0), False), (C(D=48), False), (C(heads=5), False), (C(cap=5000.0), False)])
def test_tree_problems(problem, ok):
    assert (na.seq_cache_tree_attention_workspace_bytes(problem) > 0) == ok


def test_tree_arguments():
    lib, at = na.load(), lambda n: ctypes.c_void_p(4096 + 16 * n)
    p = C(n=4)
    need = na.seq_cache_tree_attention_workspace_bytes(p)
    names = ("q", "k", "v", "parents", "kp", "vp", "ks", "vs", "table", "lengths", "slopes", "out", "ws")
    own = S(2 * 4 * 64, 4 * 64, 64)

    def call(p=p, k_strides=own, v_strides=own, n=need, **x):
        return lib.seq_cache_tree_attention(ctypes.byref(p), k_strides, v_strides, *({m: at(i) for i, m in enumerate(names)} | x).values(), n, None)
    assert lib.seq_cache_tree_attention(None, own, own, *[at(1)] * 13, 1 << 30, None) == -1
    for name in ("q", "k", "v", "parents", "kp", "vp", "ks", "vs", "table", "lengths", "out"):
        assert call(**{name: None}) == -1
    assert call(k_strides=None) == -1 and call(k_strides=None, v_strides=None) == -1
    assert call(k_strides=S(512, 256, 60)) == -7 and call(v_strides=S(-512, 256, 64)) == -6 and call(C(n=65)) == -6 and call(C(n=4, dtype=0)) == -2
    assert call(k=ctypes.c_void_p(4100)) == -7 and call(parents=ctypes.c_void_p(4097)) == -7
    assert call(out=at(0)) == -10 and call(out=at(1)) == -10 and call(out=at(2)) == -10
    assert call(ws=None) == -8 and call(n=need - 1) == -8 and call(ws=ctypes.c_void_p(4104)) == -8


def V(B=2, n=5, size=1000, dtype=1, drafted=0, batch=5000, row=1000, draft_batch=4000, draft_row=1000):
    return na.SeqVerifyProblem(B, n, size, dtype, drafted, batch, row, draft_batch, draft_row)


@pytest.mark.parametrize("problem,code", [
    (V(), 0), (V(drafted=1), 0), (V(n=64), 0), (V(n=1, drafted=1), 0), (V(size=1 << 24), 0), (V(size=1, row=0, batch=0), 0), (V(row=7), 0),
    (V(dtype=3), -2), (V(B=0), -6), (V(n=0), -6), (V(n=65), -6), (V(size=0), -6), (V(size=(1 << 24) + 1), -6), (V(drafted=2), -6), (V(batch=-1), -6), (V(row=1 << 46), -6),
    (V(B=1 << 20, batch=1 << 45), -6), (V(B=1 << 24, n=64, size=1 << 24), -6),
])
def test_verify_problems(problem, code):
    assert na.seq_verify_validate(problem) == code
    assert (na.seq_verify_workspace_bytes(problem) > 0) == (code == 0)


@pytest.mark.parametrize("drafted", [0, 1])
def test_verify_arguments(drafted):
    lib, at, p = na.load(), lambda n: ctypes.c_void_p(4096 + 16 * n), V(drafted=drafted)
    need = na.seq_verify_workspace_bytes(p)
    names = ("logits", "draft", "tokens", "parents", "uniforms", "temperatures", "path", "counts", "next", "ws")
    usual = {"parents": None} if drafted else {"draft": None}

    def call(p=p, n=need, **x):
        return lib.seq_verify(ctypes.byref(p), *({m: at(i) for i, m in enumerate(names)} | usual | x).values(), n, None)
    assert lib.seq_verify(None, *[at(1)] * 10, 1 << 30, None) == -1
    for name in ("logits", "tokens", "uniforms", "path", "counts", "next"):
        assert call(**{name: None}) == -1
    assert call(**({"draft": None} if drafted else {"draft": at(1)})) == (-1 if drafted else -6)
    if drafted:
        assert call(parents=at(3)) == -6
    assert call(logits=ctypes.c_void_p(4097)) == -7 and call(tokens=ctypes.c_void_p(4098)) == -7 and call(temperatures=ctypes.c_void_p(4098)) == -7
    assert call(path=at(2)) == -10 and call(counts=at(6)) == -10 and call(next=at(0)) == -10
    assert call(ws=None) == -8 and call(n=need - 1) == -8 and call(ws=ctypes.c_void_p(4104)) == -8


def test_python_arguments():
    x = lambda *s, **k: torch.zeros(s, **k)
    q, kv = x(2, 4, 5, 32, dtype=torch.half), x(2, 2, 5, 32, dtype=torch.half)
    cache, table, lengths, parents = F.SeqCache.empty(2, 2, 16, 32, device="cpu"), *(torch.zeros(s, dtype=torch.int32) for s in ((2, 1), (2,), (2, 5)))
    for args in ((q[0], kv, kv), (q, kv, kv[:, :1]), (q, x(2, 3, 5, 32), x(2, 3, 5, 32))):
        with pytest.raises(ValueError):
            F.seq_cache_tree_attention(*args, parents, cache, table, lengths)
    for more in (dict(window=0), dict(softcap=-1.0), dict(slopes=x(4, requires_grad=True))):
        with pytest.raises(ValueError):
            F.seq_cache_tree_attention(q, kv, kv, parents, cache, table, lengths, **more)
    with pytest.raises(ValueError, match="GPU tensors only"):
        F.seq_cache_tree_attention(q, kv, kv, parents, cache, table, lengths)
    logits, tokens, u = x(2, 5, 100), torch.zeros((2, 5), dtype=torch.int32), x(2, 5)
    with pytest.raises(ValueError, match="no parents"):
        F.seq_verify(logits, tokens, u, parents=parents, draft=x(2, 4, 100))
    with pytest.raises(ValueError, match="GPU tensors only"):
        F.seq_verify(logits, tokens, u, parents=parents)
    with pytest.raises(ValueError):
        F.seq_verify(logits[0], tokens, u)
