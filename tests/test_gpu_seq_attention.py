"""Attention over sequences (seq_attention), forward and backward, against the 64-bit oracle through its bounds."""
import numpy as np
import pytest
import torch

from oracle import seq_oracle
from paper_2204_07143_amd import binding as na
from paper_2204_07143_amd import functional as F

from seq_util import FP32, HALF, TINY, TYPES, check, expect, f64, normal

pytestmark = pytest.mark.gpu


def _marks(g, B, L, docs, prefix, padding=3):
    documents = marks = None
    if docs:
        documents = np.sort(g.integers(0, docs, (B, L))).astype(np.int32)
        if padding:
            documents[:, -min(padding, L - 1) if L > 1 else L:] = -1
        documents = torch.from_numpy(documents).cuda()
    if prefix:
        marks = torch.from_numpy(g.random((B, L)) < 0.3).cuda()
    return documents, marks


def _run(q, k, v, dout, **mask):
    leaves = [x.detach().requires_grad_() for x in (q, k, v)]
    out = F.seq_attention(*leaves, **mask)
    return (out.detach(), *torch.autograd.grad(out, leaves, dout))


def _check(seed, B, heads, kv, Lq, Lk, D, dtype, docs=0, prefix=False, slopes=False, dout_std=1.0, q_std=1.0, **mask):
    g = np.random.default_rng(seed)
    q, k, v = normal(g, (B, heads, Lq, D), dtype, q_std), normal(g, (B, kv, Lk, D), dtype), normal(g, (B, kv, Lk, D), dtype)
    dout = normal(g, (B, heads, Lq, D), dtype, dout_std)
    mask["documents"], mask["prefix"] = _marks(g, B, Lk, docs, prefix)
    mask["slopes"] = torch.from_numpy(g.uniform(-0.1, 0.3, heads).astype(np.float32)).cuda() if slopes else None
    got = _run(q, k, v, dout, **mask)
    want, bound = expect(q, k, v, dout, dtype, **mask)
    for name, x in zip(("out", "dq", "dk", "dv"), got):
        check(name, x, want[name], bound[name])
    return got


TYPE = pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])


@TYPE
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("cap", [None, 4.0])
def test_types_and_head_dims(dtype, D, cap):
    _check(D, 2, 4, 2, 150, 150, D, dtype, causal=True, softcap=cap)


@TYPE
@pytest.mark.parametrize("Lq,Lk", [(1, 1), (1, 2), (3, 1), (15, 16), (16, 17), (63, 64), (64, 65), (65, 63), (127, 129), (129, 400), (1, 333), (200, 7)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(dtype, Lq, Lk, causal):
    _check(Lq * 1000 + Lk, 1, 2, 1, Lq, Lk, 32, dtype, causal=causal, softcap=None if Lq % 2 else 3.0)


MASKS = {
    "window": dict(window=20), "causal_window": dict(causal=True, window=70), "window_of_one": dict(causal=True, window=1),
    "slopes": dict(slopes=True), "causal_slopes": dict(causal=True, slopes=True, softcap=5.0),
    "documents": dict(docs=3), "causal_documents": dict(causal=True, docs=5, slopes=True), "many_documents": dict(causal=True, docs=90, window=9),
    "prefix": dict(causal=True, prefix=True), "prefix_window": dict(causal=True, window=11, prefix=True, softcap=2.0),
    "prefix_documents": dict(causal=True, prefix=True, docs=4, window=40, slopes=True),
}


@TYPE
@pytest.mark.parametrize("name", MASKS)
@pytest.mark.parametrize("Lq,Lk", [(260, 260), (37, 301)])
def test_masks(dtype, name, Lq, Lk):
    _check(len(name), 2, 6, 2, Lq, Lk, 64, dtype, **MASKS[name])


@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 1), (6, 3), (5, 5), (16, 2)])
def test_shared_heads(heads, kv):
    _check(heads, 3, heads, kv, 70, 70, 64, "bf16", causal=True)


@TYPE
def test_masks_that_leave_rows_empty(dtype):
    # more queries than keys in causal order: the first ones stand before every key
    got = _check(5, 1, 2, 2, 90, 20, 32, dtype, causal=True)
    assert (got[0][:, :, :69] == 0).all() and (got[1][:, :, :69] == 0).all()
    # nothing but padding
    q = torch.ones((1, 2, 66, 32), dtype=TYPES[dtype], device="cuda")
    got = _run(q, q, q, q, documents=torch.full((1, 66), -7, dtype=torch.int32, device="cuda"))
    assert all((x == 0).all() for x in got)


@TYPE
@pytest.mark.parametrize("prefix", [False, True])
def test_padding_may_hold_anything(dtype, prefix):
    g = np.random.default_rng(6)
    shape = (2, 4, 150, 64)
    q, k, v, dout = (normal(g, shape, dtype) for _ in range(4))
    documents, marks = _marks(g, 2, 150, 3, prefix, padding=0)
    documents[:, ::7] = -1
    documents[1, 64:128] = -2
    mask = dict(documents=documents, prefix=marks, causal=True, softcap=6.0)
    clean = _run(q, k, v, dout, **mask)
    dead = (documents < 0)[:, None, :, None]
    for value in (float("nan"), float("inf")):
        fouled = _run(*(x.masked_fill(dead, value) for x in (q, k, v, dout)), **mask)
        for a, b in zip(clean, fouled):
            assert torch.equal(a, b) and torch.isfinite(a).all()
    want, bound = expect(q, k, v, dout, dtype, **mask)
    for name, x in zip(("out", "dq", "dk", "dv"), clean):
        check(name, x, want[name], bound[name])


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.5])
@pytest.mark.parametrize("cap", [None, 10.0])
def test_scales(scale, cap):
    for dtype in ("bf16", "f32"):
        _check(7, 1, 2, 2, 100, 130, 32, dtype, scale=scale, softcap=cap, causal=True, q_std=2.0)


def test_scores_far_apart():
    """A running maximum that rises all along, and one that falls."""
    for sign in (1, -1):
        g = np.random.default_rng(8)
        q, k, v, dout = (normal(g, (1, 1, 300, 32), "f32") for _ in range(4))
        slopes = torch.tensor([sign * 0.7], device="cuda")
        got = _run(q, k, v, dout, slopes=slopes)
        want, bound = expect(q, k, v, dout, "f32", slopes=slopes)
        for name, x in zip(("out", "dq", "dk", "dv"), got):
            check(name, x, want[name], 16 * bound[name])   # scores reach 0.7 * 300, eight times "a few tens": so does what their fp32 rounding makes of a weight


@pytest.mark.parametrize("std", [1e-5, 1e-3, 300.0])
def test_gradients_of_any_size_in_fp16(std):
    g = np.random.default_rng(9)
    q, k, v = (normal(g, (1, 2, 200, 64), "f16") for _ in range(3))
    dout = normal(g, (1, 2, 200, 64), "f16", std)
    got = _run(q, k, v, dout, causal=True)
    want, bound = expect(q, k, v, dout, "f16", causal=True)
    for name, x in zip(("out", "dq", "dk", "dv"), got):
        check(name, x, want[name], bound[name])


@TYPE
def test_strided_tensors(dtype):
    g = np.random.default_rng(10)
    fused = normal(g, (2, 77, 8, 64), dtype)                # a projection's output: 4 query heads, 2 of keys, 2 of values
    q, k, v = (x.transpose(1, 2) for x in fused.split((4, 2, 2), 2))
    dout = normal(g, (2, 77, 4, 64), dtype).transpose(1, 2)
    got = _run(q, k, v, dout, causal=True)
    dense = _run(*(x.contiguous() for x in (q, k, v, dout)), causal=True)
    assert all(torch.equal(a, b) for a, b in zip(got, dense))
    # rows that are not whole 16 bytes apart, a view that begins off them, an order with D outside, broadcast keys: copied or read as they lie
    odd = torch.empty((2, 4, 77, 65), dtype=TYPES[dtype], device="cuda")[..., 1:].copy_(q)
    off = torch.empty(q.numel() + 1, dtype=TYPES[dtype], device="cuda")[1:].view(q.shape).copy_(q)
    inside_out = q.transpose(2, 3).contiguous().transpose(2, 3)
    for x in (odd, off, inside_out):
        assert torch.equal(F.seq_attention(x, k, v, causal=True), dense[0])
    one = k[:, :1].contiguous()
    assert torch.equal(F.seq_attention(q, one.expand(2, 2, 77, 64), v, causal=True), F.seq_attention(q, one.repeat(1, 2, 1, 1), v, causal=True))
    assert torch.equal(F.seq_attention(q, one, one, causal=True), F.seq_attention(q, one.repeat(1, 4, 1, 1), one.repeat(1, 4, 1, 1), causal=True))


def test_broadcast_inputs_have_summed_gradients():
    g = np.random.default_rng(11)
    q, dout = normal(g, (3, 2, 40, 32), "f32"), normal(g, (3, 2, 40, 32), "f32")
    k = normal(g, (1, 1, 40, 32), "f32").requires_grad_()
    grad, = torch.autograd.grad(F.seq_attention(q, k.expand(3, 2, 40, 32), k.expand(3, 2, 40, 32)), k, dout)
    wide = k.detach().expand(3, 2, 40, 32).contiguous()
    want, bound = expect(q, wide, wide, dout, "f32")
    total, most = ((x["dk"] + x["dv"]).sum((0, 1), keepdims=True) for x in (want, bound))
    check("dk + dv", grad, total, 2 * most)   # and six fp32 sums on top


@TYPE
def test_same_bits_again_and_on_another_stream(dtype):
    g = np.random.default_rng(12)
    q, k, v, dout = (normal(g, (2, 4, 300, 64), dtype) for _ in range(4))
    documents, prefix = _marks(g, 2, 300, 3, True)
    mask = dict(causal=True, documents=documents, prefix=prefix)
    first = _run(q, k, v, dout, **mask)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        second = _run(q, k, v, dout, **mask)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))


@TYPE
def test_lse_of_the_forward(dtype):
    g = np.random.default_rng(13)
    q, k, v = (normal(g, (2, 2, 90, 64), dtype) for _ in range(3))
    out, lse = torch.empty_like(q), torch.full((2, 2, 90), float("nan"), device="cuda")
    na.seq_attention_fwd(q, k, v, None, None, None, out, lse, causal=True, scale=0.125)
    want, bound = expect(q, k, v, None, dtype, causal=True)
    check("lse", lse, want["lse"], bound["lse"])


def test_gradient_against_differences():
    g = np.random.default_rng(14)
    q, k, v, dout = (normal(g, (1, 2, 80, 32), "f32") for _ in range(4))
    mask = dict(causal=True, softcap=3.0, prefix=torch.from_numpy(g.random((1, 80)) < 0.2).cuda())
    grads = _run(q, k, v, dout, **mask)[1:]
    for at, grad in enumerate(grads):
        step = normal(g, q.shape, "f32")
        sides = [(F.seq_attention(*(x + s * 1e-2 * step if i == at else x for i, x in enumerate((q, k, v))), **mask).double() * dout.double()).sum() for s in (1, -1)]
        change = float((sides[0] - sides[1]) / 2e-2)
        # the third derivative's share, (1e-2)^2 / 6 of terms of the gradient's size, and fp32: below 1e-3 of the gradient's length
        assert abs(change - float((grad.double() * step.double()).sum())) < 1e-3 * float(grad.double().norm() * step.double().norm()), at


def test_empty_tensors():
    for B, Lq, Lk in ((0, 5, 5), (2, 0, 5), (2, 5, 0)):
        q, k = (torch.zeros((B, 2, L, 32), device="cuda", requires_grad=True) for L in (Lq, Lk))
        out = F.seq_attention(q, k, k)
        assert out.shape == q.shape and (out == 0).all()
        out.sum().backward()
        assert q.grad.shape == q.shape and (q.grad == 0).all() and (k.grad == 0).all()


def test_no_second_derivative():
    q = torch.ones((1, 1, 4, 32), device="cuda", requires_grad=True)
    grad, = torch.autograd.grad(F.seq_attention(q, q, q).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivative"):
        grad.sum().backward()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 64), ("f32", 32)])
def test_replayed_graphs(dtype, D):
    g = np.random.default_rng(15)
    q, k, v = (normal(g, (2, 4, 140, D), dtype).requires_grad_() for _ in range(3))
    dout = normal(g, (2, 4, 140, D), dtype)
    documents, prefix = _marks(g, 2, 140, 2, True)

    def run():
        out = F.seq_attention(q, k, v, causal=True, documents=documents, prefix=prefix, softcap=5.0)
        return (out.detach(), *torch.autograd.grad(out, (q, k, v), dout))
    eager = [x.clone() for x in run()]
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):   # two graphs, each with workspaces of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = run()
        graphs.append((graph, outs))
    for _ in range(3):
        for _, outs in graphs:
            for x in outs:
                x.fill_(float("nan"))
        run()
        torch.cuda.synchronize()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, outs in graphs:
            assert all(torch.equal(a, b) for a, b in zip(outs, eager))


@TYPE
def test_native_and_interpreted_host_sides(dtype):
    """The same bits, gradients and refusals; kept for a second pass; saved-tensor hooks; what only the interpreted side takes."""
    g = np.random.default_rng(16)
    q, k, v = (normal(g, (2, 77, h, 64), dtype).transpose(1, 2).requires_grad_() for h in (4, 2, 2))
    dout = normal(g, (2, 4, 77, 64), dtype)
    documents, prefix = _marks(g, 2, 77, 2, True)
    slopes = torch.rand(4, device="cuda")
    settings = dict(causal=True, window=9, softcap=3.0, scale=0.2)
    native = F.seq_attention(q, k, v, slopes=slopes, documents=documents, prefix=prefix, **settings)
    plain = F._SeqAttention.apply(q, k, v, slopes, documents, prefix, settings)
    assert type(native.grad_fn).__name__ != type(plain.grad_fn).__name__ and torch.equal(native, plain) and native.stride() == plain.stride()
    for _ in range(2):
        for a, b in zip(torch.autograd.grad(native, (q, k, v), dout, retain_graph=True), torch.autograd.grad(plain, (q, k, v), dout, retain_graph=True)):
            assert torch.equal(a, b) and a.stride() == b.stride()
    with torch.no_grad():
        assert torch.equal(F.seq_attention(q, k, v, slopes=slopes, documents=documents, prefix=prefix, **settings), plain)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.cpu(), lambda t: t.cuda()):
        hooked = F.seq_attention(q, k, v, slopes=slopes, documents=documents, prefix=prefix, **settings)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(hooked, (q, k, v), dout), torch.autograd.grad(plain, (q, k, v), dout)))
    for bad in (dict(slopes=slopes.double()), dict(slopes=slopes[:3]), dict(documents=documents.long()), dict(documents=documents[:, 1:]), dict(prefix=prefix.int()),
                dict(prefix=prefix.cpu()), dict(documents=documents.t().contiguous().t())):
        with pytest.raises(ValueError):
            F.seq_attention(q, k, v, **bad)
    with pytest.raises(ValueError):
        F.seq_attention(q, k.float() if dtype != "f32" else k.half(), v)
    with pytest.raises(na.Na2dError) as e:
        F.seq_attention(q[..., :48], k[..., :48], v[..., :48])
    assert e.value.status == -5
    with pytest.raises(na.Na2dError) as e:
        F.seq_attention(q, k[:, :, 1:], v[:, :, 1:], documents=documents[:, 1:].contiguous())
    assert e.value.status == -6


@TYPE
@pytest.mark.parametrize("Lq,Lk", [(5, 1500), (700, 700), (64, 2000)])
@pytest.mark.parametrize("name", ["causal_slopes", "causal_documents", "prefix_documents", "causal_window", "documents"])
def test_work_split_along_the_keys_and_the_queries(dtype, Lq, Lk, name):
    """Few rows: a tile's work is split over workgroups and joined, parts without work among them."""
    D = {5: 128, 700: 64, 64: 32}[Lq]
    mask = dict(MASKS[name])
    settings = dict(causal=mask.get("causal", False), window=mask.get("window", 0), softcap=mask.get("softcap", 0.0), scale=1.0)
    q, k = (torch.empty((1, h, L, D), dtype=TYPES[dtype], device="cuda") for h, L in ((4, Lq), (2, Lk)))
    p = na.seq_problem(q, k, v=k, out=q, **settings)
    if name != "causal_window":
        assert na.seq_attention_workspace_bytes(p, "docs" in mask) > 4 * q.numel()   # (it is split)
    _check(Lq, 1, 4, 2, Lq, Lk, D, dtype, **mask)


def test_offsets_that_pass_32_bits():
    """Planes behind 2^32 bytes: the last tokens of the last heads see, through a window, the last keys alone."""
    L, D, last, window = 1 << 17, 128, 10, 64
    torch.manual_seed(17)
    q, dout = (torch.randn((3, 44, L, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = (torch.randn((3, 22, L, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert q.numel() * 2 > 1 << 32
    got = _run(q, k, v, dout, causal=True, window=window)
    reach = last + window - 1
    ends = q[2:, 42:, -last:], k[2:, 21:, -reach:], v[2:, 21:, -reach:], dout[2:, 42:, -last:]
    want, bound = expect(*ends, "bf16", causal=True, window=window)
    for name, x in zip(("out", "dq", "dk", "dv"), got):   # (of a key, all queries that see it stand behind it)
        check(name, x[2:, -want[name].shape[1]:, -last:], want[name][:, :, -last:], bound[name][:, :, -last:])


@TYPE
def test_broadcast_gradients_and_queries(dtype):
    """What is broadcast to a call is read where it lies, or copied: a gradient that is one number, queries that heads and sequences share."""
    g = np.random.default_rng(18)
    q, k, v = normal(g, (1, 1, 50, 64), dtype), *(normal(g, (2, 2, 50, 64), dtype) for _ in range(2))
    wide = q.expand(2, 4, 50, 64)
    one = torch.ones((), dtype=TYPES[dtype], device="cuda").expand(2, 4, 50, 64)
    row = normal(g, (1, 1, 1, 64), dtype).expand(2, 4, 50, 64)
    for dout in (one, row):
        for a, b in zip(_run(wide, k, v, dout, causal=True), _run(wide.contiguous(), k, v, dout.contiguous(), causal=True)):
            assert torch.equal(a, b)


@TYPE
def test_two_calls_at_once(dtype):
    g = np.random.default_rng(19)
    sets = [[normal(g, (1, 4, 900, 64), dtype) for _ in range(4)] for _ in range(2)]
    masks = [dict(zip(("documents", "prefix"), _marks(g, 1, 900, 3, True))) for _ in range(2)]
    want = [_run(*x, causal=True, **m) for x, m in zip(sets, masks)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(3):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(_run(*sets[i], causal=True, **masks[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for outs in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(outs, want[i]))


@TYPE
@pytest.mark.parametrize("cap", [0.5, 50.0, 55.45, 55.46, 300.0])   # weights from e^-cap to e^cap
@pytest.mark.parametrize("std", [0.01, 30.0])
def test_caps_that_are_reached(dtype, cap, std):
    _check(20, 1, 2, 1, 150, 150, 64, dtype, q_std=std, causal=True, softcap=cap, docs=2)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("name", ["plain", "causal_cap", "window_prefix_documents_slopes"])
def test_many_heads(dtype, D, name):
    """Enough rows for two blocks of them to a wave, where the order of the work allows it."""
    mask = {"plain": dict(), "causal_cap": dict(causal=True, softcap=20.0), "window_prefix_documents_slopes": dict(window=90, prefix=True, docs=3, slopes=True)}[name]
    _check(21, 2, 128, 128, 190, 190, D, dtype, **mask)


@TYPE
@pytest.mark.parametrize("Lq,Lk", [(3, 10), (65, 130), (37, 301), (100, 164), (64, 100), (1, 65)])
def test_padding_behind_fewer_queries_than_keys_may_hold_anything(dtype, Lq, Lk):
    """The last queries' tile begins inside the last keys' tile: what is staged behind the last query, which is padding, enters no product."""
    g = np.random.default_rng(22)
    q, dout = (normal(g, (2, 4, Lq, 64), dtype) for _ in range(2))
    k, v = (normal(g, (2, 2, Lk, 64), dtype) for _ in range(2))
    documents = torch.zeros((2, Lk), dtype=torch.int32, device="cuda")
    documents[:, -1] = -1
    documents[1, :Lk // 3] = -1
    dead = (documents < 0)[:, None, :, None]
    mine = dead[:, :, Lk - Lq:]
    mask = dict(documents=documents, causal=True)
    clean = _run(q, k, v, dout, **mask)
    for value in (float("nan"), float("inf")):
        fouled = _run(q.masked_fill(mine, value), k.masked_fill(dead, value), v.masked_fill(dead, value), dout.masked_fill(mine, value), **mask)
        for a, b in zip(clean, fouled):
            assert torch.isfinite(b).all() and torch.equal(a, b)
    want, bound = expect(q, k, v, dout, dtype, **mask)
    for name, x in zip(("out", "dq", "dk", "dv"), clean):
        check(name, x, want[name], bound[name])


def test_flat_rows_over_a_million_keys_in_fp16():
    """Weights of 2^-20 each, and dS with them: both keep fp16's digits.

    A rounding is taken as independent of the others, of mean zero and within half a step, so a sum of n of them stays (Hoeffding) within 6 times the root of the sum of their
    squares but in 2 of 10^8 cases.  Of dS: u |dS|, or half of 2^-24 on the scale it is held on, 2^15 of |dout| |v| for the largest there are, each taken to its power of two.
    """
    Lq, Lk, D, u = 2, 1 << 20, 32, HALF["f16"]
    torch.manual_seed(23)
    q, dout = (torch.randn((1, 1, Lq, D), device="cuda").mul_(s).half() for s in (1.0, 1000.0))   # (dk is of 2^-9 or so then, and none of fp16's smallest)
    k, v = (torch.randn((1, 1, Lk, D), device="cuda").half() for _ in range(2))
    got = _run(q, k, v, dout)
    size = float(v.double().abs().sum(-1).max())
    want, bound = expect(q, k, v, dout, "f16")
    check("out", got[0], want["out"], bound["out"])
    step = 2.0 ** -40 * 2 * size * 4   # of |dout|'s largest element in a row; 4: the other row's may be larger, and its power of two
    bounds = seq_oracle.attention(*(f64(x) for x in (q, k, v, dout)), u=u, e=FP32, tiny=step)[1]
    check("dk", got[2], want["dk"], bounds["dk"] + 2.0 ** -25)
    # P: half of 2^-24 on a scale of 2^10
    bounds = seq_oracle.attention(*(f64(x) for x in (q, k, v, dout)), u=u, e=FP32, tiny=2.0 ** -35)[1]
    check("dv", got[3], want["dv"], bounds["dv"] + 2.0 ** -25)
    q, k, v, dout = (x[0, 0].double() for x in (q, k, v, dout))
    p = torch.softmax(q @ k.T * D ** -0.5, 1)
    out = p @ v
    ds = p * (dout @ v.T - (dout * out).sum(1, keepdim=True)) * D ** -0.5
    off = u * ds.abs() + step * D ** -0.5 * dout.abs().amax(1, keepdim=True)
    # the sum: a rounding to fp32 for every four keys at most, each within 2^-24 of the largest partial sum
    partial = torch.stack([(row[:, None] * k).cumsum(0).abs().amax(0) for row in ds])
    of_delta = (u + FP32) * (dout * out).abs().sum(1, keepdim=True) * (p @ k).abs() * D ** -0.5
    tol = 6 * torch.sqrt(off.square() @ k.square()) + 6 * (Lk / 4) ** 0.5 * 2.0 ** -24 * partial + of_delta + (u + FP32) * (ds @ k).abs() + 2.0 ** -25
    check("dq", got[1][0, 0], (ds @ k).cpu().numpy(), tol.cpu().numpy())


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("cap", [None, 50.0])
def test_products_of_dout_and_values_beyond_fp16(D, cap):
    """|dP| reaches D * 4000, dS half of that: held on a scale that takes in the values' size, as gradients that fp16 holds."""
    g = np.random.default_rng(24)
    q, k = normal(g, (1, 2, 40, D), "f16", 0.3), normal(g, (1, 1, 40, D), "f16", 0.05)
    signs = torch.from_numpy(g.choice([-1.0, 1.0], (1, 1, 40, 1)).astype(np.float32)).cuda()
    v = (4000 * signs.expand(1, 1, 40, D)).half().contiguous()
    dout = (1 + normal(g, (1, 2, 40, D), "f32", 0.01)).half()
    mask = dict(causal=True, softcap=cap)
    got = _run(q, k, v, dout, **mask)
    want, bound = expect(q, k, v, dout, "f16", **mask)
    for name, x in zip(("out", "dq", "dk", "dv"), got):
        check(name, x, want[name], bound[name])


def _lse_of_one_key(dtype, cap, std):
    """A query that sees one key has that score as its lse: (lse, the score in 64 bits, the size of the products that it is the sum of)."""
    g = np.random.default_rng(25)
    q, k = normal(g, (1, 1, 4096, 32), dtype, std), normal(g, (1, 1, 1, 32), dtype)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    na.seq_attention_fwd(q, k, k, None, None, None, out, lse, scale=32 ** -0.5, softcap=cap)
    scale = float(np.float32(32 ** -0.5))
    size = (np.abs(f64(q)) @ np.abs(f64(k)).swapaxes(2, 3))[..., 0] * scale
    return f64(lse), cap * np.tanh((f64(q) @ f64(k).swapaxes(2, 3))[..., 0] * scale / cap), size


# <q, k> is a sum of 32 products in fp32, each rounding within 2^-24 of a partial sum: 2^-19 of their size.  The score from it, in base 2, and lse: factors of fp32 and their products,
# and a tanh of a few 2^-24 or the sigmoid's form; 2^-19 of the score leaves 32 x 2^-24 for these.
@pytest.mark.parametrize("dtype,cap", [("f16", 50.0), ("f16", 1024.0), ("bf16", 50.0), ("bf16", 1024.0), ("bf16", 4096.0)])
@pytest.mark.parametrize("std", [0.1, 30.0, 3000.0])
def test_capped_scores_are_off_by_little_of_the_cap(dtype, cap, std):
    """1 - 2 / (1 + e^2z): 2^-24 of the fraction for the sum, 2^-23 each for the exponential and the reciprocal, and it counts twice at most: 6 x 2^-24, and one each for the exponent's
    and the score's own rounding: 8 x 2^-24 = 2^-21 of the cap."""
    lse, want, size = _lse_of_one_key(dtype, cap, std)
    assert (np.abs(lse - want) <= 2.0 ** -21 * cap + 2.0 ** -19 * (size + np.abs(want))).all()


@pytest.mark.parametrize("dtype,cap", [("f16", 1025.0), ("f16", 4096.0), ("f32", 50.0), ("f32", 4096.0), ("f32", 1e6)])
@pytest.mark.parametrize("std", [0.1, 1.0, 300.0])
def test_scores_far_below_a_large_cap_keep_their_digits(dtype, cap, std):
    lse, want, size = _lse_of_one_key(dtype, cap, std)
    assert (np.abs(lse - want) <= 2.0 ** -19 * (size + np.abs(want))).all()


@TYPE
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("cap", [1000.0, 1500.0, 4096.0])
def test_large_caps(dtype, D, cap):
    """A weight is off by what its score is off by: 2^-21 of the cap where that is the sigmoid's (up to 1024 in fp16)."""
    e = FP32 + (cap * 2.0 ** -21 if dtype == "bf16" or (dtype == "f16" and cap <= 1024) else 0.0)
    g = np.random.default_rng(26)
    for mask in (dict(causal=True, docs=2), dict(window=50, prefix=True)):
        q, k, v, dout = normal(g, (2, 4, 150, D), dtype, 10.0), normal(g, (2, 2, 190, D), dtype), normal(g, (2, 2, 190, D), dtype), normal(g, (2, 4, 150, D), dtype)
        mask["documents"], mask["prefix"] = _marks(g, 2, 190, mask.pop("docs", 0), mask.pop("prefix", False))
        mask["softcap"] = cap
        if not mask.get("causal"):
            mask["slopes"] = torch.from_numpy(g.uniform(-0.1, 0.3, 4).astype(np.float32)).cuda()
        got = _run(q, k, v, dout, **mask)
        host = {n: (f64(x) if n == "slopes" else x.cpu().numpy()) if isinstance(x, torch.Tensor) else x for n, x in mask.items()}
        want, bound = seq_oracle.attention(*(f64(x) for x in (q, k, v, dout)), u=HALF[dtype], e=e, tiny=TINY[dtype], **host)
        for name, x in zip(("out", "dq", "dk", "dv"), got):
            check(name, x, want[name], bound[name])


@pytest.mark.parametrize("window", [None, 4096])
def test_large_values_that_a_query_does_not_see_in_fp16(window):
    """Values of 30000 in another document, or before the window, leave the scale of dS as it is."""
    Lq, Lk, D, seen = 4, 5120, 64, 4096
    g = np.random.default_rng(28)
    q, dout = normal(g, (1, 2, Lq, D), "f16", 0.1), normal(g, (1, 2, Lq, D), "f16", 100.0)
    k, v = normal(g, (1, 1, Lk, D), "f16"), normal(g, (1, 1, Lk, D), "f16")
    v[:, :, :Lk - seen - Lq - 60] = 30000.0   # (960 keys: whole tiles)
    mask = dict(causal=True, window=window)
    if window is None:
        mask["documents"] = (torch.arange(Lk, device="cuda") >= Lk - seen - Lq - 60).int()[None]
    got = _run(q, k, v, dout, **mask)
    want, bound = expect(q, k, v, dout, "f16", **mask)
    for name, x in zip(("out", "dq"), got):
        check(name, x, want[name], bound[name])
    near = v[:, :, -seen - Lq - 60:]
    step = 2.0 ** -40 * 2 * float(near.double().abs().sum(-1).max()) * 8   # half a step of dS on its scale, see above; 8: the largest |dout| of another row or head, and its power of two
    host = {n: x.cpu().numpy() if isinstance(x, torch.Tensor) else x for n, x in mask.items()}
    bounds = seq_oracle.attention(*(f64(x) for x in (q, k, v, dout)), u=HALF["f16"], e=FP32, tiny=step, **host)[1]
    check("dk", got[2], want["dk"], bounds["dk"] + 2.0 ** -25)
    bounds = seq_oracle.attention(*(f64(x) for x in (q, k, v, dout)), u=HALF["f16"], e=FP32, tiny=2.0 ** -35, **host)[1]
    check("dv", got[3], want["dv"], bounds["dv"] + 2.0 ** -25)
