"""Rotation by position with the norm before it, forward and backward, against the 64-bit oracle; before attention on sequences and on maps."""
import numpy as np
import pytest
import torch

from oracle import seq_oracle
from paper_2204_07143_amd import functional as F

from seq_util import HALF, TINY, TYPES, check, f64, normal

pytestmark = pytest.mark.gpu


def _freqs(pairs, base=10000.0):
    return torch.tensor([base ** (-i / pairs) for i in range(pairs)], dtype=torch.float32, device="cuda")


def _compare(dtype, q, k, positions, freqs, sections, qw=None, kw=None, eps=1e-6, interleaved=False, dz=None):
    """Both passes; dz: the outputs' gradients, or None for normal ones."""
    leaves = [t.requires_grad_() for t in (q, k, qw, kw) if t is not None]
    z = F.seq_rotary(q, k, positions, freqs, sections=sections, q_weight=qw, k_weight=kw, eps=eps, interleaved=interleaved)
    outs = [t for t in z if t is not None]
    dz = [normal(np.random.default_rng(1), tuple(t.shape), dtype) for t in outs] if dz is None else dz
    grads = iter(torch.autograd.grad(outs, leaves, dz))
    dx = [next(grads) for _ in outs]
    flat = lambda t: f64(t).reshape(t.shape[0], t.shape[1], -1, t.shape[-1])
    at = positions.flatten(-2) if q.dim() == 5 else positions
    for name, x, w, z, d, got in zip("qk", (q, k), (qw, kw), outs, dz, dx):
        res, bound = seq_oracle.rotary(flat(x), at.cpu().numpy(), f64(freqs), sections or (freqs.numel(),), f64(w), eps, interleaved, flat(d), u=HALF[dtype], tiny=TINY[dtype])
        check(name, z.reshape(res["z"].shape), res["z"], bound["z"])
        check("d" + name, got.reshape(res["dx"].shape), res["dx"], bound["dx"])
        if w is not None:
            assert w.dtype == torch.float32 or w.dtype == TYPES[dtype]
            rounding = (HALF[dtype] if w.dtype != torch.float32 else 0.0) * np.abs(res["dw"])
            check(f"d{name}_weight", next(grads), res["dw"], bound["dw"] + rounding)


def _weights(g, D, dtype):
    return [torch.from_numpy(g.uniform(0.5, 1.5, D).astype(np.float32)).to(TYPES[dtype]).cuda() for _ in range(2)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,sections", [(16, (8,)), (32, (16,)), (32, (3, 5)), (64, (8, 12, 12)), (64, (16,)), (128, (64,)), (128, (16, 24, 8)), (128, (1, 1, 5, 1)), (128, (10, 20, 30, 4))])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("normed", [False, True])
def test_both_passes(dtype, D, sections, interleaved, normed):
    g = np.random.default_rng(D + len(sections))
    B, heads, kv, L = 2, 5, 2, 37
    q, k = (normal(g, (B, L, h, D), dtype).transpose(1, 2) for h in (heads, kv))
    positions = torch.from_numpy(g.integers(-1000, 100000, (B, len(sections), L)).astype(np.int32)).cuda()
    weights = _weights(g, D, dtype if interleaved else "f32") if normed else (None, None)
    _compare(dtype, q, k, positions, _freqs(sum(sections)), sections, *weights, interleaved=interleaved)


@pytest.mark.parametrize("B,heads,kv,L,D", [(1, 1, 1, 1, 64), (3, 1, 7, 1, 128), (1, 33, 2, 2, 32), (1, 2, 1, 1031, 64), (40, 3, 3, 5, 16), (1, 130, 1, 3, 128), (2, 4, 4, 700, 128)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sizes(B, heads, kv, L, D, dtype):
    g = np.random.default_rng(B + heads + L)
    q, k = (normal(g, (B, h, L, D), dtype) for h in (heads, kv))
    _compare(dtype, q, k, torch.arange(L, dtype=torch.int32, device="cuda")[None], _freqs(D // 2), None, *_weights(g, D, dtype))


def test_many_workgroups_leave_sums_of_the_weights_gradient():
    g = np.random.default_rng(2)
    q, k = normal(g, (2, 3, 9001, 32), "f32"), normal(g, (2, 1, 9001, 32), "f32")
    _compare("f32", q, k, torch.arange(9001, dtype=torch.int32, device="cuda")[None], _freqs(16), None, *_weights(g, 32, "f32"))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_far_positions(dtype):
    g = np.random.default_rng(3)
    positions = torch.tensor([[2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, 123456789, -987654321, 0, 1, -1]], dtype=torch.int32, device="cuda")
    q = normal(g, (1, 2, 8, 64), dtype)
    _compare(dtype, q, q.clone(), positions, _freqs(32), None)


def test_one_side_alone_and_one_weight():
    g = np.random.default_rng(4)
    q, positions = normal(g, (2, 4, 9, 64), "bf16"), torch.arange(9, dtype=torch.int32, device="cuda")[None]
    z, none = F.seq_rotary(q, None, positions, _freqs(32))
    assert none is None
    _compare("bf16", q, None, positions, _freqs(32), None, _weights(g, 64, "bf16")[0])
    k = normal(g, (2, 2, 9, 64), "bf16")
    _compare("bf16", q, k, positions, _freqs(32), None, None, _weights(g, 64, "f32")[0])
    _compare("bf16", q, k, positions, _freqs(32), None, _weights(g, 64, "f32")[0], None)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("D", [16, 32])
def test_maps(dtype, D):
    g = np.random.default_rng(5)
    q, k = (normal(g, (3, 2, 7, 11, D), dtype) for _ in range(2))
    grid = torch.stack(torch.meshgrid(torch.arange(7), torch.arange(11), indexing="ij")).to(torch.int32).cuda()
    _compare(dtype, q, k, grid, _freqs(8, 100.0), (4, 4), *_weights(g, D, dtype))
    _compare(dtype, q.transpose(2, 3), k.transpose(2, 3), grid.transpose(1, 2).contiguous(), _freqs(8, 100.0), (4, 4))


@pytest.mark.parametrize("std", [1e-7, 1e4])
def test_sizes_of_values(std):
    """The norm of small values is eps's, of large ones their own."""
    g = np.random.default_rng(6)
    q = normal(g, (1, 2, 20, 64), "f32", std)
    _compare("f32", q, q.clone(), torch.arange(20, dtype=torch.int32, device="cuda")[None], _freqs(32), None, *_weights(g, 64, "f32"), eps=1e-12)


def test_zero_rows_and_values_that_are_no_numbers_stay_where_they_are():
    g = np.random.default_rng(7)
    q, w = normal(g, (1, 3, 6, 64), "f32"), _weights(g, 64, "f32")[0]
    q[0, 1, 2] = 0
    want = F.seq_rotary(q, None, torch.arange(6, dtype=torch.int32, device="cuda")[None], _freqs(32), q_weight=w)[0]
    assert (want[0, 1, 2] == 0).all()
    q[0, 0, 4, 5] = float("nan")
    q[0, 2, 3, 7] = float("inf")
    got = F.seq_rotary(q, None, torch.arange(6, dtype=torch.int32, device="cuda")[None], _freqs(32), q_weight=w)[0]
    same = torch.ones((3, 6), dtype=torch.bool)
    same[0, 4] = same[2, 3] = False
    assert torch.equal(got[0][same.cuda()], want[0][same.cuda()]) and torch.isnan(got[0, 0, 4]).all()


def test_strides_and_broadcast_gradients():
    g = np.random.default_rng(8)
    packed = normal(g, (2, 13, 8 * 64), "f16").view(2, 13, 8, 64).transpose(1, 2)   # queries and keys of one projection
    q, k = packed[:, :5], packed[:, 5:]
    positions = torch.arange(13, dtype=torch.int32, device="cuda")[None]
    w = _weights(g, 64, "f16")
    dz = [torch.ones((), dtype=torch.float16, device="cuda").expand(2, 5, 13, 64), normal(g, (2, 1, 13, 64), "f16").expand(2, 3, 13, 64)]
    _compare("f16", q.detach(), k.detach(), positions, _freqs(32), None, *w, dz=dz)
    odd = normal(g, (2, 5, 13, 65), "f16")[..., 1:]   # rows that are not of whole 16 bytes are copied
    _compare("f16", odd, normal(g, (2, 5, 13, 130), "f16")[..., ::2][..., 1:], positions, _freqs(32), None, *w)


def test_tensors_behind_32_bits():
    g = np.random.default_rng(11)
    near = [normal(g, (2, 3, 7, 64), "f16") for _ in range(2)]
    far = [torch.empty((1 << 31) + 3 * 7 * 64, dtype=torch.float16, device="cuda").as_strided((2, 3, 7, 64), (1 << 31, 7 * 64, 64, 1)) for _ in near]
    for a, b in zip(far, near):
        a.copy_(b)
    positions, w = torch.arange(7, dtype=torch.int32, device="cuda")[None], _weights(g, 64, "f16")[0].requires_grad_()
    results = []
    for q, dz in (near, far):
        q = q.detach().requires_grad_()
        z = F.seq_rotary(q, None, positions, _freqs(32), q_weight=w)[0]
        results.append((z, *torch.autograd.grad(z, (q, w), dz)))
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_nothing_to_do():
    w = torch.ones(64, device="cuda", requires_grad=True)
    q = torch.zeros((0, 4, 5, 64), device="cuda", requires_grad=True)
    z, _ = F.seq_rotary(q, None, torch.zeros((1, 5), dtype=torch.int32, device="cuda"), _freqs(32), q_weight=w)
    z.sum().backward()
    assert z.shape == q.shape and q.grad.shape == q.shape and (w.grad == 0).all()


def test_second_derivatives_are_refused():
    q = torch.randn((1, 2, 5, 64), device="cuda", requires_grad=True)
    w = torch.ones(64, device="cuda", requires_grad=True)
    z, _ = F.seq_rotary(q, None, torch.zeros((1, 5), dtype=torch.int32, device="cuda"), _freqs(32), q_weight=w)
    dq, dw = torch.autograd.grad(z.square().sum(), (q, w), create_graph=True)
    with pytest.raises(RuntimeError, match="seq_rotary has no second derivative"):
        torch.autograd.grad(dw.sum(), q)


def test_the_interpreted_path_gives_the_same_bits():
    """With a torch-function mode on, the native code hands the call back."""
    from torch.overrides import TorchFunctionMode

    class Mode(TorchFunctionMode):
        def __torch_function__(self, f, types, args=(), kwargs=None):
            return f(*args, **(kwargs or {}))
    g = np.random.default_rng(9)
    q, k = (normal(g, (2, h, 9, 64), "bf16").requires_grad_() for h in (4, 2))
    w = [x.requires_grad_() for x in _weights(g, 64, "bf16")]
    positions, dz = torch.arange(9, dtype=torch.int32, device="cuda")[None], [normal(g, (2, h, 9, 64), "bf16") for h in (4, 2)]

    def both():
        z = F.seq_rotary(q, k, positions, _freqs(32), q_weight=w[0], k_weight=w[1])
        return (*z, *torch.autograd.grad(z, (q, k, *w), dz))
    native = both()
    with Mode():
        interpreted = both()
    for a, b in zip(native, interpreted):
        assert torch.equal(a, b)


def test_same_bits_on_another_stream_and_replayed():
    g = np.random.default_rng(10)
    q, k = (normal(g, (2, h, 300, 64), "bf16") for h in (6, 2))
    w, positions, freqs = _weights(g, 64, "bf16"), torch.arange(300, dtype=torch.int32, device="cuda")[None], _freqs(32)
    dz = [normal(g, (2, h, 300, 64), "bf16") for h in (6, 2)]

    def both(leaves):
        z = F.seq_rotary(leaves[0], leaves[1], positions, freqs, q_weight=leaves[2], k_weight=leaves[3])
        return (*(t.detach() for t in z), *torch.autograd.grad(z, leaves, dz))
    fresh = lambda: [t.detach().clone().requires_grad_() for t in (q, k, *w)]
    eager = both(fresh())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        leaves = fresh()
        again = both(leaves)
    stream.synchronize()
    for a, b in zip(eager, again):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = both(leaves)
    for _ in range(3):
        for t in out:
            t.fill_(float("nan"))
        both(fresh())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


def test_attention_sees_distances_alone():
    """Positions all moved by the same: scores, and so outputs, stay.  fp32: a score of 64 products of rotated channels is off by 2^-19 of sum |q| |k| twice (the bound of each
    rotation) and by the attention's own share; weights by that, at most 2 * 8 * 2^-18 of themselves here, and out of their sum with |v|, below 4 each."""
    g = np.random.default_rng(11)
    q, k, v = (normal(g, (2, h, 50, 64), "f32") for h in (4, 2, 2))
    w = _weights(g, 64, "f32")
    positions = torch.arange(50, dtype=torch.int32, device="cuda")[None]
    out = [F.seq_attention(*F.seq_rotary(q, k, positions + by, _freqs(32), q_weight=w[0], k_weight=w[1]), v, causal=True) for by in (0, 777777)]
    size = (f64(q) ** 2).sum(-1).max() ** 0.5 * (f64(k) ** 2).sum(-1).max() ** 0.5 * 2.25 / 8 * 2   # of scaled scores, and twice for pairs' |y_a| + |y_b|
    assert (out[0] - out[1]).abs().max() <= 4 * size * 2.0 ** -17
    # and on maps
    q, k, v = (normal(g, (2, 2, 9, 9, 32), "f32") for _ in range(3))
    grid = torch.stack(torch.meshgrid(torch.arange(9), torch.arange(9), indexing="ij")).to(torch.int32).cuda()
    out = [F.na2d(*F.seq_rotary(q, k, grid + by, _freqs(16, 100.0), sections=(8, 8), interleaved=True), v, kernel_size=5) for by in (0, 5000)]
    size = (f64(q) ** 2).sum(-1).max() ** 0.5 * (f64(k) ** 2).sum(-1).max() ** 0.5 / 32 ** 0.5 * 2
    assert (out[0] - out[1]).abs().max() <= 5 * size * 2.0 ** -17
