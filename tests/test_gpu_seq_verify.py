"""Verification of drafted tokens against the 64-bit oracle: whole numbers, all equal."""
import numpy as np
import pytest
import torch

from oracle import seq_oracle
from paper_2204_07143_amd import functional as F

from seq_util import TYPES, f64

pytestmark = pytest.mark.gpu


def _logits(g, B, n, V, dtype):
    """A few tokens far above the others."""
    x = 2 * g.standard_normal((B, n, V))
    for _ in range(min(8, V)):
        np.put_along_axis(x, g.integers(0, V, (B, n, 1)), g.uniform(9, 15, (B, n, 1)), 2)
    return torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype]).cuda()


def _int(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


def _f32(x):
    return torch.from_numpy(np.asarray(x, np.float32)).cuda()


def _tree(g, B, n, logits, spread=3):
    """Parents, and tokens that are likely at their parents."""
    parents, tokens = np.full((B, n), -1), np.zeros((B, n), int)
    best = np.argsort(-f64(logits) + g.standard_normal(logits.shape), axis=2)[:, :, :8]
    for b in range(B):
        for i in range(1, n):
            parents[b, i] = g.integers(max(0, (i - 1) // spread), i)
            tokens[b, i] = best[b, parents[b, i], (parents[b, 1:i] == parents[b, i]).sum() % best.shape[2]]
    return parents, tokens


def _compare(logits, tokens, uniforms, parents=None, draft=None, temperatures=None):
    got = F.seq_verify(logits, _int(tokens), _f32(uniforms), parents=None if parents is None else _int(parents), draft=draft, temperatures=None if temperatures is None else _f32(temperatures))
    path, counts, following = (x.cpu().numpy() for x in got)
    uniforms, lengths = np.asarray(uniforms, np.float32).astype(np.float64), []
    for b in range(logits.shape[0]):
        want, token = seq_oracle.verify(f64(logits[b]), tokens[b], uniforms[b], None if parents is None else parents[b], None if draft is None else f64(draft[b]),
                                        1.0 if temperatures is None else float(np.float32(temperatures[b])))
        assert path[b].tolist() == want + [-1] * (len(path[b]) - len(want)) and counts[b] == len(want) and following[b] == token, (b, path[b].tolist(), want, following[b], token)
        lengths.append(len(want))
    return lengths


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,n,V", [(3, 1, 1), (4, 2, 2), (5, 9, 7), (2, 64, 8), (6, 12, 255), (3, 20, 2049), (2, 33, 32000), (1, 7, 50021), (2, 3, 200003), (40, 30, 1000)])
def test_trees(dtype, B, n, V):
    g = np.random.default_rng(V)
    logits = _logits(g, B, n, V, dtype)
    parents, tokens = _tree(g, B, n, logits)
    temperatures = g.uniform(0.5, 1.5, B)
    temperatures[B // 2::3] = 0
    lengths = _compare(logits, tokens, g.random((B, n)), parents, temperatures=temperatures)
    assert n < 9 or V < 200 or max(lengths) > 1
    _compare(logits, tokens, g.random((B, n)))   # a line, at a temperature of 1


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,n,V", [(3, 1, 1), (4, 2, 2), (5, 9, 7), (2, 64, 8), (6, 12, 255), (3, 20, 2049), (2, 33, 32000), (1, 7, 50021), (2, 3, 200003), (40, 5, 1000)])
def test_lines_with_the_drafts_distributions(dtype, B, n, V):
    g = np.random.default_rng(V + 1)
    logits = _logits(g, B, n, V, dtype)
    draft = (logits[:, :n - 1].float() + torch.from_numpy(g.standard_normal((B, n - 1, V)).astype(np.float32)).cuda()).to(TYPES[dtype])
    temperatures = g.uniform(0.5, 1.5, B)
    temperatures[B // 2::3] = 0
    tokens = np.zeros((B, n), int)
    for b in range(B):
        for i in range(n - 1):
            tokens[b, i + 1] = seq_oracle._drawn(seq_oracle._probabilities(f64(draft[b, i]), temperatures[b]), g.random())
    lengths = _compare(logits, tokens, g.random((B, n + 1)), draft=draft, temperatures=temperatures)
    assert n < 9 or min(lengths) < n
    tokens[::2, n // 2:] = V   # drafts that end early
    _compare(logits, tokens, g.random((B, n + 1)), draft=draft)


def test_draws_follow_the_probabilities():
    """Every token of a small vocabulary by its number: the borders of the running sums, a little inside of each."""
    g = np.random.default_rng(2)
    x = g.standard_normal(50).astype(np.float32)
    p = seq_oracle._probabilities(x.astype(np.float64), 1.0)
    sums = np.concatenate([[0], np.cumsum(p)])
    u = np.concatenate([sums[:-1] + 1e-6, sums[1:] - 1e-6]).astype(np.float32)
    logits = torch.from_numpy(x).cuda().expand(100, 1, 50)
    _, counts, following = F.seq_verify(logits, _int(np.zeros((100, 1))), _f32(u[:, None]))
    assert following.tolist() == list(range(50)) * 2 and (counts == 1).all()


@pytest.mark.parametrize("drafted", [False, True])
def test_numbers_out_of_range(drafted):
    g = np.random.default_rng(3)
    u = [0.0, -1.0, 1.0, 1.5, float("inf"), -float("inf"), float("nan"), 1 - 2.0 ** -24, 2.0 ** -30]
    B, n, V = len(u), 3, 5000
    logits = _logits(g, B, n, V, "f32")
    tokens = np.stack([np.zeros(B, int), f64(logits[:, 0]).argmax(1), f64(logits[:, 1]).argmax(1)], 1)
    draft = _logits(g, B, n - 1, V, "f32") if drafted else None
    _compare(logits, tokens, np.repeat(np.array(u)[:, None], n + drafted, 1), draft=draft)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drafted", [False, True])
def test_logits_that_are_no_numbers_or_infinite(dtype, drafted):
    g = np.random.default_rng(4)
    B, n, V, inf = 8, 3, 3001, float("inf")
    logits = _logits(g, B, n, V, dtype)
    logits[0, :, ::2] = -inf
    logits[1, 0, 5:] = float("nan")
    logits[2, 0] = -inf             # a row that gives nothing
    logits[3, 0] = -inf
    logits[3, 0, 777] = -3.0        # one token
    logits[4, 0, 9] = inf
    logits[4, 0, 2000] = inf        # two that share all
    logits[5, :, :2048] = -inf      # whole parts of nothing
    logits[6] = float("nan")
    draft = _logits(g, B, n - 1, V, dtype) if drafted else None
    if drafted:
        draft[7, 0] = -inf
        draft[0, 0, 1::2] = -inf    # nothing in common with the target
    tokens = g.integers(0, V, (B, n))
    tokens[3, 1], tokens[4, 1] = 777, 9
    for temperatures in (None, np.zeros(B), np.full(B, 0.1)):
        _compare(logits, tokens, g.random((B, n + drafted)), draft=draft, temperatures=temperatures)


@pytest.mark.parametrize("drafted", [False, True])
def test_temperatures(drafted):
    g = np.random.default_rng(5)
    temperatures = [0.0, -1.0, float("nan"), 1e-30, 1e-3, 1e30, float("inf"), 1e-44]
    B, n, V = len(temperatures), 4, 700
    logits = _logits(g, B, n, V, "f32")
    logits[0, :, 300] = logits[0, :, 301] = logits[0].max() + 1   # ties go to the lowest
    tokens = np.concatenate([np.zeros((B, 1), int), f64(logits).argmax(2)[:, :n - 1]], 1)
    draft = logits[:, :n - 1].clone() if drafted else None        # nothing is left of p less q
    lengths = _compare(logits, tokens, g.random((B, n + drafted)), draft=draft, temperatures=temperatures)
    assert lengths[:5] == [4] * 5


def test_trees_with_numbers_that_are_no_nodes():
    g = np.random.default_rng(6)
    B, n, V = 6, 10, 3
    logits = torch.zeros((B, n, V), device="cuda")
    parents = g.integers(-3, n + 2, (B, n))
    tokens = g.integers(-1, V + 1, (B, n))
    for _ in range(5):
        _compare(logits, tokens, g.random((B, n)), parents)
    tokens[:] = 1   # children with one token: the lowest of them
    parents[:, 1:] = 0
    assert _compare(logits, tokens, np.full((B, n), 0.5), parents) == [2] * B
    logits[:] = float("nan")   # the token that is none is nobody's
    tokens[:] = -1
    assert _compare(logits, tokens, np.full((B, n), 0.5), parents) == [1] * B


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("drafted", [False, True])
def test_strides(dtype, drafted):
    """Rows at every alignment, broadcast batches, columns of a wider tensor, and what lies around the rows being anything."""
    g = np.random.default_rng(7)
    B, n = 3, 5
    for V, first in ((1000, 1), (997, 3), (4099, 5), (16, 7), (5, 2)):
        wide = torch.full((B, n, V + 9), float("inf"), dtype=TYPES[dtype], device="cuda")
        wide[:, :, first:first + V] = _logits(g, B, n, V, dtype)
        logits = wide[:, :, first:first + V]
        draft = (logits[:, :n - 1].float() * 0.9).to(TYPES[dtype])[:1].expand(B, n - 1, V) if drafted else None
        parents, tokens = _tree(g, B, n, logits, 50)
        _compare(logits, tokens, g.random((B, n + drafted)), None if drafted else parents, draft=draft)
        _compare(logits.transpose(0, 1).contiguous().transpose(0, 1), tokens, g.random((B, n + drafted)), None if drafted else parents, draft=draft)
        _compare(logits.permute(2, 0, 1).contiguous().permute(1, 2, 0), tokens, g.random((B, n + drafted)), None if drafted else parents, draft=draft)   # copied


@pytest.mark.parametrize("drafted", [False, True])
def test_same_answers_again_replayed_on_another_stream_and_interpreted(drafted):
    from torch.overrides import TorchFunctionMode

    class Mode(TorchFunctionMode):
        def __torch_function__(self, f, types, args=(), kwargs=None):
            return f(*args, **(kwargs or {}))
    g = np.random.default_rng(8)
    B, n, V = 7, 9, 40000
    logits = _logits(g, B, n, V, "bf16")
    parents, tokens = _tree(g, B, n, logits)
    draft = (logits[:, :n - 1].float() * 0.8).to(torch.bfloat16) if drafted else None
    args = (logits, _int(tokens), _f32(g.random((B, n + drafted))))
    more = dict(draft=draft, parents=None if drafted else _int(parents), temperatures=_f32([1, 0, 0.5, 1, 2, 0, 0.8]))
    eager = F.seq_verify(*args, **more)
    with Mode():
        interpreted = F.seq_verify(*args, **more)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        again = F.seq_verify(*args, **more)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = F.seq_verify(*args, **more)
    for a, b, c in zip(eager, interpreted, again):
        assert torch.equal(a, b) and torch.equal(a, c)
    for _ in range(3):
        for t in out:
            t.fill_(-7)
        F.seq_verify(*args, **more)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


@pytest.mark.parametrize("drafted", [False, True])
def test_logits_behind_32_bits(drafted):
    g = np.random.default_rng(31)
    n, V = 5, 1000
    near = [_logits(g, 2, m, V, "f16") for m in (n, n - 1)]
    far = [torch.empty((1 << 31) + 5 + x[0].numel(), dtype=torch.float16, device="cuda").as_strided(x.shape, ((1 << 31) + 5, V, 1)) for x in near]
    for a, b in zip(far, near):
        a.copy_(b)
    tokens, uniforms = _int(g.integers(0, V, (2, n))), _f32(g.uniform(0, 1, (2, n + drafted)))
    results = [F.seq_verify(x, tokens, uniforms, draft=d if drafted else None) for x, d in (near, far)]
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_nothing_to_do():
    path, counts, following = F.seq_verify(torch.zeros((0, 3, 10), device="cuda"), _int(np.zeros((0, 3))), _f32(np.zeros((0, 3))))
    assert path.shape == (0, 3) and counts.shape == following.shape == (0,)
