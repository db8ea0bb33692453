"""The append that picks rows and rotates keys on the way, against the 64-bit oracle and against the plain append."""
import numpy as np
import pytest
import torch

from oracle import seq_oracle
from paper_2204_07143_amd import functional as F

from seq_util import TYPES, f64, normal
from test_gpu_seq_cache import _cache, _int, _same, _table

pytestmark = pytest.mark.gpu

E = 2.0 ** -19   # of the channels of a pair: a rotated value in fp32, see seq_oracle.rotary()


def _freqs(pairs, base=10000.0):
    return torch.tensor([base ** (-i / pairs) for i in range(pairs)], dtype=torch.float32, device="cuda")


def _check_keys(cache, host, k, size, table, lengths, counts):
    """k: the rotated keys in 64 bits, of the tokens appended; size: of each the magnitudes that it is made of.  A page's scale is off by the share of its largest value (and its
    division's rounding, 2^-24), what is stored by half a step of it more."""
    got_cells, got_scales = cache.k_pages.cpu().numpy(), cache.k_scales.cpu().numpy().astype(np.float64)
    page = got_cells.shape[2]
    touched = np.zeros(got_scales.shape[0], bool)
    for b, L in enumerate(lengths):
        for at in range(L // page, (L + counts[b] - 1) // page + 1) if counts[b] > 0 else ():
            lo, hi, i = max(L, at * page), min(L + counts[b], (at + 1) * page), table[b, at]
            touched[i] = True
            new, off, old = k[b, :, lo - L:hi - L], E * size[b, :, lo - L:hi - L], lo - at * page
            before = host[2][i].astype(np.float64) if old else np.zeros(got_scales.shape[1])
            for h in range(new.shape[0]):
                most, worst = np.abs(new[h]).max() / 127, off[h].max() / 127
                want = max(before[h], most)
                scale = got_scales[i, h]
                assert abs(scale - want) <= worst + 2.0 ** -23 * want, (b, at, h)
                cells = got_cells[i, h].astype(np.float64) * scale
                assert (np.abs(cells[old:hi - at * page] - new[h]) <= scale * (0.5 + 2.0 ** -14) + off[h]).all(), (b, at, h)
                held = host[0][i, h, :old].astype(np.float64) * before[h]
                assert (np.abs(cells[:old] - held) <= (scale * (0.5 + 2.0 ** -14) if scale != before[h] else 0.0)).all(), (b, at, h)
                assert np.array_equal(got_cells[i, h, hi - at * page:], host[0][i, h, hi - at * page:])
    assert np.array_equal(got_cells[~touched], host[0][~touched]) and np.array_equal(cache.k_scales.cpu().numpy()[~touched], host[2][~touched])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page,D,pairs", [(16, 32, 8), (32, 64, 32), (64, 128, 64), (128, 128, 40), (128, 32, 16), (16, 128, 0)])
@pytest.mark.parametrize("n", [1, 5, 150])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotated_keys(dtype, page, D, pairs, n, interleaved):
    g = np.random.default_rng(page + n)
    lengths = [0, 1, page - 1, page, 3 * page + 2, 77]
    counts = [n, max(0, n - 1), n, 0, n // 2, n]
    table, pages = _table(g, [x + n for x in lengths], page)
    host, cache = _cache(g, pages, 2, page, D)
    k, v = (normal(g, (6, n, 2, D), dtype, std).transpose(1, 2) for std in (1.0, 4.0))
    weight = torch.from_numpy(g.uniform(0.5, 1.5, D).astype(np.float32)).to(TYPES[dtype if interleaved else "f32"]).cuda() if n != 5 or not pairs else None
    F.seq_cache_append(cache, k, v, _int(table.tolist()), _int(lengths), _int(counts), freqs=_freqs(pairs) if pairs else None, weight=weight, interleaved=interleaved)
    positions = (np.array(lengths)[:, None] + np.arange(n))[:, None]
    if pairs:
        res, bound = seq_oracle.rotary(f64(k), positions, f64(_freqs(pairs)), (pairs,), f64(weight), interleaved=interleaved)
    else:
        res, bound = seq_oracle.rotary(f64(k), positions, np.zeros(1), (1,), f64(weight))
    _check_keys(cache, host, res["z"], bound["z"] / E, table, lengths, counts)
    want = seq_oracle.append(host[1], host[3], v.float().cpu().numpy(), table, lengths, counts)   # values are not rotated
    assert np.array_equal(cache.v_pages.cpu().numpy(), want[0]) and np.array_equal(cache.v_scales.cpu().numpy(), want[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shared", [False, True])
def test_positions_of_the_rows_given(dtype, shared):
    g = np.random.default_rng(1)
    lengths, given, n, page = [0, 40, 17], 30, 19, 32
    table, pages = _table(g, [x + n for x in lengths], page)
    host, cache = _cache(g, pages, 2, page, 64)
    k, v = (normal(g, (3, 2, given, 64), dtype) for _ in range(2))
    positions = g.integers(-5, 1 << 20, (3, given) if shared else (3, 3, given)).astype(np.int32)
    rows = np.stack([g.permutation(given)[:n] for _ in range(3)]).astype(np.int32)
    counts = [n, 3, n + 5]
    F.seq_cache_append(cache, k, v, _int(table.tolist()), _int(lengths), _int(counts), rows=_int(rows.tolist()), positions=torch.from_numpy(positions).cuda(), sections=(8, 4, 4), freqs=_freqs(16))
    res, bound = seq_oracle.rotary(f64(k), positions, f64(_freqs(16)), (8, 4, 4))
    pick = lambda x: np.stack([x[b][:, rows[b]] for b in range(3)])
    _check_keys(cache, host, pick(res["z"]), pick(bound["z"]) / E, table, lengths, [min(c, n) for c in counts])
    want = seq_oracle.append(host[1], host[3], pick(v.float().cpu().numpy()), table, lengths, counts)
    assert np.array_equal(cache.v_pages.cpu().numpy(), want[0]) and np.array_equal(cache.v_scales.cpu().numpy(), want[1])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page,D", [(16, 32), (64, 64), (128, 128)])
def test_rows_alone_are_the_plain_append_of_those_rows(dtype, page, D):
    """The same row twice, rows out of order, none, and one that is no row (a token of zeros)."""
    g = np.random.default_rng(2)
    lengths, given = [0, 5, page - 2, 2 * page], 9
    table, pages = _table(g, [x + 7 for x in lengths], page)
    host, cache = _cache(g, pages, 3, page, D)
    k, v = (normal(g, (4, 3, given, D), dtype) for _ in range(2))
    rows = np.array([[0, 3, 4, 8, -1, -1, -1], [8, 8, 2, 1, 0, 3, 3], [7, 9, 0, 2 ** 31 - 1, 1, -2 ** 31, 2], [1, 2, 3, 4, 5, 6, 7]], np.int32)
    counts = [4, 7, 7, 0]
    F.seq_cache_append(cache, k, v, _int(table.tolist()), _int(lengths), _int(counts), rows=_int(rows.tolist()))
    for i, x in ((0, k), (1, v)):
        there = (rows >= 0) & (rows < given)
        picked = np.stack([x[b].float().cpu().numpy()[:, np.where(there[b], rows[b], 0)] * there[b][None, :, None] for b in range(4)])
        host[i], host[i + 2] = seq_oracle.append(host[i], host[i + 2], picked, table, lengths, counts)
    _same(cache, host)


def test_pages_behind_32_bits():
    g = np.random.default_rng(12)
    kv, page, D, lengths = 8, 64, 128, [60, 0]
    small_table, pages = _table(g, [x + 70 for x in lengths], page, spare=0)
    _, small = _cache(g, pages, kv, page, D)
    far = 70000 - 1 - 3 * np.arange(pages)
    assert far.min() * kv * page * D > 1 << 32
    where = torch.from_numpy(far).cuda()
    large = F.SeqCache(*(torch.empty((70000, *x.shape[1:]), dtype=x.dtype, device="cuda") for x in small))
    for a, b in zip(large, small):
        a[where] = b
    k, v = (normal(g, (2, kv, 70, D), "bf16") for _ in range(2))
    freqs = torch.tensor([0.9 ** i for i in range(32)], device="cuda")
    for cache, table in ((small, small_table), (large, np.where(small_table >= 0, far[np.maximum(small_table, 0)], -1))):
        F.seq_cache_append(cache, k, v, _int(table.tolist()), _int(lengths), freqs=freqs)
    for a, b in zip(large, small):
        assert torch.equal(a[where], b)


def test_more_rows_than_given():
    g = np.random.default_rng(3)
    host, cache = _cache(g, 4, 1, 16, 64)
    x = normal(g, (1, 1, 2, 64), "f16")
    rows = np.array([[0, 1] * 20], np.int32)
    F.seq_cache_append(cache, x, x, _int([[0, 1, 2, 3]]), _int([10]), rows=_int(rows.tolist()))
    for i in (0, 1):
        host[i], host[i + 2] = seq_oracle.append(host[i], host[i + 2], x.float().cpu().numpy()[:, :, rows[0]], np.array([[0, 1, 2, 3]]), [10])
    _same(cache, host)
    with pytest.raises(Exception):   # n tokens of fewer rows need rows
        F.seq_cache_append(cache, x, x[:, :, :1], _int([[0]]), _int([0]), freqs=_freqs(32))


def test_values_that_are_not_ordinary():
    nan, inf = float("nan"), float("inf")
    cache = F.SeqCache.empty(3, 1, 16, 32)
    x = torch.zeros((3, 1, 2, 32), device="cuda")
    x[0, 0, 0, 16:20] = torch.tensor([nan, 1.0, -2.0, 0.5])
    x[1, 0, 1, 16:18] = torch.tensor([inf, 1.0])
    x[2, 0, 0, 0] = 1e-44
    F.seq_cache_append(cache, x, x, _int([[0], [1], [2]]), _int([0, 0, 0]), freqs=_freqs(8))   # channels from 16 on are not rotated
    k, v = F.seq_cache_gather(cache, _int([[0], [1], [2]]), _int([2] * 3), _int([0] * 3), 2, dtype=torch.float32)
    assert torch.equal(k[:2], v[:2]) and k[0, 0, 0, 16] == 0 and k[1, 0, 1, 16] > 3.4e38
    # (the largest fp32 number over 127, rounded, and times 127 again passes it by 2^-25: read back in fp32 it is infinite, as after the plain append; 127 is what is stored)
    assert cache.k_pages[1, 0, 1, 16] == 127 and torch.isfinite(cache.k_scales).all() and torch.isfinite(k[[0, 2]]).all()


def test_pages_that_are_none_and_lengths_out_of_range():
    g = np.random.default_rng(4)
    big = 2 ** 31 - 1
    table = np.array([[1, 50, 0, -1], [2, 3, 4, 6], [5, 5, 5, 5], [5, 5, 5, 5]], np.int32)
    host, cache = _cache(g, 6, 2, 16, 64)
    x = normal(g, (4, 2, 70, 64), "f16")
    F.seq_cache_append(cache, x, x, _int(table.tolist()), _int([0, 0, -5, big]), _int([70, big, 70, 70]), rows=_int([list(range(70))] * 4))
    for i in (0, 1):
        host[i], host[i + 2] = seq_oracle.append(host[i], host[i + 2], x.float().cpu().numpy()[:2], table[:2], [0, 0])
    _same(cache, host)


def test_replayed_and_interpreted():
    from torch.overrides import TorchFunctionMode

    class Mode(TorchFunctionMode):
        def __torch_function__(self, f, types, args=(), kwargs=None):
            return f(*args, **(kwargs or {}))
    g = np.random.default_rng(5)
    table, pages = _table(g, [300, 17], 16)
    host, _ = _cache(g, pages, 2, 16, 128)
    fresh = lambda: F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
    k, v = (normal(g, (2, 2, 5, 128), "bf16") for _ in range(2))
    table, lengths, rows, freqs, w = _int(table.tolist()), _int([290, 10]), _int([[0, 2, 4], [1, 3, -1]]), _freqs(64), torch.ones(128, device="cuda", dtype=torch.bfloat16)
    call = lambda cache: F.seq_cache_append(cache, k, v, table, lengths, rows=rows, freqs=freqs, weight=w)
    eager, other, captured = fresh(), fresh(), fresh()
    call(eager)
    with Mode():
        call(other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(captured)
    for _ in range(3):
        for a, b in zip(captured, host):
            a.copy_(torch.from_numpy(b))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(eager, other, captured):
            assert torch.equal(a, b) and torch.equal(a, c)
