"""Attention of drafted trees in tiles (more than 32 rows to a key head, and enough work): what it forms in another way than the kernel of few rows, against the 64-bit oracle.  Each test
says from the size of the workspace that the call goes in tiles."""
import numpy as np
import pytest
import torch

from oracle import seq_oracle
from paper_2204_07143_amd import binding as na
from paper_2204_07143_amd import functional as F

from seq_util import TYPES, f64, normal
from test_gpu_seq_cache import _cache, _int, _table
from test_gpu_seq_tree import _check, _inputs, _parents

pytestmark = pytest.mark.gpu


def in_tiles(q, cache, table, window=None, softcap=None):
    """Whether the workspace of the call is what partial rows of tiles take: sums, maximum and total of two runs for each workgroup."""
    B, heads, n, D = q.shape
    pages, kv, page, _ = cache.k_pages.shape
    p = na.seq_cache_problem(q, cache.k_pages, table, heads=heads, window=window or 0, softcap=softcap or 0.0, out=q)
    rows, longest = heads // kv * n, table.shape[1] * page
    blocks = min(range(1, 3 if D == 128 and softcap and softcap > 1024 else 4), key=lambda rb: -(-rows // (64 * rb)) * (rb + 0.6))
    tiles = B * kv * -(-rows // (64 * blocks)) * (-(-min(longest, (window or 2 ** 31 - 1) + 64) // 64) + 1)
    return na.seq_cache_tree_attention_workspace_bytes(p) == max(1, min(512, tiles // 2)) * 2 * 64 * blocks * (D + 2) * 4


def _wide(table, page, tokens, fill=-9):
    """The table with columns for `tokens` tokens: work enough for tiles, by what it may hold."""
    return np.concatenate([table, np.full((len(table), tokens // page - table.shape[1]), fill, np.int32)], 1)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("cap,slope", [(None, 0.0), (5.0, 0.0), (None, 0.03)])
def test_scales_far_apart_pages_that_are_none_and_never_written(page, cap, slope):
    g = np.random.default_rng(2)
    table = np.array([[0, 1, 2, 3], [0, 1, 4, 4], [1, 50, 0, -1]], np.int32)
    host, _ = _cache(g, 6, 2, page, 64)
    host[3][:, 0] = [1e-6, 1e3, 1.0, 0.0, 1e-3, 1.0]
    host[2][5] = host[3][5] = float("nan")
    lengths, n = [4 * page, 4 * page - 3, 4 * page], 40
    q, k, v = _inputs(g, 3, 4, 2, n, 64, "bf16")
    cache = F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
    parents = np.tile(np.arange(-1, n - 1, dtype=np.int32), (3, 1))
    slopes = torch.full((4,), slope, device="cuda") if slope else None
    results = []
    for behind in (-1, 5):   # behind the sequences
        wide = _int(_wide(table, page, 16384, behind).tolist())
        assert in_tiles(q, cache, wide, softcap=cap)
        results.append(F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, wide, _int(lengths), softcap=cap, slopes=slopes))
        _check(results[-1], q, k, v, parents, host, table, lengths, "bf16", softcap=cap, slopes=None if slopes is None else f64(slopes))
    assert torch.equal(*results)


@pytest.mark.parametrize("window", [None, 70])
def test_lengths_out_of_range(window):
    g = np.random.default_rng(3)
    big, n, B = 2 ** 31 - 1, 40, 4 if window is None else 200
    table = np.full((B, 2), -9, np.int32)
    table[:4] = [[0, 1], [2, 3], [4, 5], [1, 3]]
    host, cache = _cache(g, 6, 1, 16, 32)
    q, k, v = _inputs(g, B, 8, 1, n, 32, "f16")
    parents = np.tile(np.arange(-1, n - 1, dtype=np.int32), (B, 1))
    wide = _int(_wide(table, 16, 4096).tolist())
    assert in_tiles(q, cache, wide, window)
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, wide, _int(([-5, big, -big - 1, 32] + [0] * B)[:B]), window=window)
    for b in range(4):   # what lies past the table has no page, and what a length leaves behind the window is not seen
        seen = 0 if b % 2 == 0 or (b == 1 and window) else 32
        _check(got[b:b + 1], q[b:b + 1], k[b:b + 1], v[b:b + 1], parents[:1], host, table[b:b + 1], [seen], "f16", window=window)


@pytest.mark.parametrize("std", [1e-3, 1e3])
@pytest.mark.parametrize("dtype,D", [("f16", 32), ("bf16", 128)])
def test_queries_of_any_size(std, dtype, D):
    g = np.random.default_rng(4)
    table, pages = _table(g, [90, 90], 16)
    host, cache = _cache(g, pages, 1, 16, D)
    q, k, v = _inputs(g, 2, 4, 1, 12, D, dtype)
    q = (q.float() * std).to(TYPES[dtype])
    parents, wide = _parents(g, 2, 12), _int(_wide(table, 16, 65536).tolist())
    assert in_tiles(q, cache, wide)
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, wide, _int([90, 90]), scale=0.2 / std)
    _check(got, q, k, v, parents, host, table, [90, 90], dtype, scale=float(np.float32(0.2 / std)))


@pytest.mark.parametrize("dtype,D", [("f16", 128), ("bf16", 64), ("bf16", 128), ("f16", 32)])
def test_values_that_are_no_numbers_within_a_window(dtype, D):
    """The rows that see them have what they are, the others their bits: of many sequences, since a window leaves few tiles to each."""
    g = np.random.default_rng(21)
    B, n, window, inf = 220, 40, 3, float("inf")
    lengths = [100, 0, 33] + [int(x) for x in g.integers(0, 64, B - 3)]
    table, pages = _table(g, lengths, 32)
    host, cache = _cache(g, pages, 2, 32, D)
    q, k, v = _inputs(g, B, 8, 2, n, D, dtype)
    parents = _parents(g, B, n)
    wild = {(1, 0): inf, (2, 7): -inf, (3, 7): float("nan"), (4, D - 1): inf, (n - 2, 9): -inf}
    for (node, channel) in wild:
        v[:, :, node, channel] = 0
    assert in_tiles(q, cache, _int(table.tolist()), window)
    call = lambda v: F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int(lengths), window=window)
    clean, bad = call(v), v.clone()
    _check(clean[:6], q[:6], k[:6], v[:6], parents[:6], host, table[:6], lengths[:6], dtype, window=window)
    see = torch.from_numpy(np.stack([seq_oracle.tree(None, None, None, x, np.zeros(0, bool), 0, window)[0] for x in parents.tolist()])).cuda()
    expected = clean.clone()
    for (node, channel), x in wild.items():
        bad[:, :, node, channel] = x
        expected[..., channel] += torch.where(see[:, None, :, node], x, 0.0).to(expected.dtype)
    got = call(bad)
    assert torch.equal(got.isnan(), expected.isnan()) and torch.equal(got.nan_to_num(nan=0.0, posinf=1e4, neginf=-1e4), expected.nan_to_num(nan=0.0, posinf=1e4, neginf=-1e4))


@pytest.mark.parametrize("dtype,D", [("f16", 64), ("bf16", 128)])
@pytest.mark.parametrize("cap", [1025.0, 4096.0])
def test_large_caps(dtype, D, cap):
    g = np.random.default_rng(5)
    lengths = [200, 33]
    table, pages = _table(g, lengths, 32)
    host, cache = _cache(g, pages, 2, 32, D)
    q, k, v = _inputs(g, 2, 4, 2, 40, D, dtype, 2.0)
    parents, wide = _parents(g, 2, 40), _int(_wide(table, 32, 16384).tolist())
    assert in_tiles(q, cache, wide, softcap=cap)
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, wide, _int(lengths), softcap=cap)
    _check(got, q, k, v, parents, host, table, lengths, dtype, softcap=cap)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,tiled", [(1, False), (6, False), (40, True)])
@pytest.mark.parametrize("window,slope", [(None, 0.0), (1, 0.0), (7, 0.02), (64, 0.0), (100, 0.01)])
def test_a_line_beside_the_cache_and_appended_to_it(dtype, n, tiled, window, slope):
    """Nodes in a line are the newest tokens: seq_cache_attention has them in the same places, with the same window.  Their keys and values are 127ths on the cache's scales, so that an append
    rounds nothing, and both calls have one oracle."""
    g = np.random.default_rng(6)
    B = 400 if tiled and window else 2
    lengths = [70, 129] + [int(x) for x in g.integers(0, 30, B - 2)]
    table, pages = _table(g, [x + n for x in lengths], 16)
    host, _ = _cache(g, pages, 2, 16, 64)
    for scales in host[2:]:
        scales[:] = 2.0 ** -6
    cache = F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
    q = next(_inputs(g, B, 8, 2, n, 64, dtype))
    k, v = (g.integers(-127, 128, (B, 2, n, 64)) for _ in range(2))
    k[..., 0] = v[..., 3] = 127
    k, v = (torch.from_numpy((x * 2.0 ** -6).astype(np.float32)).to(TYPES[dtype]).cuda() for x in (k, v))
    line = np.tile(np.arange(-1, n - 1, dtype=np.int32), (B, 1))
    slopes = torch.full((8,), slope, device="cuda") if slope else None
    few = slice(0, 8)
    wide = _int(table.tolist() if window or not tiled else _wide(table, 16, 16384).tolist())
    assert in_tiles(q, cache, wide, window) == tiled
    beside = F.seq_cache_tree_attention(q, k, v, _int(line.tolist()), cache, wide, _int(lengths), window=window, slopes=slopes)
    F.seq_cache_append(cache, k, v, wide, _int(lengths))
    assert all((x == 2.0 ** -6).all() for x in cache[2:])
    appended = F.seq_cache_attention(q, cache, wide, _int([x + n for x in lengths]), window=window, slopes=slopes)
    for got in (beside, appended):
        _check(got[few], q[few], k[few], v[few], line[few], host, table[few], lengths[few], dtype, window=window, slopes=None if slopes is None else f64(slopes))
