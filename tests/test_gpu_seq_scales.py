"""A cached value is its integer times its page's scale, whatever a caller's scales are."""
import numpy as np
import pytest
import torch

from oracle import seq_oracle
from paper_2204_07143_amd import functional as F

from seq_util import f64, normal
from test_gpu_seq_cache import _cache, _check_attention, _int, _table
from test_gpu_seq_tree import _check, _inputs, _parents
from test_gpu_seq_tree_tiles import _wide, in_tiles

pytestmark = pytest.mark.gpu


def _trees(g, host, table, lengths, n, dtype, tiled, cap=None, slope=0.0, scale=None, std=1.0):
    """Trees over a cache, in tiles or not, against the oracle."""
    kv, page, D = host[0].shape[1:]
    heads = 4 * kv
    cache = F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
    q, k, v = _inputs(g, len(lengths), heads, kv, n, D, dtype, std)
    parents = _parents(g, len(lengths), n)
    slopes = torch.full((heads,), slope, device="cuda") if slope else None
    wide = _int(_wide(table, page, 32768).tolist() if tiled else table.tolist())
    assert in_tiles(q, cache, wide, softcap=cap) == tiled
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, wide, _int(lengths), softcap=cap, slopes=slopes, scale=scale)
    assert torch.isfinite(got).all()
    _check(got, q, k, v, parents, host, table, lengths, dtype, softcap=cap, slopes=None if slopes is None else f64(slopes), scale=scale)


@pytest.mark.parametrize("dtype,D", [("f16", 64), ("bf16", 128), ("f16", 32)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("cap,slope,scale", [(None, 0.0, None), (5.0, 0.0, None), (1500.0, 0.0, None), (None, 0.02, None), (None, 0.0, -0.2)])
@pytest.mark.parametrize("tiled", [False, True])
def test_trees_with_scales_of_either_sign(dtype, D, page, cap, slope, scale, tiled):
    g = np.random.default_rng(page + D)
    lengths, n = [700, 0, 257], 40
    table, pages = _table(g, lengths, page)
    host, _ = _cache(g, pages, 2, page, D)
    for scales in host[2:]:
        scales *= g.choice([-1, 1], scales.shape).astype(np.float32)
    _trees(g, host, table, lengths, n, dtype, tiled, cap, slope, scale)


@pytest.mark.parametrize("page", [16, 64])
def test_read_back_and_attention_with_scales_of_either_sign(page):
    g = np.random.default_rng(page)
    lengths = [300, 77]
    table, pages = _table(g, lengths, page)
    host, _ = _cache(g, pages, 2, page, 64)
    for scales in host[2:]:
        scales *= g.choice([-1, 1], scales.shape).astype(np.float32)
    cache = F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
    for got, i in zip(F.seq_cache_gather(cache, _int(table.tolist()), _int(lengths), _int([0, 0]), 300, dtype=torch.float32), (0, 1)):
        assert np.array_equal(got.cpu().numpy(), seq_oracle.gather(host[i], host[i + 2], table, lengths, [0, 0], 300).astype(np.float32))   # (7 bits times 24: the 64-bit product is exact)
    for n, softcap in ((1, None), (9, None), (9, 5.0)):
        q = normal(g, (2, 8, n, 64), "f16")
        got = F.seq_cache_attention(q, cache, _int(table.tolist()), _int(lengths), softcap=softcap)
        _check_attention(got, q, host, table, lengths, "f16", softcap=softcap)


@pytest.mark.parametrize("picked", [False, True])
@pytest.mark.parametrize("std", [0.1, 1.0, 50.0])   # the page's scale holds, grows, grows much
def test_appends_to_pages_of_a_scale_below_zero(picked, std):
    g = np.random.default_rng(3)
    page, D, L, n = 32, 64, 20, 9
    host, _ = _cache(g, 2, 2, page, D)
    host[0][1, 0, 3, 5] = -128   # (a caller's: an append leaves none)
    for scales in host[2:]:
        scales *= -1
    cache = F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
    table, k, v = np.array([[1]], np.int32), *(normal(g, (1, 2, n, D), "f32", std) for _ in range(2))
    F.seq_cache_append(cache, k, v, _int(table.tolist()), _int([L]), rows=_int([list(range(n))]) if picked else None)
    for got, i, new in zip(F.seq_cache_gather(cache, _int(table.tolist()), _int([L + n]), _int([0]), L + n, dtype=torch.float32), (0, 1), (k, v)):
        want = np.concatenate([seq_oracle.gather(host[i], host[i + 2], table, [L], [0], L), f64(new)], 2)
        before, step = np.abs(host[i + 2][1]).astype(np.float64), np.abs(f64(cache[i + 2][1]))
        assert (step >= before).all() and (step >= np.abs(f64(new)[0]).max((1, 2)) / 127 * (1 - 2.0 ** -22)).all()
        want = np.clip(want, -127 * step[None, :, None, None], 127 * step[None, :, None, None])   # (128 of the old one's, where the new one has its size)
        assert (np.abs(f64(got) - want) <= (0.5 + 127 * 2.0 ** -22) * step[None, :, None, None]).all()   # half a step; the scale's own and the ratio's rounding, 127 times at most
        cells, scales = seq_oracle.append(host[i], host[i + 2], new.cpu().numpy(), table, [L])
        assert np.array_equal(cache[i].cpu().numpy(), cells) and np.array_equal(cache[i + 2].cpu().numpy(), scales)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("cap,slope", [(None, 0.0), (5.0, 0.0), (None, 0.02)])
@pytest.mark.parametrize("large,small", [(2.0 ** 20, 0.0), (2.0 ** 110, 0.0), (1e-2, 0.0), (1e-25, 0.0), (0.0, 0.0), (2.0 ** 40, 2.0 ** -60), (-1.0, -0.0)])
@pytest.mark.parametrize("tiled", [False, True])
def test_pages_of_no_values_count_in_the_sums(page, cap, slope, large, small, tiled):
    """Values that are 0, or as good as that, beside large ones: their tokens' weights are part of a row's sum all the same."""
    g = np.random.default_rng(page)
    lengths, n = [500, 64, 1, 130], 40
    table, pages = _table(g, lengths, page)
    host, _ = _cache(g, pages, 2, page, 64)
    host[3][:] = np.where(g.random(host[3].shape) < 0.3, large, small)
    host[3][table[1]] = small   # a sequence of nothing else
    _trees(g, host, table, lengths, n, "bf16", tiled, cap, slope, std=1.5)


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("score,power", [(-4, -99), (20, -99), (-6, -97), (0, -60)])
@pytest.mark.parametrize("tiled", [False, True])
def test_weights_next_to_the_least_that_count(page, score, power, tiled):
    """Scores in base 2 that are whole numbers: weight times value scale of most tokens is 2^-124 of the first page's in the first and the third case, and they are most of a row's sum."""
    g = np.random.default_rng(page)
    L, n, D, heads = 40 * page + 5, 40, 64, 4
    table, pages = _table(g, [L], page)
    host, _ = _cache(g, pages, 1, page, D)
    host[0][:] = 0
    host[0][..., 0] = score
    host[0][table[0, 0], ..., 0] = 0
    host[2][:], host[3][:], host[3][table[0, 0]] = 1.0, 2.0 ** power, 2.0 ** 21
    cache = F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
    q, k, v = (normal(g, (1, h, n, D), "bf16") for h in (heads, 1, 1))
    q[..., 0], k[..., 0] = 1, 0
    q[..., 1:], k[..., 1:] = 0, 0
    parents = np.tile(np.arange(-1, n - 1, dtype=np.int32), (1, 1))
    wide = _int(_wide(table, page, 65536).tolist() if tiled else table.tolist())
    assert in_tiles(q, cache, wide) == tiled
    scale = float(np.float32(np.log(2.0)))
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, wide, _int([L]), scale=scale)
    _check(got, q, k, v, parents, host, table, [L], "bf16", scale=scale)
