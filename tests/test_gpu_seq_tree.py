"""Attention of drafted trees over the cache against the 64-bit oracle, and all of a server's step together."""
import numpy as np
import pytest
import torch

from oracle import seq_oracle
from paper_2204_07143_amd import functional as F

from seq_util import FP32, HALF, TINY, TYPES, check, f64, normal
from test_gpu_seq_cache import _cache, _int, _table

pytestmark = pytest.mark.gpu


def _parents(g, B, n):
    """Trees, with second roots, and numbers that are no nodes."""
    parents = np.stack([[-1] + [int(g.integers(max(-1, (i - 1) // 2 - 2), i)) for i in range(1, n)] for _ in range(B)]).astype(np.int32)
    for b in range(1, B, 2):
        parents[b, g.integers(0, n)] = g.choice([-2, n, -2 ** 31, 2 ** 31 - 1, n - 1])
    return parents


def _check(got, q, k, v, parents, host, table, lengths, dtype, window=None, softcap=None, slopes=None, scale=None):
    """Over the cache as its attention has it; nodes' weights to fp16, or to 2^-17 of them: the same bound covers both."""
    B, heads, n, D = q.shape
    pages, kv, page, _ = host[0].shape
    group = heads // kv
    for b, L in enumerate(lengths):
        L = max(L, 0)
        kc, vc = (seq_oracle.gather(host[i], host[i + 2], table[b:b + 1], [L], [0], L)[0] for i in (0, 1))
        see, far = seq_oracle.tree(None, None, None, parents[b].tolist(), seq_oracle.present(pages, page, table[b], L), L, window)
        nodes = np.array(seq_oracle.depths(parents[b].tolist())) >= 0
        own = [np.where(nodes[None, :, None], f64(x[b]), 0.0) for x in (k, v)]   # the others may be anything
        for h in range(heads):
            keys, values = (np.concatenate([c[h // group], x[h // group]]) for c, x in zip((kc, vc), own))
            res, bound = seq_oracle.head(f64(q[b, h]), keys, values, None, see, scale=D ** -0.5 if scale is None else scale, softcap=softcap, slope=0.0 if slopes is None else float(slopes[h]),
                                         u=HALF["f16"], e=FP32, tiny=TINY["f16"], far=far)
            check(f"sequence {b}, head {h}", got[b, h], res["out"], bound["out"] + HALF[dtype] * np.abs(res["out"]))
            assert (got[b, h][torch.from_numpy(~nodes).cuda()] == 0).all()


def _inputs(g, B, heads, kv, n, D, dtype, std=1.0):
    return (normal(g, (B, n, h, D), dtype, std).transpose(1, 2) for h in (heads, kv, kv))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("page,D", [(16, 32), (16, 128), (32, 64), (64, 128), (128, 32), (128, 64)])
@pytest.mark.parametrize("n,heads,kv", [(1, 2, 2), (7, 4, 2), (20, 6, 1), (64, 4, 1)])
@pytest.mark.parametrize("cap", [None, 5.0])
def test_trees(dtype, page, D, n, heads, kv, cap):
    g = np.random.default_rng(D + page + n)
    lengths = [1, 0, page, 31, 33, 300]
    table, pages = _table(g, lengths, page)
    host, cache = _cache(g, pages, kv, page, D)
    q, k, v = _inputs(g, len(lengths), heads, kv, n, D, dtype)
    parents = _parents(g, len(lengths), n)
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int(lengths), softcap=cap)
    _check(got, q, k, v, parents, host, table, lengths, dtype, softcap=cap)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (16, 1), (10, 2), (5, 5)])
@pytest.mark.parametrize("n", [1, 2, 13, 16, 17, 48, 63])
def test_rows_and_slopes(heads, kv, n):
    g = np.random.default_rng(heads + n)
    lengths = [5, 150, 64, 0]
    table, pages = _table(g, lengths, 32)
    host, cache = _cache(g, pages, kv, 32, 64)
    q, k, v = (normal(g, (4, h, n, 64), "bf16") for h in (heads, kv, kv))
    slopes = torch.from_numpy(g.uniform(0, 0.2, heads).astype(np.float32)).cuda()
    parents = _parents(g, 4, n)
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int(lengths), slopes=slopes, scale=0.05)
    _check(got, q, k, v, parents, host, table, lengths, "bf16", slopes=f64(slopes), scale=0.05)


@pytest.mark.parametrize("window", [1, 2, 5, 64, 1000, 100000])
@pytest.mark.parametrize("page,n,heads", [(16, 3, 2), (64, 30, 4), (128, 64, 4)])
def test_windows_and_long_ranges(window, page, n, heads):
    g = np.random.default_rng(window)
    lengths = [5001, 40, 2]
    table, pages = _table(g, lengths, page)
    host, cache = _cache(g, pages, 1, page, 64)
    q, k, v = _inputs(g, 3, heads, 1, n, 64, "f16", 1.5)
    parents = _parents(g, 3, n)
    parents[0] = np.arange(-1, n - 1)   # a line: as deep as it gets
    slopes = torch.full((heads,), 0.01, device="cuda") if window == 1000 else None
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int(lengths), window=window, slopes=slopes)
    _check(got, q, k, v, parents, host, table, lengths, "f16", window=window, slopes=None if slopes is None else f64(slopes))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,page", [(32, 64), (64, 16), (128, 32), (128, 128)])
@pytest.mark.parametrize("n,heads", [(31, 6), (12, 8), (33, 1), (64, 3), (64, 9)])   # 186, 96, 33, 192 and 576 rows
@pytest.mark.parametrize("cap,window", [(None, None), (5.0, None), (1500.0, None), (None, 70), (5.0, 300)])
@pytest.mark.parametrize("wide", [False, True])   # a table that may hold long sequences makes it a large call: tiles
def test_many_rows_to_a_key_head(dtype, D, page, n, heads, cap, window, wide):
    g = np.random.default_rng(n + heads + D)
    lengths = [700, 64, 0, 129] + [5] * (0 if window is None or not wide else 65536 // (window // 64 + 1) // (n * heads) - 3)
    table, pages = _table(g, lengths, page, width=max(-(-700 // page), 65536 * 64 // (4 * n * heads * page) + 1) if wide else None)
    host, cache = _cache(g, pages, 1, page, D)
    q, k, v = _inputs(g, len(lengths), heads, 1, n, D, dtype)
    parents = _parents(g, len(lengths), n)
    slopes = torch.from_numpy(g.uniform(0, 0.1, heads).astype(np.float32)).cuda() if window == 300 else None
    scale = -0.1 if window == 70 else None   # a scale may be negative
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int(lengths), softcap=cap, window=window, slopes=slopes, scale=scale)
    _check(got, q, k, v, parents, host, table, lengths, dtype, softcap=cap, window=window, slopes=None if slopes is None else f64(slopes), scale=scale)


def test_many_short_sequences():
    """More sequences than a wave has lanes, some of nothing: runs that hold several rows' work, and rows that several runs hold."""
    g = np.random.default_rng(13)
    lengths = [int(x) for x in g.integers(0, 300, 150)]
    table, pages = _table(g, lengths, 16, width=40)
    host, cache = _cache(g, pages, 2, 16, 32)
    q, k, v = _inputs(g, 150, 6, 2, 20, 32, "f16")
    parents = _parents(g, 150, 20)
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int(lengths))
    _check(got, q, k, v, parents, host, table, lengths, "f16")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,width", [(5, None), (40, None), (40, 200)])   # few rows, many, and many of a large call
def test_what_is_no_node_may_be_anything(dtype, n, width):
    g = np.random.default_rng(1)
    lengths = [100, 33, 0]
    table, pages = _table(g, lengths, 32, width=width)
    host, cache = _cache(g, pages, 2, 32, 64)
    q, k, v = _inputs(g, 3, 8, 2, n, 64, dtype)
    parents = np.stack([[-1] + [0] * (n - 1), [-1, 0] + [-2] * (n - 2), [-2] + [0] * (n - 1)]).astype(np.int32)
    for t in (q, k, v):
        t[1, :, 2:] = float("nan")
        t[2] = float("inf")
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int(lengths))
    _check(got, torch.nan_to_num(q, 0, 0, 0), k, v, parents, host, table, lengths, dtype)
    assert (got[2] == 0).all() and (got[1, :, 2:] == 0).all() and torch.isfinite(got).all()


@pytest.mark.parametrize("dtype,D", [("f16", 128), ("bf16", 64), ("bf16", 128), ("f16", 32)])
@pytest.mark.parametrize("n,width,window", [(5, None, None), (40, None, 3), (40, 400, None), (40, 400, 3)])
def test_values_that_are_no_numbers_reach_the_rows_that_see_them_alone(dtype, D, n, width, window):
    """Products have 0 where a value is infinite or none: the other rows keep their bits."""
    g = np.random.default_rng(21)
    lengths = [100, 0, 33]
    table, pages = _table(g, lengths, 32, width=width)
    host, cache = _cache(g, pages, 2, 32, D)
    q, k, v = _inputs(g, 3, 8, 2, n, D, dtype)
    parents = np.stack([[-1] + [(i - 1) // 2 for i in range(1, n)], np.arange(-1, n - 1), [-1] + [max(i - 2, 0) for i in range(1, n)]]).astype(np.int32)
    wild = {(1, 0): "inf", (2, 7): "-inf", (3, 7): "nan", (4, D - 1): "inf", (n - 2, 9): "-inf"}
    for (node, channel) in wild:
        v[:, :, node, channel] = 0
    call = lambda k, v: F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int(lengths), window=window)
    clean = call(k, v)
    _check(clean, q, k, v, parents, host, table, lengths, dtype, window=window)
    expected, bad, all_of = clean.clone(), v.clone(), clean.clone()
    for b in range(3):
        see = seq_oracle.tree(None, None, None, parents[b].tolist(), np.zeros(0, bool), 0, window)[0]
        for (node, channel), x in wild.items():
            rows = torch.from_numpy(see[:, node].astype(bool)).cuda()
            expected[b, :, rows, channel] += float(x)
            all_of[b, :, rows] = float("nan") if node == 2 else all_of[b, :, rows]
    for (node, channel), x in wild.items():
        bad[:, :, node, channel] = float(x)
    got = call(k, bad)
    assert torch.equal(got.isnan(), expected.isnan()) and torch.equal(got.nan_to_num(nan=0.0, posinf=1e4, neginf=-1e4), expected.nan_to_num(nan=0.0, posinf=1e4, neginf=-1e4))
    bad = k.clone()
    bad[:, :, 2, 3] = float("nan")
    got = call(bad, v)
    assert torch.equal(got.isnan(), all_of.isnan()) and torch.equal(got.nan_to_num(nan=0.0), all_of.nan_to_num(nan=0.0))


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("n", [3, 40])
def test_scales_far_apart_pages_that_are_none_and_never_written(page, n):
    g = np.random.default_rng(2)
    table = np.array([[0, 1, 2, 3], [0, 1, 4, 4], [1, 50, 0, -1]], np.int32)
    host, _ = _cache(g, 6, 2, page, 64)
    host[3][:, 0] = [1e-6, 1e3, 1.0, 0.0, 1e-3, 1.0]
    host[2][5] = host[3][5] = float("nan")
    lengths = [4 * page, 4 * page - 3, 4 * page]
    q, k, v = _inputs(g, 3, 4, 2, n, 64, "bf16")
    results = []
    for behind in (-1, 5):   # behind the sequences
        wide = np.concatenate([table, np.full((3, 2 if n == 3 else 8192 // page), behind, np.int32)], 1)
        cache = F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
        parents = np.tile(np.arange(-1, n - 1, dtype=np.int32), (3, 1))
        results.append(F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(wide.tolist()), _int(lengths)))
        _check(results[-1], q, k, v, parents, host, table, lengths, "bf16")
    assert torch.equal(*results)


@pytest.mark.parametrize("n", [3, 40])
def test_lengths_out_of_range(n):
    g = np.random.default_rng(3)
    big = 2 ** 31 - 1
    table = np.array([[0, 1], [2, 3], [4, 5]], np.int32)
    host, cache = _cache(g, 6, 1, 16, 32)
    q, k, v = _inputs(g, 3, 2, 1, n, 32, "f16")
    parents = np.tile(np.arange(-1, n - 1, dtype=np.int32), (3, 1))
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int([-5, big, -big - 1]))
    _check(got[:1], q[:1], k[:1], v[:1], parents, host, table, [0], "f16")
    _check(got[2:], q[2:], k[2:], v[2:], parents, host, table, [0], "f16")
    _check(got[1:2], q[1:2], k[1:2], v[1:2], parents, host, table[1:], [32], "f16")   # what lies past the table has no page


@pytest.mark.parametrize("std", [1e-3, 1e3])
def test_queries_of_any_size(std):
    g = np.random.default_rng(4)
    table, pages = _table(g, [90, 90], 16)
    host, cache = _cache(g, pages, 1, 16, 32)
    for dtype in ("f16", "bf16"):
        q, k, v = _inputs(g, 2, 4, 1, 12, 32, dtype)
        q = (q.float() * std).to(TYPES[dtype])
        parents = _parents(g, 2, 12)
        got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int([90, 90]), scale=0.2 / std)
        _check(got, q, k, v, parents, host, table, [90, 90], dtype, scale=float(np.float32(0.2 / std)))


@pytest.mark.parametrize("cap", [1025.0, 4096.0])
@pytest.mark.parametrize("n", [3, 40])
def test_large_caps(cap, n):
    g = np.random.default_rng(5)
    lengths = [200, 33]
    table, pages = _table(g, lengths, 32)
    host, cache = _cache(g, pages, 2, 32, 64)
    q, k, v = _inputs(g, 2, 4, 2, n, 64, "bf16", 2.0)
    parents = _parents(g, 2, n)
    got = F.seq_cache_tree_attention(q, k, v, _int(parents.tolist()), cache, _int(table.tolist()), _int(lengths), softcap=cap)
    _check(got, q, k, v, parents, host, table, lengths, "bf16", softcap=cap)


def test_a_line_is_the_attention_of_the_newest_tokens():
    """Nodes in a line, once beside the cache and once appended to it, with one scale for all: both within their bounds of the oracle's, whose keys differ by the 8 bits alone."""
    g = np.random.default_rng(6)
    lengths, n = [70, 129], 6
    table, pages = _table(g, [x + n for x in lengths], 16)
    host, cache = _cache(g, pages, 2, 16, 64)
    q, k, v = _inputs(g, 2, 4, 2, n, 64, "f16")
    line = np.tile(np.arange(-1, n - 1, dtype=np.int32), (2, 1))
    got = F.seq_cache_tree_attention(q, k, v, _int(line.tolist()), cache, _int(table.tolist()), _int(lengths))
    _check(got, q, k, v, line, host, table, lengths, "f16")


def test_same_bits_again_replayed_on_another_stream_and_interpreted():
    from torch.overrides import TorchFunctionMode

    class Mode(TorchFunctionMode):
        def __torch_function__(self, f, types, args=(), kwargs=None):
            return f(*args, **(kwargs or {}))
    g = np.random.default_rng(7)
    for n, width in ((5, None), (48, None), (48, 700)):   # few rows, many, and many of a large call
        table, pages = _table(g, [3000, 17], 16, width=width)
        _, cache = _cache(g, pages, 2, 16, 128)
        q, k, v = _inputs(g, 2, 8, 2, n, 128, "bf16")
        args = (q, k, v, _int(_parents(g, 2, n).tolist()), cache, _int(table.tolist()), _int([2990, 10]))
        eager = F.seq_cache_tree_attention(*args)
        with Mode():
            interpreted = F.seq_cache_tree_attention(*args)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            again = F.seq_cache_tree_attention(*args)
        stream.synchronize()
        assert torch.equal(eager, again) and torch.equal(eager, interpreted)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = F.seq_cache_tree_attention(*args)
        for _ in range(3):
            out.fill_(float("nan"))
            F.seq_cache_tree_attention(*args)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager)


@pytest.mark.parametrize("n,width", [(5, None), (48, 700)])
def test_lengths_and_tables_that_change_between_replays(n, width):
    """Two graphs of one stream, each replayed after the sequences have grown and their pages have moved."""
    g = np.random.default_rng(17)
    table, pages = _table(g, [3000, 900], 16, width=width)
    _, cache = _cache(g, pages, 2, 16, 64)
    calls = []
    for _ in range(2):
        q, k, v = _inputs(g, 2, 8, 2, n, 64, "f16")
        calls.append((q, k, v, _int(_parents(g, 2, n).tolist()), cache, _int(table.tolist()), _int([1, 0])))
    F.seq_cache_tree_attention(*calls[0])
    torch.cuda.synchronize()
    graphs, outs = [], []
    for args in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(F.seq_cache_tree_attention(*args))
    for lengths in ([3000, 900], [0, 17], [64, 2000], [1500, 1]):
        moved = np.roll(table, 1, axis=0)
        for args in calls:
            args[5].copy_(torch.from_numpy(moved).cuda()), args[6].copy_(_int(lengths))
        table = moved
        for graph in graphs:
            graph.replay()
        eager = [F.seq_cache_tree_attention(*args) for args in calls]
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)


@pytest.mark.parametrize("n,width", [(5, 7), (20, 7), (20, 200)])   # few rows, many, and many of a large call
def test_pages_behind_32_bits(n, width):
    g = np.random.default_rng(8)
    kv, page, D = 8, 64, 128
    small_table, pages = _table(g, [400, 150], page, spare=0, width=width)
    _, small = _cache(g, pages, kv, page, D)
    far = 70000 - 1 - 3 * np.arange(pages)
    assert far.min() * kv * page * D > 1 << 32
    where = torch.from_numpy(far).cuda()
    large = F.SeqCache(*(torch.empty((70000, *x.shape[1:]), dtype=x.dtype, device="cuda") for x in small))
    for a, b in zip(large, small):
        a[where] = b
    table = np.where(small_table >= 0, far[small_table], -1)
    q, k, v = _inputs(g, 2, 16, kv, n, D, "bf16")
    parents, lengths = _int(_parents(g, 2, n).tolist()), _int([400, 150])
    a, b = (F.seq_cache_tree_attention(q, k, v, parents, cache, _int(t.tolist()), lengths) for cache, t in ((small, small_table), (large, table)))
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_servers_steps(dtype):
    """Prompts rotated into the cache; then, three times, a drafted tree: rotated by depth, attended over the cache, verified, and its accepted path appended."""
    g = np.random.default_rng(9)
    B, heads, kv, D, page, n, V = 3, 8, 2, 64, 32, 12, 500
    prompts, longest = [40, 64, 7], 64
    table_np, pages = _table(g, [x + 3 * n for x in prompts], page)
    table, cache = _int(table_np.tolist()), F.SeqCache.empty(pages, kv, page, D)
    freqs = torch.tensor([10000.0 ** (-i / 32) for i in range(32)], dtype=torch.float32, device="cuda")
    qw, kw = (torch.from_numpy(g.uniform(0.5, 1.5, D).astype(np.float32)).to(TYPES[dtype]).cuda() for _ in range(2))
    k, v = (normal(g, (B, longest, kv, D), dtype).transpose(1, 2) for _ in range(2))
    F.seq_cache_append(cache, k, v, table, _int([0] * B), _int(prompts), freqs=freqs, weight=kw)
    # what the cache should hold: keys rotated at their places, values as they came; a list for each sequence
    turned = seq_oracle.rotary(f64(k), np.arange(longest)[None], f64(freqs), (32,), f64(kw))[0]["z"]
    held = [[turned[b, :, :x], f64(v[b, :, :x])] for b, x in enumerate(prompts)]
    lengths = list(prompts)
    for step in range(3):
        q, k, v = _inputs(g, B, heads, kv, n, D, dtype)
        parents = np.stack([[-1] + [int(g.integers(max(0, (i - 1) // 2 - 1), i)) for i in range(1, n)] for _ in range(B)]).astype(np.int32)
        depth = np.array([seq_oracle.depths(p) for p in parents.tolist()])
        positions = (np.array(lengths)[:, None] + depth)[:, None]
        qr, kr = F.seq_rotary(q, k, _int(positions.tolist()), freqs, q_weight=qw, k_weight=kw)
        out = F.seq_cache_tree_attention(qr, kr, v, _int(parents.tolist()), cache, table, _int(lengths))
        host = [x.cpu().numpy() for x in cache]
        _check(out, qr, kr, v, parents, host, table_np, lengths, dtype)
        logits = torch.from_numpy(g.standard_normal((B, n, V)).astype(np.float32) * 3).cuda()
        tokens = np.zeros((B, n), int)
        order = np.argsort(-f64(logits), axis=2)
        for b in range(B):
            for i in range(1, n):
                tokens[b, i] = order[b, parents[b, i], (parents[b, 1:i] == parents[b, i]).sum()]
        u = g.random((B, n)).astype(np.float32)
        path, counts, following = F.seq_verify(logits, _int(tokens.tolist()), torch.from_numpy(u).cuda(), parents=_int(parents.tolist()))
        F.seq_cache_append(cache, kr, v, table, _int(lengths), counts, rows=path)
        for b in range(B):
            want, token = seq_oracle.verify(f64(logits[b]), tokens[b], u[b].astype(np.float64), parents[b].tolist())
            assert path[b].tolist()[:len(want)] == want and int(counts[b]) == len(want) and int(following[b]) == token
            assert depth[b, want].tolist() == list(range(len(want)))   # accepted nodes stand where they are appended
            held[b] = [np.concatenate([held[b][0], f64(kr[b])[:, want]], 1), np.concatenate([held[b][1], f64(v[b])[:, want]], 1)]
            lengths[b] += len(want)
    got = F.seq_cache_gather(cache, table, _int(lengths), _int([0] * B), max(lengths), dtype=torch.float32)
    scales = [x.cpu().numpy() for x in cache[2:]]
    for x, i, s in zip(got, (0, 1), scales):
        for b, L in enumerate(lengths):
            step = s[table_np[b, np.arange(L) // page]].T[:, :, None]   # half of it, and half again each of three times that a page may have grown; keys' own error, 2^-18 of at most 2 * 5 * 1.5
            assert (np.abs(f64(x[b, :, :L]) - held[b][i]) <= 2.0 * step + 15 * 2.0 ** -18).all()
