"""The cache in 8 bits (append, gather, attention over it), and all of it together, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import seq_oracle
from paper_2204_07143_amd import functional as F

from seq_util import FP32, HALF, TINY, TYPES, check, f64, normal

pytestmark = pytest.mark.gpu


def _table(g, lengths, page, spare=3, width=None):
    used = [-(-x // page) for x in lengths]
    pages = sum(used) + spare
    order = g.permutation(pages).astype(np.int32)
    table = np.full((len(lengths), max([1, *used]) if width is None else width), -9, np.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pages


def _cache(g, pages, kv, page, D):
    """A cache full of anything: numpy, and on the GPU."""
    host = [g.integers(-127, 128, (pages, kv, page, D)).astype(np.int8) for _ in range(2)] + [g.uniform(0.01, 0.03, (pages, kv)).astype(np.float32) for _ in range(2)]
    return host, F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _same(cache, host):
    for got, want in zip(cache, host):
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page,D", [(16, 32), (32, 64), (64, 128), (128, 128), (16, 128)])
@pytest.mark.parametrize("n", [1, 5, 150])
def test_append(dtype, page, D, n):
    g = np.random.default_rng(page + n)
    lengths = [0, 1, page - 1, page, 3 * page + 2, 77]
    counts = [n, max(0, n - 1), n, 0, n // 2, n]
    table, pages = _table(g, [x + n for x in lengths], page)
    host, cache = _cache(g, pages, 2, page, D)
    k, v = (normal(g, (6, 2, n, D), dtype, std) for std in (1.0, 4.0))
    k[:, :, -1] *= 3   # a page's scale grows within the call
    for c in (None, counts):
        F.seq_cache_append(cache, k, v, _int(table.tolist()), _int(lengths), None if c is None else _int(c))
        for i, x in ((0, k), (1, v)):
            host[i], host[i + 2] = seq_oracle.append(host[i], host[i + 2], x.float().cpu().numpy(), table, lengths, c)
        _same(cache, host)


def test_append_by_tokens_stays_within_its_roundings():
    """A page filled a token at a time: at most half a step of the scale at the time for each time that it grew, the first rounding included."""
    g = np.random.default_rng(1)
    x = normal(g, (1, 1, 64, 32), "f32") * torch.linspace(0.1, 3.0, 64, device="cuda")[:, None]
    cache, table = F.SeqCache.empty(1, 1, 64, 32), _int([[0]])
    off = torch.zeros(64, device="cuda")
    for t in range(64):
        before = float(cache.k_scales[0, 0])
        F.seq_cache_append(cache, x[:, :, t:t + 1], x[:, :, t:t + 1], table, _int([t]))
        now = float(cache.k_scales[0, 0])
        off[:t + 1] += now / 2 if now != before else 0
        off[t] = now / 2
    k, v = F.seq_cache_gather(cache, table, _int([64]), _int([0]), 64, dtype=torch.float32)
    assert torch.equal(k, v) and ((k - x)[0, 0].abs().amax(1) <= off * (1 + 1e-5)).all()


def test_append_values_that_are_not_ordinary():
    nan, inf = float("nan"), float("inf")
    cache = F.SeqCache.empty(4, 1, 16, 32)
    x = torch.zeros((4, 1, 2, 32), device="cuda")
    x[0, 0, 0, :4] = torch.tensor([nan, 1.0, -2.0, 0.5])
    x[1, 0, 1, :3] = torch.tensor([inf, -inf, 1.0])
    x[3, 0, 0, 0] = 1e-44   # its scale is no number above 0
    F.seq_cache_append(cache, x, x, _int([[0], [1], [2], [3]]), _int([0, 0, 0, 0]))
    k, _ = F.seq_cache_gather(cache, _int([[0], [1], [2], [3]]), _int([2] * 4), _int([0] * 4), 2, dtype=torch.float32)
    assert k[0, 0, 0, 0] == 0 and abs(float(k[0, 0, 0, 2]) + 2) < 1e-6
    assert k[1, 0, 1, 0] > 3.4e38 and k[1, 0, 1, 1] < -3.4e38 and k[1, 0, 1, 2] == 0
    assert (k[2] == 0).all() and torch.isfinite(k[3]).all() and k[3].abs().max() < 1e-42


def test_pages_that_are_none_are_passed_over():
    g = np.random.default_rng(2)
    table = np.array([[1, 50, 0, -1], [2, 3, 4, 6]], np.int32)
    host, cache = _cache(g, 6, 2, 16, 64)
    x = normal(g, (2, 2, 70, 64), "f16")
    F.seq_cache_append(cache, x, x, _int(table.tolist()), _int([0, 0]))   # 64 positions each at most: the rest has no page either
    for i in (0, 1):
        host[i], host[i + 2] = seq_oracle.append(host[i], host[i + 2], x.float().cpu().numpy(), table, [0, 0])
    _same(cache, host)
    k, v = F.seq_cache_gather(cache, _int(table.tolist()), _int([70, 70]), _int([0, 0]), 70, dtype=torch.float16)
    for got, i in ((k, 0), (v, 1)):
        want = seq_oracle.gather(host[i], host[i + 2], table, [70, 70], [0, 0], 70)
        check("gather", got, want, np.abs(want) * HALF["f16"] * 1.01)
    q = normal(g, (2, 4, 1, 64), "f16")
    got = F.seq_cache_attention(q, cache, _int(table.tolist()), _int([60, 60]))
    _check_attention(got, q, host, table, [60, 60], "f16")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page,D", [(16, 64), (64, 32), (128, 128)])
def test_gather(dtype, page, D):
    g = np.random.default_rng(3)
    lengths, first = [0, 5, 200, 131, 64], [0, -3, 150, 131, 63]
    table, pages = _table(g, lengths, page)
    host, cache = _cache(g, pages, 3, page, D)
    got = F.seq_cache_gather(cache, _int(table.tolist()), _int(lengths), _int(first), 67, dtype=TYPES[dtype])
    for x, i in zip(got, (0, 1)):
        want = seq_oracle.gather(host[i], host[i + 2], table, lengths, first, 67)
        check("gather", x, want, np.abs(want) * HALF[dtype] * (2 if dtype != "f32" else 1.01))   # 16 bit: rounded to fp32, then to the type


def _check_attention(got, q, host, table, lengths, dtype, window=None, softcap=None, slopes=None, scale=None):
    """Weights are rounded to fp16, q to fp16 on a scale of its row (2^-24 of its largest element at worst, so 2^-24 D of a score's scale), the result to its type."""
    B, heads, n, D = q.shape
    pages, kv, page, _ = host[0].shape
    for b, L in enumerate(lengths):
        if L == 0:
            assert (got[b] == 0).all()
            continue
        at = slice(max(0, n - L), n)   # a query that stands before the sequence sees nothing
        assert (got[b, :, :max(0, n - L)] == 0).all()
        k, v = (seq_oracle.gather(host[i], host[i + 2], table[b:b + 1], [L], [0], L) for i in (0, 1))
        documents = np.where(seq_oracle.present(pages, page, table[b], L), 0, -1)[None]
        qq = f64(q[b:b + 1, :, at])
        mine = documents.copy()
        mine[:, L - qq.shape[2]:] = 0   # (a query is there even where its own token's page is none)
        res, bound = _attend(qq, k, v, documents, mine, window, softcap, slopes, scale)
        u = HALF[dtype]
        check(f"sequence {b}", got[b:b + 1, :, at], res, bound + u * np.abs(res))


def _attend(q, k, v, documents, mine, window, softcap, slopes, scale):
    outs, bounds = [], []
    B, heads, n, D = q.shape
    L, group = k.shape[2], heads // k.shape[1]
    see = seq_oracle.visible(n, L, True, window) & (documents[0] >= 0)[None]
    for h in range(heads):
        r, o = seq_oracle.head(q[0, h], k[0, h // group], v[0, h // group], None, see, scale=D ** -0.5 if scale is None else scale, softcap=softcap,
                               slope=0.0 if slopes is None else float(slopes[h]), u=HALF["f16"], e=FP32, tiny=TINY["f16"])
        outs.append(r["out"])
        bounds.append(o["out"])
    return np.stack(outs)[None], np.stack(bounds)[None]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("page,D", [(16, 32), (16, 64), (16, 128), (32, 128), (64, 64), (128, 32), (64, 128)])
@pytest.mark.parametrize("cap", [None, 5.0])
def test_attention_of_one_token(dtype, page, D, cap):
    g = np.random.default_rng(D + page)
    lengths = [1, 0, page, 31, 32, 33, 500, 129]
    table, pages = _table(g, lengths, page)
    host, cache = _cache(g, pages, 2, page, D)
    q = normal(g, (len(lengths), 8, 1, D), dtype)
    got = F.seq_cache_attention(q, cache, _int(table.tolist()), _int(lengths), softcap=cap)
    _check_attention(got, q, host, table, lengths, dtype, softcap=cap)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (16, 1), (40, 2), (7, 7), (64, 1)])
@pytest.mark.parametrize("n", [1, 2, 7, 40])
def test_attention_rows(heads, kv, n):
    g = np.random.default_rng(heads + n)
    lengths = [n, 150, 300, max(0, n - 2)]
    table, pages = _table(g, lengths, 32)
    host, cache = _cache(g, pages, kv, 32, 64)
    q = normal(g, (4, n, heads, 64), "bf16").transpose(1, 2)
    slopes = torch.from_numpy(g.uniform(0, 0.2, heads).astype(np.float32)).cuda()
    got = F.seq_cache_attention(q, cache, _int(table.tolist()), _int(lengths), slopes=slopes, scale=0.05)
    _check_attention(got, q, host, table, lengths, "bf16", slopes=f64(slopes), scale=0.05)


@pytest.mark.parametrize("window", [1, 5, 64, 1000, 100000])
@pytest.mark.parametrize("page,n", [(16, 1), (64, 4)])
def test_attention_windows_and_long_ranges(window, page, n):
    """One long sequence and a short one: ranges are split over workgroups, some of which have nothing to do."""
    g = np.random.default_rng(window)
    lengths = [6001, 40]
    table, pages = _table(g, lengths, page)
    host, cache = _cache(g, pages, 1, page, 64)
    q = normal(g, (2, 2, n, 64), "f16", 3.0)
    got = F.seq_cache_attention(q, cache, _int(table.tolist()), _int(lengths), window=window)
    # scores reach 3 * 127 * 0.03 * 8 = 90, and a sum has 6000 terms: four times what the bound's share of fp32 is made for, below fp16's 2^-11
    _check_attention(got, q, host, table, lengths, "f16", window=window)


@pytest.mark.parametrize("std", [1e-4, 1e4])
def test_queries_of_any_size(std):
    g = np.random.default_rng(4)
    table, pages = _table(g, [90, 90], 16)
    host, cache = _cache(g, pages, 1, 16, 32)
    for dtype in ("f16", "bf16"):
        q = normal(g, (2, 4, 1, 32), dtype, std)
        got = F.seq_cache_attention(q, cache, _int(table.tolist()), _int([90, 90]), scale=0.2 / std)
        _check_attention(got, q, host, table, [90, 90], dtype, scale=0.2 / std)


def test_scales_far_apart_and_shared_pages():
    g = np.random.default_rng(5)
    table = np.array([[0, 1, 2, 3], [0, 1, 4, 4]], np.int32)   # a prefix that two sequences share, and a page twice
    for page in (16, 64):
        host, _ = _cache(g, 5, 2, page, 64)
        host[3][:, 0] = [1e-6, 1e3, 1.0, 0.0, 1e-3]
        cache = F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
        q = normal(g, (2, 4, 1, 64), "bf16", 4.0)
        got = F.seq_cache_attention(q, cache, _int(table.tolist()), _int([4 * page, 4 * page - 3]))
        _check_attention(got, q, host, table, [4 * page, 4 * page - 3], "bf16")


def test_same_bits_again_and_replayed():
    g = np.random.default_rng(6)
    table, pages = _table(g, [3000, 17], 16)
    _, cache = _cache(g, pages, 2, 16, 128)
    table, lengths = _int(table.tolist()), _int([2990, 10])
    q, k, v = (normal(g, (2, h, 1, 128), "bf16") for h in (8, 2, 2))

    def run():
        F.seq_cache_append(cache, k, v, table, lengths)
        return F.seq_cache_attention(q, cache, table, lengths + 1)
    eager = run().clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        again = run()
    stream.synchronize()
    assert torch.equal(eager, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for _ in range(3):
        out.fill_(float("nan"))
        run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_prompt_a_second_chunk_and_tokens(dtype):
    """As a server uses them: a prompt attended and cached, its next chunk attended over what is read back, then tokens one by one."""
    g = np.random.default_rng(7)
    B, heads, kv, D, page, cap = 3, 8, 2, 64, 32, 20.0
    first, chunk, steps = [100, 64, 7], 50, 3
    total = [x + chunk + steps for x in first]
    table_np, pages = _table(g, total, page)
    table, cache = _int(table_np.tolist()), F.SeqCache.empty(pages, kv, page, D)
    host = [np.zeros((pages, kv, page, D), np.int8), np.zeros((pages, kv, page, D), np.int8), np.zeros((pages, kv), np.float32), np.zeros((pages, kv), np.float32)]

    def both(k, v, lengths, counts=None):
        F.seq_cache_append(cache, k, v, table, _int(lengths), None if counts is None else _int(counts))
        for i, x in ((0, k), (1, v)):
            host[i], host[i + 2] = seq_oracle.append(host[i], host[i + 2], x.float().cpu().numpy(), table_np, lengths, counts)
        _same(cache, host)
    longest = max(first)
    k, v = (normal(g, (B, longest, kv, D), dtype).transpose(1, 2) for _ in range(2))
    both(k, v, [0] * B, first)
    lengths = first
    # the chunk: read back so that every sequence ends at the last position, what lies before its beginning being padding
    k, v = (normal(g, (B, chunk, kv, D), dtype).transpose(1, 2) for _ in range(2))
    both(k, v, lengths)
    lengths = [x + chunk for x in lengths]
    reach = max(lengths)
    kk, vv = F.seq_cache_gather(cache, table, _int(lengths), _int([x - reach for x in lengths]), reach, dtype=TYPES[dtype])
    documents = torch.tensor([[-1] * (reach - x) + [0] * x for x in lengths], dtype=torch.int32, device="cuda")
    q = normal(g, (B, chunk, heads, D), dtype).transpose(1, 2)
    dense = F.seq_attention(q, kk, vv, causal=True, softcap=cap, documents=documents)
    paged = F.seq_cache_attention(q, cache, table, _int(lengths), softcap=cap)
    _check_attention(paged, q, host, table_np, lengths, dtype, softcap=cap)
    # the values read back are rounded to the type; a weight is off by the scores' share of that, sum |q| |k| scale of them at most
    a, b = f64(dense), f64(paged)
    assert np.abs(a - b).max() <= 16 * HALF[dtype] * np.abs(b).max()
    for _ in range(steps):
        k, v = (normal(g, (B, kv, 1, D), dtype) for _ in range(2))
        both(k, v, lengths)
        lengths = [x + 1 for x in lengths]
        q = normal(g, (B, heads, 1, D), dtype)
        got = F.seq_cache_attention(q, cache, table, _int(lengths), softcap=cap)
        _check_attention(got, q, host, table_np, lengths, dtype, softcap=cap)


def test_rows_behind_the_counts_are_left_as_they_are():
    g = np.random.default_rng(8)
    host, cache = _cache(g, 4, 1, 16, 32)
    x = normal(g, (2, 1, 9, 32), "f32")
    F.seq_cache_append(cache, x, x, _int([[0, 1], [2, 3]]), _int([3, -1]), _int([4, 9]))
    assert np.array_equal(cache.k_pages[1:].cpu().numpy(), host[0][1:]) and np.array_equal(cache.k_pages[0, :, 7:].cpu().numpy(), host[0][0, :, 7:])


def test_pages_behind_32_bits():
    """Cells whose offsets pass 2^32 bytes: the same as in a small cache."""
    g = np.random.default_rng(9)
    kv, page, D, n = 8, 64, 128, 150
    small_table, pages = _table(g, [400, 7 + n], page, spare=0)
    _, small = _cache(g, pages, kv, page, D)
    far = 70000 - 1 - 3 * np.arange(pages)   # of 64 KiB each, from 2^32 bytes on
    assert far.min() * kv * page * D > 1 << 32
    where = torch.from_numpy(far).cuda()
    large = F.SeqCache(*(torch.empty((70000, *x.shape[1:]), dtype=x.dtype, device="cuda") for x in small))
    for a, b in zip(large, small):
        a[where] = b
    table = np.where(small_table >= 0, far[small_table], -1)
    tables, lengths = [_int(x.tolist()) for x in (small_table, table)], _int([400 - n, 7])
    k, v = (normal(g, (2, kv, n, D), "bf16") for _ in range(2))
    q = normal(g, (2, 16, 3, D), "bf16")
    results = []
    for cache, t in zip((small, large), tables):
        F.seq_cache_append(cache, k, v, t, lengths)
        results.append((*F.seq_cache_gather(cache, t, lengths + n, _int([0, -5]), 400), F.seq_cache_attention(q, cache, t, lengths + n)))
    for a, b in zip(large, small):
        assert torch.equal(a[where], b)
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_counts_and_lengths_out_of_range():
    """Counts above n are n; of negative counts and lengths nothing is stored or seen; what lies past the table has no page."""
    g = np.random.default_rng(10)
    big = 2 ** 31 - 1
    table = np.array([[0, 1], [2, 3], [4, 5], [6, 7]], np.int32)
    host, cache = _cache(g, 8, 2, 16, 32)
    x = normal(g, (4, 2, 9, 32), "f16")
    F.seq_cache_append(cache, x, x, _int(table.tolist()), _int([0, -5, big, 4]), _int([big, 9, 9, -big - 1]))
    for i in (0, 1):
        host[i], host[i + 2] = seq_oracle.append(host[i], host[i + 2], x.float().cpu().numpy()[:1], table[:1], [0])
    _same(cache, host)
    k, _ = F.seq_cache_gather(cache, _int(table.tolist()), _int([9, -5, big, 32]), _int([big - 3, -big - 1, 28, 28]), 9, dtype=torch.float32)
    want = seq_oracle.gather(host[0], host[2], table, [9, 0, 32, 32], [40, 0, 28, 28], 9)
    assert np.abs(k.cpu().numpy() - want).max() <= 2 * FP32 * np.abs(want).max()
    q = normal(g, (4, 4, 2, 32), "f16")
    got = F.seq_cache_attention(q, cache, _int(table.tolist()), _int([9, -5, -big - 1, 0]))
    _check_attention(got[:1], q[:1], host, table[:1], [9], "f16")
    assert (got[1:] == 0).all()


@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("n,window", [(1, None), (5, None), (1, 5), (3, 20)])   # four heads share a key head: one block of rows, and two
def test_entries_that_no_query_reaches_may_name_pages_never_written(page, n, window):
    g = np.random.default_rng(11)
    lengths = [10, 33, 48, 7, 100, 5 * page + 1, 1000]
    table, pages = _table(g, lengths, page, spare=1, width=-(-1000 // page) + 3)
    never, = set(range(pages)) - set(table.ravel().tolist())
    host, _ = _cache(g, pages, 2, page, 64)
    q = normal(g, (len(lengths), 8, n, 64), "f16")
    dead = np.ones_like(table, dtype=bool)   # entries all of whose positions lie behind the sequence, or before every query's window
    for b, L in enumerate(lengths):
        first = max(0, L - n - (window or L + n) + 1)
        dead[b, first // page:(L - 1) // page + 1] = False
    results = []
    for entry, scale in ((-1, 0.02), (never, float("nan")), (never, float("inf"))):
        host[2][never] = host[3][never] = scale
        cache = F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
        results.append(F.seq_cache_attention(q, cache, _int(np.where(dead, entry, table).tolist()), _int(lengths), window=window))
    assert torch.isfinite(results[0]).all()
    for x in results[1:]:
        assert torch.equal(x, results[0])


def test_queries_up_to_the_types_largest():
    g = np.random.default_rng(12)
    table, pages = _table(g, [90, 90], 32)
    host, _ = _cache(g, pages, 1, 32, 32)
    host[2] /= 8   # (scores of a few units)
    cache = F.SeqCache(*(torch.from_numpy(x).cuda() for x in host))
    q = torch.from_numpy(g.uniform(-3.3e38, 3.3e38, (2, 4, 1, 32)).astype(np.float32)).to(torch.bfloat16).cuda()
    assert (q.abs().amax(-1) >= 2.0 ** 127).all()
    got = F.seq_cache_attention(q, cache, _int(table.tolist()), _int([90, 90]), scale=2e-38)
    _check_attention(got, q, host, table, [90, 90], "bf16", scale=float(np.float32(2e-38)))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("page,D", [(16, 32), (64, 64), (16, 128), (128, 128)])
@pytest.mark.parametrize("cap", [1025.0, 4096.0])
@pytest.mark.parametrize("n", [1, 6])
def test_large_caps(dtype, page, D, cap, n):
    """Beyond a cap of 1024 scores are off by no more than without one."""
    g = np.random.default_rng(13)
    lengths = [n, 33, 500, 129]
    table, pages = _table(g, lengths, page)
    host, cache = _cache(g, pages, 2, page, D)
    q = normal(g, (len(lengths), 8, n, D), dtype, 3.0)
    got = F.seq_cache_attention(q, cache, _int(table.tolist()), _int(lengths), softcap=cap)
    _check_attention(got, q, host, table, lengths, dtype, softcap=cap)
