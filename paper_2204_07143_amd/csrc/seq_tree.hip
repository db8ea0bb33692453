// Attention of a tree of drafted tokens over a cache in 8 bits: rows as in seq_decode.hpp, their last part being the nodes' own keys and values.
#include "seq_decode.hpp"

namespace seq {

namespace {

template <typename T, int D, int CAP> struct TreeAttention {
    static hipError_t go(const CacheArgs &a, hipStream_t st) {
        const int64_t blocks = (int64_t)a.B * a.kv * a.row_groups * a.splits;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        const bool wide = rows_each(a) > 16, page16 = a.page_log2 == 4;
        auto *kernel = wide ? page16 ? decode_kernel<T, D, 2, CAP, true, true> : decode_kernel<T, D, 2, CAP, false, true>
                            : page16 ? decode_kernel<T, D, 1, CAP, true, true> : decode_kernel<T, D, 1, CAP, false, true>;
        kernel<<<(unsigned)blocks, kThreads, 0, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        const int64_t rows = (int64_t)a.B * a.heads * a.n;
        if (!launch_holds(rows, kThreads)) return hipErrorInvalidValue;
        join_kernel<T, D><<<(unsigned)rows, kThreads, 0, st>>>(a, rows_each(a));
        return hipGetLastError();
    }
};

}  // namespace

void plan_cache_tree(CacheArgs &a, int64_t longest, int D) {
    // More than 32 rows to a key head go in tiles of 64 tokens (seq_tree_tile.hip), which look at the cache once for up to 192 rows but take 20 us before the first tile, where these
    // take 12, if there is enough work: 81 rows, bf16, D 128, us here / in tiles: 20 sequences and key heads with a window of 2048 (640 tiles) 21 / 33; 192 rows, 128
    // sequences and key heads to 8000 tokens (9000 tiles) 225 / 127.
    const int64_t rows = (int64_t)a.group * a.n, reach = longest < (int64_t)a.window ? longest : (int64_t)a.window, tiles = (int64_t)a.B * a.kv * ((reach + kTile - 1) / kTile);
    a.tiled = rows > 32 && (double)tiles * rows >= 65536;
    if (a.tiled) return plan_tree_tiles(a, longest, D);
    // There is a join in any case: parts of 128 tokens, where workgroups are few (fewer than the 256 compute units: 5 sequences, 12 heads over 4, 27 nodes, window 2048, capped, 17 + 4 us, up to 512
    // workgroups 21 + 4).
    plan_cache_attention(a, longest);
    const int64_t units = (int64_t)a.B * a.kv * a.row_groups, wanted = (256 + units - 1) / units, most = reach / 128;
    const int64_t s = wanted < most ? wanted : most;
    a.splits = (int)(s > 128 ? 128 : s > a.splits ? s : a.splits) + 1;   // and the nodes' own part
}
size_t cache_tree_bytes(const CacheArgs &a, int D) {
    if (a.tiled) return tree_tile_bytes(a, D);
    return (size_t)a.B * a.kv * a.row_groups * a.splits * rows_each(a) * (D + 2) * sizeof(float);
}

hipError_t launch_cache_tree(const CacheArgs &a, int dtype, int D, int cap, hipStream_t st) {
    if (a.tiled) return launch_tree_tiles(a, dtype, D, cap, st);
#define SEQ_D(T, N) (cap == kNoCap ? TreeAttention<T, N, kNoCap>::go(a, st) : cap == kSigmoidCap ? TreeAttention<T, N, kSigmoidCap>::go(a, st) : TreeAttention<T, N, kTanhCap>::go(a, st))
#define SEQ_T(T) (D == 32 ? SEQ_D(T, 32) : D == 64 ? SEQ_D(T, 64) : SEQ_D(T, 128))
    return dtype == NA2D_F16 ? SEQ_T(f16_t) : SEQ_T(bf16_t);
#undef SEQ_T
#undef SEQ_D
}

}  // namespace seq
