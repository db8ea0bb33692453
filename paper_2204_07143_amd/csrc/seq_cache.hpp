// The cache in 8 bits: what its kernels take.
#pragma once

#include "seq_rotary.hpp"

namespace seq {

struct CacheArgs {
    View tk, tv;           // a tree of nodes: their own keys and values,
    const int *parents;    // [B, n]
    bool tanh, tiled;      // scores are capped by the library's tanh; in tiles (seq_tree_tile.hip)
    View a, b;             // append: new keys and values; gather: keys and values read; attention: q and out
    int8_t *k, *v;
    float *ks, *vs;
    const int *table, *lengths, *extra;   // extra: counts (append, or null), first (gather)
    const float *slopes;
    float *part;           // attention over split ranges: per (sequence, key head, row group, split) the rows' sums, then maxima and totals
    int B, heads, kv, group, page_log2, pages, width, n, window, splits, row_groups;
    float c, cap;
};

__device__ __forceinline__ bool page_at(const CacheArgs &p, int b, int64_t position, int &id) {
    const int64_t at = position >> p.page_log2;
    if (at >= p.width) return false;
    id = p.table[(int64_t)b * p.width + at];
    return (unsigned)id < (unsigned)p.pages;
}

hipError_t launch_append(const CacheArgs &a, int dtype, int D, hipStream_t st);
// Of `given` rows of each sequence the n that `rows` names (null: the first n), keys normed and rotated where `r` says so.
struct RowsArgs {
    CacheArgs c;
    Rotation r;            // positions of the given rows; null: a token's place in its sequence
    const int *rows;       // [B, n]
    int given;
};
hipError_t launch_append_rows(const RowsArgs &a, int dtype, int D, hipStream_t st);
hipError_t launch_gather(const CacheArgs &a, int dtype, int D, hipStream_t st);
hipError_t launch_cache_attention(const CacheArgs &a, int dtype, int D, int cap, hipStream_t st);   // cap: the CapForm of fp16 weights, whatever the type of q
hipError_t launch_cache_tree(const CacheArgs &a, int dtype, int D, int cap, hipStream_t st);
void plan_cache_tree(CacheArgs &a, int64_t longest, int D);
size_t cache_tree_bytes(const CacheArgs &a, int D);
// the same where a key head has many rows (seq_tree_tile.hip)
int tree_row_blocks(const CacheArgs &a, int D);
void plan_tree_tiles(CacheArgs &a, int64_t longest, int D);
size_t tree_tile_bytes(const CacheArgs &a, int D);
hipError_t launch_tree_tiles(const CacheArgs &a, int dtype, int D, int cap, hipStream_t st);
void plan_cache_attention(CacheArgs &a, int64_t longest);   // splits, row_groups
size_t cache_attention_bytes(const CacheArgs &a, int D);

}  // namespace seq
