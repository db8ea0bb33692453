// The cache in 8 bits: what its kernels take.
#pragma once

#include "seq_common.hpp"

namespace seq {

struct CacheArgs {
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
hipError_t launch_gather(const CacheArgs &a, int dtype, int D, hipStream_t st);
hipError_t launch_cache_attention(const CacheArgs &a, int dtype, int D, int cap, hipStream_t st);   // cap: the CapForm of fp16 weights, whatever the type of q
void plan_cache_attention(CacheArgs &a, int64_t longest);   // splits, row_groups
size_t cache_attention_bytes(const CacheArgs &a, int D);

}  // namespace seq
