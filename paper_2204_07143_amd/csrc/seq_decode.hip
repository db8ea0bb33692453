// Attention of a few new tokens over a cache in 8 bits: the launches of seq_decode.hpp's kernels.
#include "seq_decode.hpp"

namespace seq {

namespace {

template <typename T, int D, int CAP> struct Decode {
    static hipError_t go(const CacheArgs &a, hipStream_t st) {
        const int64_t blocks = (int64_t)a.B * a.kv * a.row_groups * a.splits;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        const bool wide = rows_each(a) > 16, page16 = a.page_log2 == 4;
        auto *kernel = wide ? page16 ? decode_kernel<T, D, 2, CAP, true, false> : decode_kernel<T, D, 2, CAP, false, false> : page16 ? decode_kernel<T, D, 1, CAP, true, false> : decode_kernel<T, D, 1, CAP, false, false>;
        kernel<<<(unsigned)blocks, kThreads, 0, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess || a.splits == 1) return e;
        const int64_t rows = (int64_t)a.B * a.heads * a.n;
        if (!launch_holds(rows, kThreads)) return hipErrorInvalidValue;
        join_kernel<T, D><<<(unsigned)rows, kThreads, 0, st>>>(a, rows_each(a));
        return hipGetLastError();
    }
};

}  // namespace

// Ranges are split until there are about sixteen workgroups to each of the 256 compute units (sequences differ in length), but no split is given less than 256
// tokens of the longest sequence that the table can hold (the lengths are on the GPU), or 512 where a workgroup leaves 32 rows; a table far wider than the sequences costs workgroups
// that have nothing to do: 16 sequences of 500 tokens, 32 heads over 8, table of 32 pages of 16 9.5 us, of 8192 pages 36.  us, 64 sequences of 9000 tokens, 8 x 128, for 1024, 2048 and
// 4096 workgroups 260, 251, 243; one of 16000 tokens in 256s and 512s 23 and 22; 4 of 8000, 32 rows, 36 and 28.
void plan_cache_attention(CacheArgs &a, int64_t longest) {
    a.row_groups = (a.group * a.n + rows_each(a) - 1) / rows_each(a);
    const int64_t reach = longest < (int64_t)a.window + a.n ? longest : (int64_t)a.window + a.n;
    const int64_t units = (int64_t)a.B * a.kv * a.row_groups, wanted = (4096 + units - 1) / units, most = reach / (rows_each(a) > 16 ? 512 : 256);
    const int64_t s = wanted < most ? wanted : most;
    a.splits = (int)(s < 1 ? 1 : s > 128 ? 128 : s);
}
size_t cache_attention_bytes(const CacheArgs &a, int D) {
    return a.splits == 1 ? 0 : (size_t)a.B * a.kv * a.row_groups * a.splits * rows_each(a) * (D + 2) * sizeof(float);
}

hipError_t launch_cache_attention(const CacheArgs &a, int dtype, int D, int cap, hipStream_t st) {
#define SEQ_D(T, N) (cap == kNoCap ? Decode<T, N, kNoCap>::go(a, st) : cap == kSigmoidCap ? Decode<T, N, kSigmoidCap>::go(a, st) : Decode<T, N, kTanhCap>::go(a, st))
#define SEQ_T(T) (D == 32 ? SEQ_D(T, 32) : D == 64 ? SEQ_D(T, 64) : SEQ_D(T, 128))
    return dtype == NA2D_F16 ? SEQ_T(f16_t) : SEQ_T(bf16_t);
#undef SEQ_T
#undef SEQ_D
}

}  // namespace seq
