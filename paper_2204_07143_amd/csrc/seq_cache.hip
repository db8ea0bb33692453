// The cache of keys and values in 8 bits, one scale for each page and head: append and gather.  Both are bound by memory (or, for a token at a
// time, by the launch): a workgroup per page, head and side appends, a thread per 16 bytes of output gathers.
#include "seq_cache.hpp"

namespace seq {

namespace {

constexpr float kMost = 3.402823466e38f;

template <typename T> __device__ __forceinline__ float finite(T x) {   // NaN: 0; infinite: the largest finite value
    const float f = (float)x;
    return f != f ? 0.f : fminf(fmaxf(f, -kMost), kMost);
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void append_kernel(const CacheArgs p, int touched) {
    constexpr int E = 16 / (int)sizeof(T), CH = D / E;   // elements of a chunk, chunks of a row
    typedef T vec __attribute__((ext_vector_type(E)));
    typedef int8_t bytes __attribute__((ext_vector_type(E)));
    __shared__ float most_of[kWaves];
    const int tid = threadIdx.x;
    int id = blockIdx.x;
    const bool values = id & 1;
    id >>= 1;
    const int kh = id % p.kv;
    id /= p.kv;
    const int b = id / touched, page = 1 << p.page_log2;
    const int64_t length = p.lengths[b];
    const int count = p.extra ? min(p.extra[b], p.n) : p.n;
    if (length < 0 || count <= 0) return;
    const int64_t at = (length >> p.page_log2) + id % touched, start = at << p.page_log2;
    const int64_t lo = length > start ? length : start, hi = length + count < start + page ? length + count : start + page;
    int to;
    if (lo >= hi || !page_at(p, b, start, to)) return;
    const int64_t unit = (int64_t)to * p.kv + kh;
    int8_t *cells = (values ? p.v : p.k) + unit * page * D;
    float *scales = values ? p.vs : p.ks;
    const View &x = values ? p.b : p.a;
    const char *rows = x.at + b * x.b + kh * x.h;
    const int old = (int)(lo - start), fresh = (int)(hi - lo), skip = (int)(lo - length);

    float most = 0.f;
    for (int i = tid; i < fresh * CH; i += kThreads) {
        const vec y = *reinterpret_cast<const vec *>(rows + (int64_t)(skip + i / CH) * x.row + i % CH * 16);
#pragma unroll
        for (int e = 0; e < E; ++e) most = fmaxf(most, fabsf(finite(y[e])));
    }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    if (tid % kWave == 0) most_of[tid / kWave] = most;
    const float before = old ? scales[unit] : 0.f;
    workgroup_sync();
    most = fmaxf(fmaxf(most_of[0], most_of[1]), fmaxf(most_of[2], most_of[3]));
    const float scale = fmaxf(before, most / 127.f), by = scale > 0.f ? scale : 1.f;
    if (tid == 0) scales[unit] = scale;
    if (old && scale != before) {
        const float ratio = before / by;
        uint32_t *words = reinterpret_cast<uint32_t *>(cells);
        for (int i = tid; i < old * D / 4; i += kThreads) {
            const uint32_t w = words[i];
            uint32_t r = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) r |= (uint32_t)(uint8_t)(int8_t)rintf((float)(int8_t)(w >> 8 * e) * ratio) << 8 * e;
            words[i] = r;
        }
    }
    for (int i = tid; i < fresh * CH; i += kThreads) {
        const vec y = *reinterpret_cast<const vec *>(rows + (int64_t)(skip + i / CH) * x.row + i % CH * 16);
        bytes r;
#pragma unroll
        for (int e = 0; e < E; ++e) r[e] = (int8_t)fminf(fmaxf(rintf(finite(y[e]) / by), -127.f), 127.f);
        *reinterpret_cast<bytes *>(cells + (int64_t)(old + i / CH) * D + i % CH * E) = r;
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void gather_kernel(const CacheArgs p, int64_t total) {
    constexpr int E = 16 / (int)sizeof(T), CH = D / E;
    typedef T vec __attribute__((ext_vector_type(E)));
    typedef float fvec __attribute__((ext_vector_type(E)));
    typedef int8_t bytes __attribute__((ext_vector_type(E)));
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= total) return;
    const int c = (int)(i % CH);
    const int64_t row = i / CH;
    const int at = (int)(row % p.n), plane = (int)(row / p.n), kh = plane % p.kv, b = plane / p.kv;
    const int64_t position = (int64_t)p.extra[b] + at;
    int id;
    vec k, v;
#pragma unroll
    for (int e = 0; e < E; ++e) k[e] = v[e] = (T)0.f;
    if (position >= 0 && position < p.lengths[b] && page_at(p, b, position, id)) {
        const int64_t unit = (int64_t)id * p.kv + kh, cell = ((unit << p.page_log2) + (position & ((1 << p.page_log2) - 1))) * D + c * E;
        const bytes x = *reinterpret_cast<const bytes *>(p.k + cell), y = *reinterpret_cast<const bytes *>(p.v + cell);
        k = __builtin_convertvector(__builtin_convertvector(x, fvec) * p.ks[unit], vec);
        v = __builtin_convertvector(__builtin_convertvector(y, fvec) * p.vs[unit], vec);
    }
    *reinterpret_cast<vec *>(const_cast<char *>(p.a.at) + b * p.a.b + kh * p.a.h + (int64_t)at * p.a.row + c * 16) = k;
    *reinterpret_cast<vec *>(const_cast<char *>(p.b.at) + b * p.b.b + kh * p.b.h + (int64_t)at * p.b.row + c * 16) = v;
}

template <typename T, int D, bool> struct Append {
    static hipError_t go(const CacheArgs &a, hipStream_t st) {
        const int page = 1 << a.page_log2, touched = (a.n + page - 2) / page + 1;   // pages that n tokens can lie in
        const int64_t blocks = (int64_t)a.B * touched * a.kv * 2;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        append_kernel<T, D><<<(unsigned)blocks, kThreads, 0, st>>>(a, touched);
        return hipGetLastError();
    }
};
template <typename T, int D, bool> struct Gather {
    static hipError_t go(const CacheArgs &a, hipStream_t st) {
        const int64_t total = (int64_t)a.B * a.kv * a.n * (D * (int)sizeof(T) / 16), blocks = (total + kThreads - 1) / kThreads;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        gather_kernel<T, D><<<(unsigned)blocks, kThreads, 0, st>>>(a, total);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_append(const CacheArgs &a, int dtype, int D, hipStream_t st) { return dispatch<Append>(dtype, D, false, a, st); }
hipError_t launch_gather(const CacheArgs &a, int dtype, int D, hipStream_t st) { return dispatch<Gather>(dtype, D, false, a, st); }

}  // namespace seq
