// The cache of keys and values in 8 bits, one scale for each page and head: append and gather.  Both are bound by memory (or, for a token at a
// time, by the launch): a workgroup per page, head and side appends, a thread per 16 bytes of output gathers.  8 prompts of 1000 tokens, 8 heads, D 128, bf16: 16 us
// (49 MB, 13.5 in a run of appends alone: length, table, rows and scale are reads that wait for each other; tokens kept in registers between a page's maximum and its rounding 16 too), read back 11; 4 sequences of 8192
// positions, 8 heads, D 128, fp16, read back in 27 us (181 MB: 6.6 TB/s, a part of it in the last-level cache); a token of 64 sequences 4.
#include "seq_cache.hpp"

namespace seq {

namespace {

constexpr float kMost = 3.402823466e38f;

__device__ __forceinline__ float finite(float x) { return x != x ? 0.f : fminf(fmaxf(x, -kMost), kMost); }

// The largest magnitude of 16 bytes, as bits: at or above those of infinity if one is not finite.
template <typename T> __device__ __forceinline__ uint32_t most_of(u32x4 x) {
    uint32_t m = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) m = max(m, x[e] & 0x7fffffffu);
    } else {
        typedef uint16_t h2 __attribute__((ext_vector_type(2)));
        h2 y = __builtin_bit_cast(h2, x[0] & 0x7fff7fffu);
#pragma unroll
        for (int e = 1; e < 4; ++e) y = __builtin_elementwise_max(y, __builtin_bit_cast(h2, x[e] & 0x7fff7fffu));
        m = max((uint32_t)y[0], (uint32_t)y[1]);
    }
    return m;
}
template <typename T> __device__ __forceinline__ float from_bits(uint32_t m) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(m);
    else return (float)__builtin_bit_cast(T, (uint16_t)m);
}

// x / by to the nearest whole number, even ones from the middle, within -127 .. 127: x `over` (1 / by) is off by less than 2^-15 there, so the division is
// needed only next to a middle.  A NaN gives 0.
__device__ __forceinline__ int whole(float x, float by, float over) {
    float r = x * over;
    if (__builtin_expect(fabsf(fabsf(r - __builtin_rintf(r)) - 0.5f) < 0x1p-14f, 0)) r = x / by;
    return max(-127, min(127, (int)__builtin_rintf(r)));
}

// What a page held, in words of four bytes, on its new scale; of one below zero with the other sign (and -128 as 127).
__device__ __forceinline__ void round_again(int8_t *cells, int count, float ratio, int tid) {
    uint32_t *words = reinterpret_cast<uint32_t *>(cells);
    for (int i = tid; i < count; i += kThreads) {
        const uint32_t w = words[i];
        uint32_t r = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) r |= (uint32_t)(uint8_t)(int8_t)__builtin_rintf(fminf((float)(int8_t)(w >> 8 * e) * ratio, 127.f)) << 8 * e;
        words[i] = r;
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void append_kernel(const CacheArgs p, int touched) {
    constexpr int E = 16 / (int)sizeof(T), CH = D / E;   // elements of a chunk, chunks of a row
    typedef T vec __attribute__((ext_vector_type(E)));
    typedef int8_t bytes __attribute__((ext_vector_type(E)));
    __shared__ uint32_t mosts[kWaves];
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
    const int old = (int)(lo - start), fresh = (int)(hi - lo);
    const char *rows = x.at + b * x.b + kh * x.h + (lo - length) * x.row;

    uint32_t bits = 0;
#pragma unroll 4
    for (int i = tid; i < fresh * CH; i += kThreads) bits = max(bits, most_of<T>(*reinterpret_cast<const u32x4 *>(rows + (int64_t)(i / CH) * x.row + i % CH * 16)));
    const float before = old ? scales[unit] : 0.f;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) bits = max(bits, (uint32_t)__shfl_xor((int)bits, d));
    if (tid % kWave == 0) mosts[tid / kWave] = bits;
    workgroup_sync();
    float most = from_bits<T>(max(max(mosts[0], mosts[1]), max(mosts[2], mosts[3])));
    const bool ordinary = most < INFINITY;   // (the bits of a NaN are larger)
    if (!ordinary) {   // once more, without what is no number
        most = 0.f;
        for (int i = tid; i < fresh * CH; i += kThreads) {
            const vec y = *reinterpret_cast<const vec *>(rows + (int64_t)(i / CH) * x.row + i % CH * 16);
#pragma unroll
            for (int e = 0; e < E; ++e) most = fmaxf(most, fabsf(finite((float)y[e])));
        }
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        workgroup_sync();
        if (tid % kWave == 0) mosts[tid / kWave] = __float_as_uint(most);
        workgroup_sync();
        most = __uint_as_float(max(max(mosts[0], mosts[1]), max(mosts[2], mosts[3])));
    }
    const float scale = fmaxf(fabsf(before), most / 127.f), by = scale > 0.f ? scale : 1.f;
    if (tid == 0) scales[unit] = scale;
    if (old && scale != before) round_again(cells, old * D / 4, before / by, tid);
    // every element is divided where 1 / by may be no ordinary number either
    const bool divide = !ordinary || !(by > 0x1p-100f && by < 0x1p100f);
    const float over = 1.f / by;
#pragma unroll 2
    for (int i = tid; i < fresh * CH; i += kThreads) {
        const vec y = *reinterpret_cast<const vec *>(rows + (int64_t)(i / CH) * x.row + i % CH * 16);
        bytes r;
        if (divide) {
#pragma unroll
            for (int e = 0; e < E; ++e) r[e] = (int8_t)max(-127, min(127, (int)__builtin_rintf(finite((float)y[e]) / by)));
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) r[e] = (int8_t)whole((float)y[e], by, over);
        }
        *reinterpret_cast<bytes *>(cells + (int64_t)(old + i / CH) * D + i % CH * E) = r;
    }
}

// x / by to whole numbers, nearest even, as bytes, where |x / by| is at most 127 and a little: x over (1 / by) is off by less than 2^-17 there, and behind 1.5 2^23 it is rounded in
// place, the byte at the bottom.  Where an element of the wave lies next to a middle all are divided (one chunk of a wave in ten or so).
template <int E> __device__ __forceinline__ void whole_bytes(const float (&x)[E], float by, float over, uint32_t (&r)[E / 4]) {
    constexpr float kMagic = 0x1.8p23f;
    float y[E], near = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        y[e] = __builtin_fmaf(x[e], over, kMagic);
        near = fmaxf(near, fabsf(__builtin_fmaf(x[e], over, -(y[e] - kMagic))));
    }
    if (__any(near > 0.5f - 0x1p-14f)) {
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = __builtin_rintf(x[e] / by) + kMagic;
    }
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
        const uint32_t a = __builtin_amdgcn_perm(__float_as_uint(y[4 * i + 1]), __float_as_uint(y[4 * i]), 0x0c0c0400u), b = __builtin_amdgcn_perm(__float_as_uint(y[4 * i + 3]), __float_as_uint(y[4 * i + 2]), 0x04000c0cu);
        r[i] = a | b;
    }
}

// The same with rows picked out of those given, and keys normed and rotated on the way: a page's fresh tokens stay in registers, in fp32, from their one read to the
// bytes that are stored, lanes and chunks as seq_rotary.hpp has them.  What is stored is rounded once, from the rotated value.  A workgroup to a page of a head, of keys or of values:
// the page's scale needs all of its tokens, and a page's length decides the registers (STEPS; in 16 bit and 128 channels a round is 32 rows: up to 64 tokens leave room for 5 workgroups a unit, 128 for 3).
// Bound by memory and by the reads that wait for each other (length and count, frequencies, the norm's weights one by one, table, row, values).  8 x 8 x 1000 tokens after 700, D 128, pages of 64, bf16: 24 us (49 MB, 2.0 TB/s; 38 with a division and a clamp for each
// byte and one size of registers), vector instructions 40 % of the cycles, waves wait 50 % of theirs; one token of 64 sequences 7.6 us, latency.
template <typename T, int D, int STEPS>   // STEPS: how often the workgroup's rows go into a page
__global__ __launch_bounds__(kThreads, STEPS <= 2 ? 5 : 3) void append_rows_kernel(const RowsArgs a, int touched) {
    using S = HeadShape<T, D>;
    constexpr int E = S::E, ROWS = kThreads / S::LANES;   // rows of the workgroup at a time
    typedef typename S::vec vec;
    typedef int8_t bytes __attribute__((ext_vector_type(E)));
    __shared__ uint32_t mosts[kWaves];
    const CacheArgs &p = a.c;
    const int tid = threadIdx.x;
    int id = blockIdx.x;
    const bool values = id & 1;
    id >>= 1;
    const int kh = id % p.kv;
    id /= p.kv;
    const int b = id / touched, page = 1 << p.page_log2;
    const int64_t length = p.lengths[b];
    const int count = p.extra ? min(p.extra[b], p.n) : p.n;
    const int i = tid % S::LANES, row0 = tid / S::LANES;
    const bool turned = !values && a.r.pairs, normed = !values && a.r.weight;
    int c0, c1;
    chunks_of<E>(a.r, i, c0, c1);
    // what depends on neither length nor table; a read at a time, waited for, in front of the table's
    float freqs[E], wl[E], wh[E];
#pragma unroll
    for (int e = 0; e < E; ++e) freqs[e] = 0.f, wl[e] = wh[e] = 1.f;
    if (turned && E * i < a.r.pairs) {
#pragma unroll
        for (int e = 0; e < E; ++e) freqs[e] = a.r.freqs[E * i + e];
    }
    if (normed) load_weight<T, E>(a.r, a.r.weight, c0, c1, wl, wh);
    if (length < 0 || count <= 0) return;
    const int64_t at = (length >> p.page_log2) + id % touched, start = at << p.page_log2;
    const int64_t lo = length > start ? length : start, hi = length + count < start + page ? length + count : start + page;
    int to;
    if (lo >= hi || !page_at(p, b, start, to)) return;
    const int64_t unit = (int64_t)to * p.kv + kh;
    int8_t *cells = (values ? p.v : p.k) + unit * page * D;
    float *scales = values ? p.vs : p.ks;
    const View &x = values ? p.b : p.a;
    const int old = (int)(lo - start), fresh = (int)(hi - lo), first = (int)(lo - length);
    const char *plane = x.at + b * x.b + kh * x.h;
    const float before = old ? scales[unit] : 0.f;

    float l[STEPS][E], h[STEPS][E];
    uint32_t bits = 0;   // of the largest magnitude; at or above those of infinity if one is not finite
    int src[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int row = s * ROWS + row0;
        src[s] = -1;
        if (row < fresh) {
            src[s] = a.rows ? a.rows[(int64_t)b * p.n + first + row] : first + row;
            if ((unsigned)src[s] >= (unsigned)a.given) src[s] = -1;
        }
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        vec y{}, z{};
        if (src[s] >= 0) {
            const char *row = plane + (int64_t)src[s] * x.row;
            y = *reinterpret_cast<const vec *>(row + c0 * sizeof(T)), z = *reinterpret_cast<const vec *>(row + c1 * sizeof(T));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) l[s][e] = (float)y[e], h[s][e] = (float)z[e];
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        if (s * ROWS >= fresh) break;
        if (normed) {
            const float r = over_rms<D, S::LANES>(l[s], h[s], a.r.eps);
#pragma unroll
            for (int e = 0; e < E; ++e) l[s][e] *= r * wl[e], h[s][e] *= r * wh[e];
        }
        if (turned && src[s] >= 0) {
            Angles<E, false> angles;
            int position[4] = {(int)(lo + s * ROWS + row0), 0, 0, 0};
            if (a.r.positions) a.r.load(position, a.r.positions + b * a.r.batch + src[s], a.given);
            angles.set(a.r, i, freqs, position);
            angles.template turn<false>(a.r.interleaved, l[s], h[s]);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) bits = max(bits, max(__float_as_uint(l[s][e]) & 0x7fffffffu, __float_as_uint(h[s][e]) & 0x7fffffffu));
    }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) bits = max(bits, (uint32_t)__shfl_xor((int)bits, d));
    if (tid % kWave == 0) mosts[tid / kWave] = bits;
    workgroup_sync();
    float most = __uint_as_float(max(max(mosts[0], mosts[1]), max(mosts[2], mosts[3])));
    if (!(most < INFINITY)) {   // once more, without what is no number
        most = 0.f;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                l[s][e] = finite(l[s][e]), h[s][e] = finite(h[s][e]);
                most = fmaxf(most, fmaxf(fabsf(l[s][e]), fabsf(h[s][e])));
            }
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        workgroup_sync();
        if (tid % kWave == 0) mosts[tid / kWave] = __float_as_uint(most);
        workgroup_sync();
        most = __uint_as_float(max(max(mosts[0], mosts[1]), max(mosts[2], mosts[3])));
    }
    const float scale = fmaxf(fabsf(before), most / 127.f), by = scale > 0.f ? scale : 1.f;
    if (tid == 0) scales[unit] = scale;
    if (old && scale != before) round_again(cells, old * D / 4, before / by, tid);
    const bool divide = !(by > 0x1p-100f && by < 0x1p100f);
    const float over = 1.f / by;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int row = s * ROWS + row0;
        if (row >= fresh) break;
        bytes u, w;
        if (divide) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                u[e] = (int8_t)max(-127, min(127, (int)__builtin_rintf(l[s][e] / by)));
                w[e] = (int8_t)max(-127, min(127, (int)__builtin_rintf(h[s][e] / by)));
            }
        } else {
            uint32_t a[E / 4], b[E / 4];
            whole_bytes<E>(l[s], by, over, a), whole_bytes<E>(h[s], by, over, b);
            u = __builtin_bit_cast(bytes, a), w = __builtin_bit_cast(bytes, b);
        }
        int8_t *cell = cells + (int64_t)(old + row) * D;
        *reinterpret_cast<bytes *>(cell + c0) = u, *reinterpret_cast<bytes *>(cell + c1) = w;
    }
}

// A thread per 16 bytes of the output, of keys and of values, of kRows rows; a row's page, its scales and its cells are three reads that wait for each other,
// the rows' are on their way together.
constexpr int kRows = 4;

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void gather_kernel(const CacheArgs p, int blocks_each) {
    constexpr int E = 16 / (int)sizeof(T), CH = D / E, STEP = kThreads / CH;   // STEP: rows of a workgroup at a time
    typedef T vec __attribute__((ext_vector_type(E)));
    typedef float fvec __attribute__((ext_vector_type(E)));
    typedef int8_t bytes __attribute__((ext_vector_type(E)));
    const int plane = blockIdx.x / blocks_each, row0 = (int)(blockIdx.x % blocks_each) * (STEP * kRows) + threadIdx.x / CH, c = threadIdx.x % CH;
    const int b = plane / p.kv, kh = plane % p.kv;
    const int64_t first = p.extra[b], length = p.lengths[b];
    bool there[kRows];
    int64_t unit[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int64_t position = first + row0 + i * STEP;
        int id = 0;
        there[i] = position >= 0 && position < length && row0 + i * STEP < p.n && page_at(p, b, position, id);
        unit[i] = (int64_t)id * p.kv + kh;
    }
    bytes x[kRows], y[kRows];
    float ks[kRows], vs[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        x[i] = y[i] = bytes{}, ks[i] = vs[i] = 0.f;
        if (there[i]) {
            const int64_t cell = ((unit[i] << p.page_log2) + ((first + row0 + i * STEP) & ((1 << p.page_log2) - 1))) * D + c * E;
            x[i] = *reinterpret_cast<const bytes *>(p.k + cell), y[i] = *reinterpret_cast<const bytes *>(p.v + cell);
            ks[i] = p.ks[unit[i]], vs[i] = p.vs[unit[i]];
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int at = row0 + i * STEP;
        if (at >= p.n) break;
        __builtin_nontemporal_store(__builtin_convertvector(__builtin_convertvector(x[i], fvec) * ks[i], vec),
                                    reinterpret_cast<vec *>(const_cast<char *>(p.a.at) + b * p.a.b + kh * p.a.h + (int64_t)at * p.a.row + c * 16));
        __builtin_nontemporal_store(__builtin_convertvector(__builtin_convertvector(y[i], fvec) * vs[i], vec),
                                    reinterpret_cast<vec *>(const_cast<char *>(p.b.at) + b * p.b.b + kh * p.b.h + (int64_t)at * p.b.row + c * 16));
    }
}

int pages_touched(const CacheArgs &a) {   // that n tokens can lie in
    const int page = 1 << a.page_log2;
    return (a.n + page - 2) / page + 1;
}
template <typename T, int D, int> struct Append {
    static hipError_t go(const CacheArgs &a, hipStream_t st) {
        const int touched = pages_touched(a);
        const int64_t blocks = (int64_t)a.B * touched * a.kv * 2;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        append_kernel<T, D><<<(unsigned)blocks, kThreads, 0, st>>>(a, touched);
        return hipGetLastError();
    }
};
template <typename T, int D, int> struct AppendRows {
    static hipError_t go(const RowsArgs &a, hipStream_t st) {
        const int touched = pages_touched(a.c);
        const int64_t blocks = (int64_t)a.c.B * touched * a.c.kv * 2;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        constexpr int rows = kThreads / HeadShape<T, D>::LANES;
        const int steps = (1 << a.c.page_log2) / rows;
        auto *kernel = steps <= 1 ? append_rows_kernel<T, D, 1> : steps == 2 ? append_rows_kernel<T, D, 2> : append_rows_kernel<T, D, 128 / rows>;
        kernel<<<(unsigned)blocks, kThreads, 0, st>>>(a, touched);
        return hipGetLastError();
    }
};
template <typename T, int D, int> struct Gather {
    static hipError_t go(const CacheArgs &a, hipStream_t st) {
        constexpr int rows = kThreads / (D * (int)sizeof(T) / 16) * kRows;
        const int each = (a.n + rows - 1) / rows;
        const int64_t blocks = (int64_t)a.B * a.kv * each;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        gather_kernel<T, D><<<(unsigned)blocks, kThreads, 0, st>>>(a, each);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_append(const CacheArgs &a, int dtype, int D, hipStream_t st) { return dispatch<Append>(dtype, D, false, a, st); }
hipError_t launch_append_rows(const RowsArgs &a, int dtype, int D, hipStream_t st) { return dispatch<AppendRows>(dtype, D, false, a, st); }
hipError_t launch_gather(const CacheArgs &a, int dtype, int D, hipStream_t st) { return dispatch<Gather>(dtype, D, false, a, st); }

}  // namespace seq
