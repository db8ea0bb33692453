// Attention of a few new tokens over a cache in 8 bits.
//
// The rows of a key head, its query heads times the new tokens, are columns of the products, 16 to a block; tokens come in steps of 32.  A wave
// takes every fourth step of its workgroup's range, straight from memory into registers, the next step's bytes on their way while one is
// worked on:
//   S^T = K Q^T     a byte b enters as fp16: (b ^ 0x80) behind the byte 0x64 is 1152 + b, exactly; the page's scale multiplies the sums
//   P = exp2(S' - ref), rounded to fp16
//   O^T += vs V^T P  a lane holds D / 16 channels of its eight tokens; product block db takes channel db of each lane, so no value changes lanes
// The four waves' parts are joined through LDS.  Few sequences: their ranges are split over workgroups, and a second kernel joins the splits in order.
#include "seq_cache.hpp"

namespace seq {

namespace {

constexpr int kStep = 32;
constexpr float kSlack = 8.f;

__device__ __forceinline__ uint32_t perm(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }
__device__ __forceinline__ uint32_t minus1152(uint32_t x) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, x) - f16x2{(f16_t)1152.f, (f16_t)1152.f}); }
// bytes 0, 1 and bytes 2, 3 of four (each ^ 0x80) as fp16
__device__ __forceinline__ uint32_t low_pair(uint32_t x) { return minus1152(perm(0x64646464u, x, 0x04010400u)); }
__device__ __forceinline__ uint32_t high_pair(uint32_t x) { return minus1152(perm(0x64646464u, x, 0x04030402u)); }

template <int D> struct Shape {
    static constexpr int KW = D / 32;        // words of a token's keys in a lane for each group of 8 channels per product step, two words each
    static constexpr int STEPS = D / 32;     // products over the head vector
    static constexpr int DB = D / 16;        // channels of a lane's values, blocks of 16 channels
};

// A step's bytes: two blocks of 16 keys, lane (j, g) 8 bytes of row j for each product step; of the values, channels DB j .. of the tokens 4 g + e of both blocks.
template <int D> struct Bytes {
    uint32_t k[2][2 * (D / 32)];
    uint32_t v[8][D >= 64 ? D / 64 : 1];
    __device__ __forceinline__ void load(const int8_t *const (&kp)[2], const int8_t *const (&vp)[2], int lane) {
        const int j = lane & 15, g = lane >> 4;
        typedef uint32_t w2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (D >= 64) {   // 16 bytes: two product steps
#pragma unroll
                for (int u = 0; u < D / 64; ++u) {
                    const u32x4 x = *reinterpret_cast<const u32x4 *>(kp[i] + j * D + u * 64 + g * 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) k[i][4 * u + e] = x[e];
                }
            } else {
                const w2 x = *reinterpret_cast<const w2 *>(kp[i] + j * D + g * 8);
                k[i][0] = x[0], k[i][1] = x[1];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int8_t *at = vp[i] + (4 * g + e) * D + j * (D / 16);
                if constexpr (D == 128) {
                    const w2 x = *reinterpret_cast<const w2 *>(at);
                    v[4 * i + e][0] = x[0], v[4 * i + e][1] = x[1];
                } else if constexpr (D == 64) {
                    v[4 * i + e][0] = *reinterpret_cast<const uint32_t *>(at);
                } else {
                    v[4 * i + e][0] = *reinterpret_cast<const uint16_t *>(at);
                }
            }
        }
    }
    // keys of block i for product step s
    __device__ __forceinline__ u32x4 keys(int i, int s) const {
        const uint32_t x = k[i][2 * s] ^ 0x80808080u, y = k[i][2 * s + 1] ^ 0x80808080u;
        return u32x4{low_pair(x), high_pair(x), low_pair(y), high_pair(y)};
    }
    // channel db of the eight tokens
    __device__ __forceinline__ u32x4 values(int db) const {
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = v[2 * i][db / 4] ^ 0x80808080u, y = v[2 * i + 1][db / 4] ^ 0x80808080u;
            r[i] = minus1152(perm(y, x, 0x0c000c00u | (uint32_t)(db % 4) | (uint32_t)(db % 4 + 4) << 16) | 0x64006400u);
        }
        return r;
    }
};

template <typename T, int D, int RT, bool CAP>
__global__ __launch_bounds__(kThreads, (RT == 1 ? 3 : 2) - (D == 128)) void decode_kernel(const CacheArgs p) {
    using S = Shape<D>;
    constexpr int ROWS = 16 * RT;
    __shared__ __align__(16) float parts[kWaves][16][D + 4];
    __shared__ float refs[kWaves][ROWS], sums[kWaves][ROWS];
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave), j = lane & 15, g = lane >> 4;
    int id = blockIdx.x;
    const int split = id % p.splits;
    id /= p.splits;
    const int rg = id % p.row_groups;
    id /= p.row_groups;
    const int kh = id % p.kv, b = id / p.kv, page = 1 << p.page_log2;
    const int all_rows = p.group * p.n, row0 = rg * ROWS;
    const int64_t most_tokens = (int64_t)p.width << p.page_log2;
    const int length = (int)min((int64_t)p.lengths[b], most_tokens), first_query = p.lengths[b] - p.n;

    // rows as fp16 on a power of two of their own
    u32x4 q[RT][S::STEPS];
    int pos[RT];
    float c[RT], slope[RT];
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        const int row = min(row0 + 16 * n + j, all_rows - 1), h = kh * p.group + row / p.n, i = row % p.n;
        const char *at = p.a.at + b * p.a.b + h * p.a.h + (int64_t)i * p.a.row;
        pos[n] = first_query + i;
        slope[n] = p.slopes ? p.slopes[h] * kLog2e : 0.f;
        typedef T vec __attribute__((ext_vector_type(8)));
        vec x[S::STEPS];
        float most = 0.f;
#pragma unroll
        for (int s = 0; s < S::STEPS; ++s) {
            const int channel = D >= 64 ? s / 2 * 64 + g * 16 + s % 2 * 8 : g * 8;
            x[s] = *reinterpret_cast<const vec *>(at + channel * (int)sizeof(T));
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf((float)x[s][e]));
        }
        most = column_max(most);
        const int power = most > 0.f && most < INFINITY ? __builtin_amdgcn_frexp_expf(most) : 0;
        c[n] = p.c * __builtin_amdgcn_ldexpf(1.f, power);
#pragma unroll
        for (int s = 0; s < S::STEPS; ++s) {
            f16x8 y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (f16_t)__builtin_amdgcn_ldexpf((float)x[s][e], -power);
            q[n][s] = __builtin_bit_cast(u32x4, y);
        }
    }

    // the range that any row sees, in steps, and this workgroup's part of it
    const int begin = max(0, first_query - p.window + 1) / kStep, end = length > 0 ? (length + kStep - 1) / kStep : 0;
    const int each = max(0, (end - begin + p.splits - 1) / p.splits), from = begin + split * each, to = min(end, from + each);

    f32x4 out[RT][S::DB];
    float ref[RT], sum[RT];
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        ref[n] = kLowest, sum[n] = 0.f;
#pragma unroll
        for (int db = 0; db < S::DB; ++db) out[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // a lane looks up one of the wave's next 64 steps: its pages (two where they are of 16 tokens) and their scales
    int unit[2];
    float ks[2], vs[2];
    auto look_up = [&](int step) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int page_id = 0;
            const bool there = step < to && page_at(p, b, (int64_t)step * kStep + (page == 16 ? 16 * i : 0), page_id);
            unit[i] = there ? page_id : -1;
            const int64_t u = (int64_t)(there ? page_id : 0) * p.kv + kh;
            ks[i] = there ? p.ks[u] : 0.f, vs[i] = there ? p.vs[u] : 0.f;
        }
    };
    struct Step {
        bool there[2];
        float ks[2], vs[2];
    };
    auto fetch = [&](Bytes<D> &bytes, Step &info, int step, int slot) {
        const int8_t *kp[2], *vp[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int u = __builtin_amdgcn_readlane(unit[i], slot);
            info.there[i] = u >= 0;
            info.ks[i] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks[i]), slot));
            info.vs[i] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs[i]), slot));
            const int64_t cell = (((int64_t)max(u, 0) * p.kv + kh) * page + ((step * kStep + 16 * i) & (page - 1))) * D;
            kp[i] = p.k + cell, vp[i] = p.v + cell;
        }
        bytes.load(kp, vp, lane);
    };
    auto work = [&](const Bytes<D> &bytes, const Step &info, int step) {
        const int t0 = step * kStep;
        f32x4 s[RT][2];
#pragma unroll
        for (int n = 0; n < RT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) s[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < S::STEPS; ++st)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x4 a = bytes.keys(i, st);
#pragma unroll
                for (int n = 0; n < RT; ++n) s[n][i] = mma<f16_t>(a, q[n][st], s[n][i]);
            }
        // every row sees all of it
        const bool all = info.there[0] && info.there[1] && t0 + kStep - 1 <= first_query && first_query + p.n - 1 - t0 < p.window;
        u32x4 w[RT];
#pragma unroll
        for (int n = 0; n < RT; ++n) {
            float most = -INFINITY;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = t0 + 16 * i + 4 * g + r;
                    float x = s[n][i][r] * (c[n] * info.ks[i]);
                    if constexpr (CAP) x = __builtin_fmaf(-p.cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x)), 0.5f * p.cap);
                    if (p.slopes) x = __builtin_fmaf((float)(pos[n] - key), -slope[n], x);
                    if (!all && !(info.there[i] && key <= pos[n] && pos[n] - key < p.window)) x = -INFINITY;
                    s[n][i][r] = x;
                    most = fmaxf(most, x);
                }
            most = column_max(most);
            const float now = most > ref[n] + kSlack ? most : ref[n];
            if (__any(now != ref[n])) {
                const float by = __builtin_amdgcn_exp2f(ref[n] - now);
                sum[n] *= by;
#pragma unroll
                for (int db = 0; db < S::DB; ++db) out[n][db] *= by;
                ref[n] = now;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[n][i][r] = __builtin_amdgcn_exp2f(s[n][i][r] - ref[n]);
                    sum[n] += s[n][i][r];
                }
            w[n] = pack<f16_t>(s[n]);
        }
        if (page == 16) {   // the two blocks have scales of their own
#pragma unroll
            for (int db = 0; db < S::DB; ++db) {
                const u32x4 a = bytes.values(db);
#pragma unroll
                for (int n = 0; n < RT; ++n) {
                    const f32x4 zero{0.f, 0.f, 0.f, 0.f};
                    const f32x4 x = mma<f16_t>(a, u32x4{w[n][0], w[n][1], 0u, 0u}, zero), y = mma<f16_t>(a, u32x4{0u, 0u, w[n][2], w[n][3]}, zero);
#pragma unroll
                    for (int r = 0; r < 4; ++r) out[n][db][r] = __builtin_fmaf(y[r], info.vs[1], __builtin_fmaf(x[r], info.vs[0], out[n][db][r]));
                }
            }
        } else {
#pragma unroll
            for (int db = 0; db < S::DB; ++db) {
                const u32x4 a = bytes.values(db);
#pragma unroll
                for (int n = 0; n < RT; ++n) {
                    const f32x4 x = mma<f16_t>(a, w[n], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                    for (int r = 0; r < 4; ++r) out[n][db][r] = __builtin_fmaf(x[r], info.vs[0], out[n][db][r]);
                }
            }
        }
    };

#pragma unroll 1
    for (int base = from + wave; base < to; base += kWave * kWaves) {
        look_up(base + lane * kWaves);
        const int steps = min(kWave, (to - base + kWaves - 1) / kWaves);
        Bytes<D> here, ahead;
        Step info, info_ahead;
        fetch(here, info, base, 0);
#pragma unroll 1
        for (int i = 0; i < steps; ++i) {
            const int next = min(i + 1, steps - 1);
            fetch(ahead, info_ahead, base + next * kWaves, next);
            work(here, info, base + i * kWaves);
            here = ahead, info = info_ahead;
        }
    }

    // the four waves' parts, then this workgroup's
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        settle_products(out[n]);
        const float total = column_sum(sum[n]);
        if (g == 0) refs[wave][16 * n + j] = ref[n], sums[wave][16 * n + j] = total;
    }
    const int64_t unit_rows = (int64_t)ROWS, item = (((int64_t)b * p.kv + kh) * p.row_groups + rg) * p.splits + split;
    const int64_t items = (int64_t)p.B * p.kv * p.row_groups * p.splits;
    float *part = p.part + item * unit_rows * D, *stats = p.part + items * unit_rows * D + item * unit_rows * 2;
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        workgroup_sync();   // (also before parts are written again)
        float most = refs[0][16 * n + j];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) most = fmaxf(most, refs[w][16 * n + j]);
        const float by = __builtin_amdgcn_exp2f(ref[n] - most);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int db = 0; db < S::DB; ++db) parts[wave][j][S::DB * (4 * g + r) + db] = out[n][db][r] * by;
        workgroup_sync();
        for (int i = tid; i < 16 * D / 8; i += kThreads) {
            const int r = i / (D / 8), d = i % (D / 8) * 8, row = row0 + 16 * n + r;
            if (row >= all_rows) continue;
            float m = refs[0][16 * n + r], total = 0.f;
#pragma unroll
            for (int w = 1; w < kWaves; ++w) m = fmaxf(m, refs[w][16 * n + r]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) total += sums[w][16 * n + r] * __builtin_amdgcn_exp2f(refs[w][16 * n + r] - m);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = parts[0][r][d + e] + parts[1][r][d + e] + parts[2][r][d + e] + parts[3][r][d + e];
            if (p.splits == 1) {
                const float by_sum = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= by_sum;
                const int h = kh * p.group + row / p.n;
                store_vec32<T, 8>(const_cast<char *>(p.b.at) + b * p.b.b + h * p.b.h + (int64_t)(row % p.n) * p.b.row + d * (int)sizeof(T), x);
            } else {
                store_vec32<float, 8>(part + (16 * n + r) * D + d, x);
                if (d == 0) stats[2 * (16 * n + r)] = m, stats[2 * (16 * n + r) + 1] = total;
            }
        }
    }
}

// The splits of a row, in order; a thread per 8 channels.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void join_kernel(const CacheArgs p, int rows_each, int64_t total) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= total) return;
    const int d = (int)(i % (D / 8)) * 8, all_rows = p.group * p.n;
    const int64_t at = i / (D / 8);
    const int row = (int)(at % all_rows), plane = (int)(at / all_rows), b = plane / p.kv, kh = plane % p.kv;
    const int64_t items = (int64_t)p.B * p.kv * p.row_groups * p.splits, first = ((int64_t)plane * p.row_groups + row / rows_each) * p.splits;
    const float *stats = p.part + items * rows_each * D;
    const int r = row % rows_each;
    float m = kLowest;
    for (int s = 0; s < p.splits; ++s) m = fmaxf(m, stats[((first + s) * rows_each + r) * 2]);
    float x[8] = {}, sum = 0.f;
    for (int s = 0; s < p.splits; ++s) {
        const float *st = stats + ((first + s) * rows_each + r) * 2;
        const float by = __builtin_amdgcn_exp2f(st[0] - m);
        const f32x4 *y = reinterpret_cast<const f32x4 *>(p.part + ((first + s) * rows_each + r) * D + d);
        const f32x4 lo = y[0], hi = y[1];
        sum = __builtin_fmaf(st[1], by, sum);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(lo[e], by, x[e]), x[4 + e] = __builtin_fmaf(hi[e], by, x[4 + e]);
    }
    const float by = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= by;
    const int h = kh * p.group + row / p.n;
    store_vec32<T, 8>(const_cast<char *>(p.b.at) + b * p.b.b + h * p.b.h + (int64_t)(row % p.n) * p.b.row + d * (int)sizeof(T), x);
}

int rows_each(const CacheArgs &a) { return a.group * a.n > 16 ? 32 : 16; }

template <typename T, int D, bool CAP> struct Decode {
    static hipError_t go(const CacheArgs &a, hipStream_t st) {
        const int64_t blocks = (int64_t)a.B * a.kv * a.row_groups * a.splits;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        if (rows_each(a) == 16) decode_kernel<T, D, 1, CAP><<<(unsigned)blocks, kThreads, 0, st>>>(a);
        else decode_kernel<T, D, 2, CAP><<<(unsigned)blocks, kThreads, 0, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess || a.splits == 1) return e;
        const int64_t total = (int64_t)a.B * a.heads * a.n * (D / 8), joins = (total + kThreads - 1) / kThreads;
        if (!launch_holds(joins, kThreads)) return hipErrorInvalidValue;
        join_kernel<T, D><<<(unsigned)joins, kThreads, 0, st>>>(a, rows_each(a), total);
        return hipGetLastError();
    }
};

}  // namespace

// Ranges are split where whole sequences would leave compute units without work: until there are about four workgroups to each of the 256, but no
// split is given less than 256 tokens of the longest sequence that the table can hold.
void plan_cache_attention(CacheArgs &a, int D, int64_t longest) {
    (void)D;
    a.row_groups = (a.group * a.n + rows_each(a) - 1) / rows_each(a);
    const int64_t reach = longest < (int64_t)a.window + a.n ? longest : (int64_t)a.window + a.n;
    const int64_t units = (int64_t)a.B * a.kv * a.row_groups, wanted = (1024 + units - 1) / units, most = reach / 256;
    int64_t s = wanted < most ? wanted : most;
    a.splits = (int)(s < 1 ? 1 : s > 128 ? 128 : s);
}
size_t cache_attention_bytes(const CacheArgs &a, int D) {
    return a.splits == 1 ? 0 : (size_t)a.B * a.kv * a.row_groups * a.splits * rows_each(a) * (D + 2) * sizeof(float);
}

hipError_t launch_cache_attention(const CacheArgs &a, int dtype, int D, bool capped, hipStream_t st) {
#define SEQ_D(T, N) (capped ? Decode<T, N, true>::go(a, st) : Decode<T, N, false>::go(a, st))
#define SEQ_T(T) (D == 32 ? SEQ_D(T, 32) : D == 64 ? SEQ_D(T, 64) : SEQ_D(T, 128))
    return dtype == NA2D_F16 ? SEQ_T(f16_t) : SEQ_T(bf16_t);
#undef SEQ_T
#undef SEQ_D
}

}  // namespace seq
