// Norm of queries' and keys' head vectors and their rotation by position, forward and backward.
//
//   y = x w / sqrt(mean x^2 + eps),  (z_a, z_b) = (y_a cos - y_b sin, y_b cos + y_a sin)
//   dy: dz turned back;  with r = 1 / sqrt(mean x^2 + eps) and g = w dy:  dx = r (g - x r^2 mean(g x)),  dw = sum over tokens and heads of dy x r
//
// Bound by memory: about seven operations an element, and each element read and written once.  A wave has the tokens of a group, LANES lanes to each, and walks their heads,
// so that angles (in 64 bits) are formed once for all of them.
#include "seq_rotary.hpp"

namespace seq {

namespace {

constexpr int kHeads = 4, kHeadsBack = 2;   // heads whose reads are on their way together
constexpr int kMostBlocks = 1024;           // workgroups that leave sums of a weight's gradient

// This lane's token, and the heads of its unit.
template <typename T, int D> struct Place {
    int b, t, i, h0, h1;
    bool there;
    __device__ __forceinline__ Place(const RotaryArgs &p, int64_t unit, int lane) {
        using S = HeadShape<T, D>;
        const int64_t group = unit / p.head_parts;
        const int part = (int)(unit - group * p.head_parts);
        const int64_t token = group * S::TOKENS + lane / S::LANES;
        there = token < p.tokens;
        const uint32_t at = (uint32_t)(there ? token : 0);
        b = (int)(at / (uint32_t)p.L), t = (int)(at - (uint32_t)b * (uint32_t)p.L), i = lane % S::LANES;
        const int each = (p.heads + p.head_parts - 1) / p.head_parts;
        h0 = part * each, h1 = min(p.heads, h0 + each);
    }
    __device__ __forceinline__ void angles(const RotaryArgs &p, Angles<HeadShape<T, D>::E> &a) const { a.set(p.r, i, p.r.positions + b * p.r.batch + t, p.L, 0); }
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs p) {
    using S = HeadShape<T, D>;
    constexpr int E = S::E;
    typedef typename S::vec vec;
    const int lane = threadIdx.x % kWave;
    const int64_t unit = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave;
    if (unit >= p.units) return;
    const Place<T, D> at(p, unit, lane);
    if (!at.there) return;
    int lo, hi;
    chunks_of<E>(p.r, at.i, lo, hi);
    const char *x = p.x.at + at.b * p.x.b + (int64_t)at.t * p.x.row;
    char *z = const_cast<char *>(p.z.at) + at.b * p.z.b + (int64_t)at.t * p.z.row;
    vec xl[kHeads], xh[kHeads];
    auto read = [&](int h0) {
#pragma unroll
        for (int u = 0; u < kHeads; ++u) {
            const char *row = x + (int64_t)min(h0 + u, at.h1 - 1) * p.x.h;
            xl[u] = *reinterpret_cast<const vec *>(row + lo * sizeof(T)), xh[u] = *reinterpret_cast<const vec *>(row + hi * sizeof(T));
        }
    };
    if (at.h0 < at.h1) read(at.h0);   // (before the angles: they take a while)
    Angles<E> angles;
    at.angles(p, angles);
    float wl[E], wh[E];
    load_weight<T, E>(p.r, lo, hi, wl, wh);
#pragma unroll 1
    for (int h0 = at.h0; h0 < at.h1; h0 += kHeads) {
        if (h0 != at.h0) read(h0);
#pragma unroll
        for (int u = 0; u < kHeads; ++u) {
            if (h0 + u >= at.h1) break;
            float l[E], h[E];
#pragma unroll
            for (int e = 0; e < E; ++e) l[e] = (float)xl[u][e], h[e] = (float)xh[u][e];
            if (p.r.weight) {
                const float r = over_rms<D, S::LANES>(l, h, p.r.eps);
#pragma unroll
                for (int e = 0; e < E; ++e) l[e] *= r * wl[e], h[e] *= r * wh[e];
            }
            angles.template turn<false>(p.r.interleaved, l, h);
            vec yl, yh;
#pragma unroll
            for (int e = 0; e < E; ++e) yl[e] = (T)l[e], yh[e] = (T)h[e];
            char *row = z + (int64_t)(h0 + u) * p.z.h;
            *reinterpret_cast<vec *>(row + lo * sizeof(T)) = yl, *reinterpret_cast<vec *>(row + hi * sizeof(T)) = yh;
        }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void rotary_bwd_kernel(const RotaryArgs p) {
    using S = HeadShape<T, D>;
    constexpr int E = S::E;
    typedef typename S::vec vec;
    __shared__ float sums[kWaves][D];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int lo, hi;
    chunks_of<E>(p.r, lane % S::LANES, lo, hi);
    float wl[E], wh[E], dl[E], dh[E];
    load_weight<T, E>(p.r, lo, hi, wl, wh);
#pragma unroll
    for (int e = 0; e < E; ++e) dl[e] = dh[e] = 0.f;
#pragma unroll 1
    for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < p.units; unit += (int64_t)gridDim.x * kWaves) {
        const Place<T, D> at(p, unit, lane);
        Angles<E> angles;
        at.angles(p, angles);
        const char *x = p.x.at + at.b * p.x.b + (int64_t)at.t * p.x.row, *z = p.z.at + at.b * p.z.b + (int64_t)at.t * p.z.row;
        char *dx = const_cast<char *>(p.dx.at) + at.b * p.dx.b + (int64_t)at.t * p.dx.row;
#pragma unroll 1
        for (int h0 = at.h0; h0 < at.h1; h0 += kHeadsBack) {
            vec xl[kHeadsBack], xh[kHeadsBack], zl[kHeadsBack], zh[kHeadsBack];
#pragma unroll
            for (int u = 0; u < kHeadsBack; ++u) {
                const int head = min(h0 + u, at.h1 - 1);
                const char *row = z + (int64_t)head * p.z.h;
                zl[u] = *reinterpret_cast<const vec *>(row + lo * sizeof(T)), zh[u] = *reinterpret_cast<const vec *>(row + hi * sizeof(T));
                if (p.r.weight) {
                    row = x + (int64_t)head * p.x.h;
                    xl[u] = *reinterpret_cast<const vec *>(row + lo * sizeof(T)), xh[u] = *reinterpret_cast<const vec *>(row + hi * sizeof(T));
                }
            }
#pragma unroll
            for (int u = 0; u < kHeadsBack; ++u) {
                if (h0 + u >= at.h1) break;
                float gl[E], gh[E];
#pragma unroll
                for (int e = 0; e < E; ++e) gl[e] = (float)zl[u][e], gh[e] = (float)zh[u][e];
                angles.template turn<true>(p.r.interleaved, gl, gh);
                if (p.r.weight) {
                    float l[E], h[E], dot = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) l[e] = (float)xl[u][e], h[e] = (float)xh[u][e];
                    const float r = over_rms<D, S::LANES>(l, h, p.r.eps);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        l[e] *= r, h[e] *= r;   // x r from here on
                        if (at.there) dl[e] = __builtin_fmaf(gl[e], l[e], dl[e]), dh[e] = __builtin_fmaf(gh[e], h[e], dh[e]);
                        gl[e] *= wl[e], gh[e] *= wh[e];
                        dot = __builtin_fmaf(gl[e], l[e], __builtin_fmaf(gh[e], h[e], dot));
                    }
                    dot = lanes_sum<S::LANES>(dot) * (1.f / D);
#pragma unroll
                    for (int e = 0; e < E; ++e) gl[e] = r * __builtin_fmaf(-l[e], dot, gl[e]), gh[e] = r * __builtin_fmaf(-h[e], dot, gh[e]);
                }
                if (at.there) {
                    vec yl, yh;
#pragma unroll
                    for (int e = 0; e < E; ++e) yl[e] = (T)gl[e], yh[e] = (T)gh[e];
                    char *row = dx + (int64_t)(h0 + u) * p.dx.h;
                    *reinterpret_cast<vec *>(row + lo * sizeof(T)) = yl, *reinterpret_cast<vec *>(row + hi * sizeof(T)) = yh;
                }
            }
        }
    }
    if (!p.r.weight) return;
    // the lanes of a wave that have the same channels, then the waves, in order
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
        for (int d = S::LANES; d < kWave; d *= 2) dl[e] += __shfl_xor(dl[e], d), dh[e] += __shfl_xor(dh[e], d);
        if (lane < S::LANES) sums[wave][lo + e] = dl[e], sums[wave][hi + e] = dh[e];
    }
    workgroup_sync();
    for (int d = threadIdx.x; d < D; d += kThreads) p.parts[(int64_t)blockIdx.x * D + d] = (sums[0][d] + sums[1][d]) + (sums[2][d] + sums[3][d]);
}

// The workgroups' sums, in order: a workgroup per 16 channels, a thread per channel and every 16th of the parts.
template <typename W>
__global__ __launch_bounds__(kThreads) void weight_grad_kernel(const float *parts, W *out, int blocks, int D) {
    __shared__ float sums[16][17];
    const int c = threadIdx.x % 16, g = threadIdx.x / 16, d = blockIdx.x * 16 + c;
    float s = 0.f;
#pragma unroll 8
    for (int i = g; i < blocks; i += 16) s += parts[(int64_t)i * D + d];
    sums[g][c] = s;
    workgroup_sync();
    if (g) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += sums[i][c];
    out[d] = (W)s;
}

template <typename T, int D> struct Rotary {
    static hipError_t go(const RotaryArgs &a, hipStream_t st) {
        const int64_t blocks = (a.units + kWaves - 1) / kWaves;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        rotary_kernel<T, D><<<(unsigned)blocks, kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
    static hipError_t back(const RotaryArgs &a, void *weight_grad, hipStream_t st) {
        const int blocks = rotary_bwd_blocks(a);
        rotary_bwd_kernel<T, D><<<(unsigned)blocks, kThreads, 0, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess || !a.r.weight) return e;
        if (a.r.weight32) weight_grad_kernel<float><<<D / 16, kThreads, 0, st>>>(a.parts, static_cast<float *>(weight_grad), blocks, D);
        else weight_grad_kernel<T><<<D / 16, kThreads, 0, st>>>(a.parts, static_cast<T *>(weight_grad), blocks, D);
        return hipGetLastError();
    }
};

}  // namespace

// Waves for every SIMD of the chip, four to each, where there are heads to share among them.
void plan_rotary(RotaryArgs &a, int dtype, int D) {
    const int tokens = kWave / (D * (dtype == NA2D_F32 ? 4 : 2) / 32);
    const int64_t groups = (a.tokens + tokens - 1) / tokens, wanted = (4096 + groups - 1) / groups, most = (a.heads + kHeads - 1) / kHeads;
    a.head_parts = (int)(wanted < most ? wanted : most);
    a.units = groups * a.head_parts;
}
int rotary_bwd_blocks(const RotaryArgs &a) {
    const int64_t blocks = (a.units + kWaves - 1) / kWaves;
    return (int)(blocks < kMostBlocks ? blocks : kMostBlocks);
}

#define SEQ_ALL(call)                                                                                                                 \
    do {                                                                                                                              \
        const auto of = [&](auto t) {                                                                                                 \
            using T = decltype(t);                                                                                                    \
            return D == 16 ? Rotary<T, 16>::call : D == 32 ? Rotary<T, 32>::call : D == 64 ? Rotary<T, 64>::call : Rotary<T, 128>::call; \
        };                                                                                                                            \
        return dtype == NA2D_F32 ? of(float{}) : dtype == NA2D_F16 ? of(f16_t{}) : of(bf16_t{});                                      \
    } while (0)
hipError_t launch_rotary(const RotaryArgs &a, int dtype, int D, hipStream_t st) { SEQ_ALL(go(a, st)); }
hipError_t launch_rotary_bwd(const RotaryArgs &a, int dtype, int D, void *weight_grad, hipStream_t st) { SEQ_ALL(back(a, weight_grad, st)); }
#undef SEQ_ALL

}  // namespace seq
