// Norm of queries' and keys' head vectors and their rotation by position, forward and backward.
//
//   y = x w / sqrt(mean x^2 + eps),  (z_a, z_b) = (y_a cos - y_b sin, y_b cos + y_a sin)
//   dy: dz turned back;  with r = 1 / sqrt(mean x^2 + eps) and g = w dy:  dx = r (g - x r^2 mean(g x)),  dw = sum over tokens and heads of dy x r
//
// Bound by memory: about seven operations an element, and each element read and written once.  A wave takes the tokens of a group, LANES lanes to each, and walks their heads, so
// that angles (in 64 bits) are formed once for all of them.  All (group, head) steps are shared evenly by as many waves as there are at once; a wave reads the next step's vectors
// while it works on one.  2 x (16 + 4) x 8192 tokens, D 128, bf16, three axes, norms: forward 34 us (168 MB, 4.9 TB/s, where a copy of 1 GiB reaches 5.2), backward 50 and 4 (252 MB, 5.0);
// as a launch for each of queries and keys, a wave to a token, 40 and 65.  Vector instructions take 45 % of the cycles; with the library's sine and cosine 40 and 52.  64 x (2 + 2) x 3136, D 32, fp16: 23.5 (103 MB) and 34 + 4.  Eight tokens, one each of 8 sequences, of 40 heads: 6.5, a launch,
// and reads that wait for each other: a lane's frequencies in pairs, the positions, the first row, and the norm's weights one by one (their type is looked up for each).
#include "seq_rotary.hpp"

namespace seq {

namespace {

// A wave's steps, and of the one at hand this lane's token.
template <typename T, int D> struct Steps {
    using S = HeadShape<T, D>;
    const RotaryArgs &p;
    const RotarySide &side;
    const int lane;
    int64_t left, group;
    int head, b, t;
    bool there;
    float freqs[S::E];
    int position[4];
    __device__ __forceinline__ Steps(const RotaryArgs &p_, const RotarySide &side_, int64_t wave, int lane_) : p(p_), side(side_), lane(lane_) {
        const int64_t waves = (int64_t)side.blocks * kWaves, from = side.steps * wave / waves;
        left = side.steps * (wave + 1) / waves - from;
        group = from / side.heads, head = (int)(from - group * side.heads);
        const int i = lane % S::LANES;
#pragma unroll
        for (int e = 0; e < S::E; ++e) freqs[e] = S::E * i < p.r.pairs ? p.r.freqs[S::E * i + e] : 0.f;
        token();
    }
    __device__ __forceinline__ void token() {
        const int64_t at = group * S::TOKENS + lane / S::LANES;
        there = at < p.tokens;
        const uint32_t x = (uint32_t)(there ? at : 0);
        b = (int)(x / (uint32_t)p.L), t = (int)(x - (uint32_t)b * (uint32_t)p.L);
        p.r.load(position, p.r.positions + b * p.r.batch + t, p.L);
    }
    __device__ __forceinline__ void angles(Angles<S::E, sizeof(T) == 4> &a) const { a.set(p.r, lane % S::LANES, freqs, position); }
    __device__ __forceinline__ const char *of(const View &v) const { return v.at + b * v.b + (int64_t)t * v.row + (int64_t)head * v.h; }
    // to the next one; true where its tokens are others
    __device__ __forceinline__ bool next() {
        --left;
        if (++head < side.heads) return false;
        head = 0, ++group;
        token();
        return true;
    }
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 4) void rotary_kernel(const RotaryArgs p) {
    using S = HeadShape<T, D>;
    constexpr int E = S::E;
    typedef typename S::vec vec;
    const bool keys = (int)blockIdx.x >= p.side[0].blocks;
    const RotarySide &side = p.side[keys];
    const int lane = threadIdx.x % kWave;
    Steps<T, D> at(p, side, (int64_t)((int)blockIdx.x - (keys ? p.side[0].blocks : 0)) * kWaves + uniform(threadIdx.x / kWave), lane);
    if (at.left <= 0) return;
    int lo, hi;
    chunks_of<E>(p.r, lane % S::LANES, lo, hi);
    vec xl, xh;
    auto read = [&] {
        const char *row = at.of(side.x);
        xl = *reinterpret_cast<const vec *>(row + lo * sizeof(T)), xh = *reinterpret_cast<const vec *>(row + hi * sizeof(T));
    };
    read();
    float wl[E], wh[E];
    load_weight<T, E>(p.r, side.weight, lo, hi, wl, wh);
    Angles<E, sizeof(T) == 4> angles;
    at.angles(angles);
#pragma unroll 1
    while (true) {
        float l[E], h[E];
#pragma unroll
        for (int e = 0; e < E; ++e) l[e] = (float)xl[e], h[e] = (float)xh[e];
        char *row = const_cast<char *>(at.of(side.z));
        const bool there = at.there, more = at.left > 1;
        bool others = false;
        if (more) {
            others = at.next();
            read();
        }
        if (side.weight) {
            const float r = over_rms<D, S::LANES>(l, h, p.r.eps);
#pragma unroll
            for (int e = 0; e < E; ++e) l[e] *= r * wl[e], h[e] *= r * wh[e];
        }
        angles.template turn<false>(p.r.interleaved, l, h);
        vec yl, yh;
#pragma unroll
        for (int e = 0; e < E; ++e) yl[e] = (T)l[e], yh[e] = (T)h[e];
        if (there) *reinterpret_cast<vec *>(row + lo * sizeof(T)) = yl, *reinterpret_cast<vec *>(row + hi * sizeof(T)) = yh;
        if (!more) return;
        if (others) at.angles(angles);
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void rotary_bwd_kernel(const RotaryArgs p) {
    using S = HeadShape<T, D>;
    constexpr int E = S::E;
    typedef typename S::vec vec;
    __shared__ float sums[kWaves][D];
    const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
    const bool keys = (int)blockIdx.x >= p.side[0].blocks;
    const RotarySide &side = p.side[keys];
    const int block = (int)blockIdx.x - (keys ? p.side[0].blocks : 0);
    Steps<T, D> at(p, side, (int64_t)block * kWaves + wave, lane);
    int lo, hi;
    chunks_of<E>(p.r, lane % S::LANES, lo, hi);
    float wl[E], wh[E], dl[E], dh[E];
#pragma unroll
    for (int e = 0; e < E; ++e) dl[e] = dh[e] = 0.f;
    if (at.left > 0) {
        vec xl{}, xh{}, zl, zh;
        auto read = [&] {
            const char *row = at.of(side.z);
            zl = *reinterpret_cast<const vec *>(row + lo * sizeof(T)), zh = *reinterpret_cast<const vec *>(row + hi * sizeof(T));
            if (side.weight) {
                row = at.of(side.x);
                xl = *reinterpret_cast<const vec *>(row + lo * sizeof(T)), xh = *reinterpret_cast<const vec *>(row + hi * sizeof(T));
            }
        };
        read();
        load_weight<T, E>(p.r, side.weight, lo, hi, wl, wh);
        Angles<E, sizeof(T) == 4> angles;
        at.angles(angles);
#pragma unroll 1
        while (true) {
            float gl[E], gh[E], l[E], h[E];
#pragma unroll
            for (int e = 0; e < E; ++e) gl[e] = (float)zl[e], gh[e] = (float)zh[e], l[e] = (float)xl[e], h[e] = (float)xh[e];
            char *row = const_cast<char *>(at.of(side.dx));
            const bool there = at.there, more = at.left > 1;
            bool others = false;
            if (more) {
                others = at.next();
                read();
            }
            angles.template turn<true>(p.r.interleaved, gl, gh);
            if (side.weight) {
                float dot = 0.f;
                const float r = over_rms<D, S::LANES>(l, h, p.r.eps);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    l[e] *= r, h[e] *= r;   // x r from here on
                    if (there) dl[e] = __builtin_fmaf(gl[e], l[e], dl[e]), dh[e] = __builtin_fmaf(gh[e], h[e], dh[e]);
                    gl[e] *= wl[e], gh[e] *= wh[e];
                    dot = __builtin_fmaf(gl[e], l[e], __builtin_fmaf(gh[e], h[e], dot));
                }
                dot = lanes_sum<S::LANES>(dot) * (1.f / D);
#pragma unroll
                for (int e = 0; e < E; ++e) gl[e] = r * __builtin_fmaf(-l[e], dot, gl[e]), gh[e] = r * __builtin_fmaf(-h[e], dot, gh[e]);
            }
            vec yl, yh;
#pragma unroll
            for (int e = 0; e < E; ++e) yl[e] = (T)gl[e], yh[e] = (T)gh[e];
            if (there) *reinterpret_cast<vec *>(row + lo * sizeof(T)) = yl, *reinterpret_cast<vec *>(row + hi * sizeof(T)) = yh;
            if (!more) break;
            if (others) at.angles(angles);
        }
    }
    if (!side.weight) return;
    // the lanes of a wave that have the same channels, then the waves, in order
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
        for (int d = S::LANES; d < kWave; d *= 2) dl[e] += __shfl_xor(dl[e], d), dh[e] += __shfl_xor(dh[e], d);
        if (lane < S::LANES) sums[wave][lo + e] = dl[e], sums[wave][hi + e] = dh[e];
    }
    workgroup_sync();
    for (int d = threadIdx.x; d < D; d += kThreads) side.parts[(int64_t)block * D + d] = (sums[0][d] + sums[1][d]) + (sums[2][d] + sums[3][d]);
}

// The workgroups' sums, in order: a workgroup per 16 channels of a weight, a thread per channel and every 64th of the parts.
template <typename T, typename W>
__global__ __launch_bounds__(1024) void weight_grad_kernel(const RotaryArgs p, int D) {
    constexpr int GROUPS = 64;
    __shared__ float sums[GROUPS][17];
    const int c = threadIdx.x % 16, g = threadIdx.x / 16, each = D / 16;
    const RotarySide &side = p.side[p.side[0].weight ? blockIdx.x / each : 1];
    const int d = (int)(blockIdx.x % each) * 16 + c;
    float s = 0.f;
#pragma unroll 8
    for (int i = g; i < side.blocks; i += GROUPS) s += side.parts[(int64_t)i * D + d];
    sums[g][c] = s;
    workgroup_sync();
    if (g) return;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) s += sums[i][c];
    static_cast<W *>(side.weight_grad)[d] = (W)s;
}

template <typename T, int D> struct Rotary {
    static unsigned blocks(const RotaryArgs &a) { return (unsigned)(a.side[0].blocks + (a.sides > 1 ? a.side[1].blocks : 0)); }
    static hipError_t go(const RotaryArgs &a, hipStream_t st) {
        rotary_kernel<T, D><<<blocks(a), kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
    static hipError_t back(const RotaryArgs &a, hipStream_t st) {
        rotary_bwd_kernel<T, D><<<blocks(a), kThreads, 0, st>>>(a);
        const int normed = (a.side[0].weight ? 1 : 0) + (a.side[1].weight ? 1 : 0);
        if (hipError_t e = hipGetLastError(); e != hipSuccess || !normed) return e;
        if (a.r.weight32) weight_grad_kernel<T, float><<<normed * (D / 16), 1024, 0, st>>>(a, D);
        else weight_grad_kernel<T, T><<<normed * (D / 16), 1024, 0, st>>>(a, D);
        return hipGetLastError();
    }
};

}  // namespace

// As many workgroups as there are at once, shared by queries and keys as their heads are; fewer where a wave would have nothing to do.
void plan_rotary(RotaryArgs &a, int dtype, int D, bool backward) {
    const int most = backward ? 768 : 1280;   // what the registers let run at once: three or five workgroups to a compute unit
    const int tokens = kWave / (D * (dtype == NA2D_F32 ? 4 : 2) / 32);
    const int64_t groups = (a.tokens + tokens - 1) / tokens;
    double all = 0;
    for (int i = 0; i < a.sides; ++i) all += a.side[i].heads;
    for (int i = 0; i < a.sides; ++i) {
        RotarySide &x = a.side[i];
        x.steps = groups * x.heads;
        const int64_t blocks = (x.steps + kWaves - 1) / kWaves, share = (int64_t)(most * x.heads / all + 0.5);
        x.blocks = (int)(blocks < share ? blocks : share > 1 ? share : 1);
    }
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
hipError_t launch_rotary_bwd(const RotaryArgs &a, int dtype, int D, hipStream_t st) { SEQ_ALL(back(a, st)); }
#undef SEQ_ALL

}  // namespace seq
