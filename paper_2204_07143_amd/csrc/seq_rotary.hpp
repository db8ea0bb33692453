// Rotation of head vectors by their tokens' positions, and the norm before it: what the kernels that do it share.
//
// A head vector is worked on by LANES lanes, each with two chunks of 16 bytes, `lo` and `hi`, such that both channels of a pair are in one lane: pair E i + e is element
// e of lane i's two chunks (channels p and p + pairs), or neighbours within them (2 p and 2 p + 1).  No channel changes lanes, and the angles of a lane's E pairs, which
// depend on the token alone, stay in registers for all of its heads.
#pragma once

#include "seq_common.hpp"

namespace seq {

struct Rotation {
    const int *positions;      // [axes, tokens] of batch item b at positions + b * batch; null: given by the kernel, on one axis
    const float *freqs;        // radians a position, [pairs]
    const void *weight;        // of the append's norm, [D]; null: no norm
    int64_t batch;
    int pairs, axes, ends[3];  // axis a has the pairs below ends[a] that the axes before it do not have
    int interleaved, weight32;
    float eps;
    // a token's positions: at the first axis', `step` from axis to axis
    __device__ __forceinline__ void load(int (&p)[4], const int *at, int64_t step) const {
        p[0] = at[0];
#pragma unroll
        for (int a = 1; a < 4; ++a) p[a] = a < axes ? at[a * step] : 0;
    }
};

// Queries, or keys.
struct RotarySide {
    View x, z, dx;             // forward: x to z.  backward: x (where there is a norm) and z's gradient to dx
    const void *weight;
    void *weight_grad;
    float *parts;              // backward with a norm: every workgroup's sums of the weight's gradient, [blocks, D]
    int64_t steps;             // groups of tokens times heads
    int heads, blocks;         // blocks: workgroups that share them
};
struct RotaryArgs {
    Rotation r;
    RotarySide side[2];
    int64_t tokens;            // B * L
    int L, sides;
};

template <typename T, int D> struct HeadShape {
    static constexpr int E = 16 / (int)sizeof(T), LANES = D / (2 * E), TOKENS = kWave / LANES;
    typedef T vec __attribute__((ext_vector_type(E)));
};

// First channels of lane i's two chunks.
template <int E> __device__ __forceinline__ void chunks_of(const Rotation &r, int i, int &lo, int &hi) {
    const bool split = !r.interleaved && E * i < r.pairs;
    lo = split ? E * i : 2 * E * i, hi = split ? r.pairs + E * i : 2 * E * i + E;
}

// cos and sin of position * freq.  The angle is formed in turns in 64 bits (2^-53 of them: 2^31 turns leave 22 bits of the last), reduced there, and rounded to fp32.  What
// becomes 16 or 8 bits takes the processor's own functions of turns, off by 2^-22.9 at most (measured over 2^22 angles).  fp32 takes the library's, and what the angle's rounding took away is put right to
// first order: off by 2^-23.6 at most, in the mean square 2^-25.7, at positions to 2^20, 2^-22.5 and 2^-25.1 at all (without that 2^-22.1 and 2^-24.7 there; 3 x (6 + 2) x 3137, D 64: 11 us for 10).
template <bool EXACT> __device__ __forceinline__ void cos_sin(int position, float freq, float &c, float &s) {
    double turns = (double)position * ((double)freq * 0.15915494309189534561);
    turns -= __builtin_rint(turns);
    if constexpr (EXACT) {
        const float near = (float)turns, rest = (float)((turns - near) * 6.2831853071795864769);
        float a, b;
        sincospif(2.f * near, &b, &a);
        c = __builtin_fmaf(-rest, b, a), s = __builtin_fmaf(rest, a, b);
    } else s = __builtin_amdgcn_sinf((float)turns), c = __builtin_amdgcn_cosf((float)turns);
}

// Of lane i's pairs, freqs theirs, at a token's positions; cos 1 and sin 0 where a pair is not rotated.
template <int E, bool EXACT> struct Angles {
    float c[E], s[E];
    __device__ __forceinline__ void set(const Rotation &r, int i, const float (&freqs)[E], const int (&p)[4]) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int pair = E * i + e;
            c[e] = 1.f, s[e] = 0.f;
            if (pair < r.pairs) {   // (all of a lane's pairs or none: pairs is a multiple of 8)
                const int position = r.axes == 1 || pair < r.ends[0] ? p[0] : pair < r.ends[1] ? p[1] : pair < r.ends[2] ? p[2] : p[3];
                cos_sin<EXACT>(position, freqs[e], c[e], s[e]);
            }
        }
    }
    // The pairs of (lo, hi), turned by the angles, or back.
    template <bool BACK> __device__ __forceinline__ void turn(bool interleaved, float (&lo)[E], float (&hi)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float cc = c[e], ss = BACK ? -s[e] : s[e];
            if (interleaved) {
                float &a = e < E / 2 ? lo[2 * e % E] : hi[2 * e % E], &b = e < E / 2 ? lo[2 * e % E + 1] : hi[2 * e % E + 1];
                const float x = a, y = b;
                a = x * cc - y * ss, b = y * cc + x * ss;
            } else {
                const float x = lo[e], y = hi[e];
                lo[e] = x * cc - y * ss, hi[e] = y * cc + x * ss;
            }
        }
    }
};

// Sum over the lanes of a head vector, in all of them.
template <int LANES> __device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) x += __shfl_xor(x, d);
    return x;
}

template <typename T, int E> __device__ __forceinline__ void load_weight(const Rotation &r, const void *weight, int lo, int hi, float (&wl)[E], float (&wh)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
        wl[e] = !weight ? 1.f : r.weight32 ? static_cast<const float *>(weight)[lo + e] : (float)static_cast<const T *>(weight)[lo + e];
        wh[e] = !weight ? 1.f : r.weight32 ? static_cast<const float *>(weight)[hi + e] : (float)static_cast<const T *>(weight)[hi + e];
    }
}

// 1 / sqrt(mean x^2 + eps) of a head vector
template <int D, int LANES, int E> __device__ __forceinline__ float over_rms(const float (&lo)[E], const float (&hi)[E], float eps) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s = __builtin_fmaf(lo[e], lo[e], __builtin_fmaf(hi[e], hi[e], s));
    return rsqrtf(lanes_sum<LANES>(s) * (1.f / D) + eps);
}

hipError_t launch_rotary(const RotaryArgs &a, int dtype, int D, hipStream_t st);
hipError_t launch_rotary_bwd(const RotaryArgs &a, int dtype, int D, hipStream_t st);
void plan_rotary(RotaryArgs &a, int dtype, int D, bool backward);   // steps, blocks

}  // namespace seq
