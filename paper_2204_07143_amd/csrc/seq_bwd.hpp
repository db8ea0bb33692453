// What the two sides of the backward pass share.
#pragma once

#include "lds_attr.hpp"
#include "seq_common.hpp"

namespace seq {

template <typename T> constexpr bool kScaled = __is_same(T, f16_t);
template <typename T> constexpr float kRaise = kScaled<T> ? 10.f : 0.f;   // weights are formed times 2^kRaise
constexpr int kNothing = -1000;   // power of two of a tile of zeros

__device__ __forceinline__ int power_of(float most, int highest) { return most > 0.f ? min(highest, __builtin_amdgcn_frexp_expf(most)) : kNothing; }   // (infinite: highest)
constexpr int kMostDout = 16, kMostValues = 23;   // fp16, and 128 of them
// The power of two that dS is raised by on the scale of |dout|, 2^power: with 2^e above every sum |v_j| that its rows see, |dP| and |delta| are below 2^(power + e); delta is the
// weights' mean of dP, so |P (dP - delta)| <= 2 P (1 - P) max |dP| is below half of that, and raised below 2^14.  Flat rows over n keys, dS of 1 / n of it, keep
// fp16's eleven digits to n of about 2^20, and one of them less for each power of two beyond.
__device__ __forceinline__ int raise_of(int e) { return 15 - (e == kNothing ? 0 : e); }
__device__ __forceinline__ float two_to(int e) { return __builtin_amdgcn_ldexpf(1.f, e); }

// Parts' sums [parts, (a and then b), B * heads, L, D], added in order into a and b (nullable); a thread per four channels.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void join_kernel(const float *sums, int parts, int heads, int L, int64_t planes, View a, View b, int64_t each) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= each) return;
    const int d = (int)(i % (D / 4)) * 4;
    const int64_t row = i / (D / 4), plane = row / L;
    f32x4 x{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < parts; ++s) x += *reinterpret_cast<const f32x4 *>(sums + (int64_t)s * each * 4 + i * 4);
    const View &to = plane < planes ? a : b;
    const int at = (int)(plane < planes ? plane : plane - planes);
    Tile<T, D>::store4(const_cast<char *>(to.at) + at / heads * to.b + at % heads * to.h + row % L * to.row + d * (int)sizeof(T), x);
}
template <typename T, int D> hipError_t join(const float *sums, int parts, int B, int heads, int L, const View &a, const View *b, hipStream_t st) {
    const int64_t planes = (int64_t)B * heads, each = planes * L * (b ? 2 : 1) * (D / 4), blocks = (each + kThreads - 1) / kThreads;
    if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
    join_kernel<T, D><<<(unsigned)blocks, kThreads, 0, st>>>(sums, parts, heads, L, planes, a, b ? *b : a, each);
    return hipGetLastError();
}

}  // namespace seq
