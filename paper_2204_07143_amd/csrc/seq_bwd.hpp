// What the two sides of the backward pass share.
#pragma once

#include "lds_attr.hpp"
#include "seq_common.hpp"

namespace seq {

template <typename T> constexpr bool kScaled = __is_same(T, f16_t);
template <typename T> constexpr float kRaise = kScaled<T> ? 8.f : 0.f;   // weights are formed times 2^kRaise
constexpr int kNothing = -1000;   // power of two of a tile of zeros

__device__ __forceinline__ int power_of(float most) { return most > 0.f ? min(16, __builtin_amdgcn_frexp_expf(most)) : kNothing; }   // (infinite: 16)
__device__ __forceinline__ float two_to(int e) { return __builtin_amdgcn_ldexpf(1.f, e); }

template <typename T> constexpr int kBlocks = sizeof(T) == 2 ? 2 : 1;   // blocks of 16 queries, or keys, that a wave keeps

}  // namespace seq
