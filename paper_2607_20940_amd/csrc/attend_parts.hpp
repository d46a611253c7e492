// What the attention kernels over caches share: types, the softmax's constants,
// wave helpers, the joint softmax of two results.  Included by the HIP kernels
// only.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace mssa {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr float kRescaleLog2 = 8.f;
constexpr float kNoMax = -__FLT_MAX__;       // a finite running maximum before the first score
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

// A value that all lanes share, in a scalar register.
__device__ inline uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// Sum over the wave's lanes up to this one.
__device__ inline uint32_t wave_prefix(uint32_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t u = __shfl_up(v, d);
    if (static_cast<int>(threadIdx.x & 63) >= d) v += u;
  }
  return v;
}

// Shares of this result (sum l with maximum m, base 2) and of the prior in
// the joint softmax, and the joint log sum (natural).  A NaN on either side
// makes all of it NaN.
struct Joined {
  float own, prior, lse;
};
__device__ inline Joined join(bool has_prior, float m, float l, float prior_lse) {
  const bool any = l > 0.f || l != l;  // keys were seen (a NaN sum stays a NaN)
  const float own = any ? m + __builtin_amdgcn_logf(l) : -INFINITY;
  if (!has_prior) return {any ? 1.f / l : 0.f, 0.f, any ? own * kLn2 : -INFINITY};
  const float prior = prior_lse * kLog2e;
  if (own == -INFINITY && prior == -INFINITY) return {0.f, 0.f, -INFINITY};
  const float top = fmaxf(own, prior);  // of a NaN and a number the number: the NaN's share is a NaN, and so is the sum
  const float wo = __builtin_amdgcn_exp2f(own - top), wp = __builtin_amdgcn_exp2f(prior - top), w = wo + wp;
  return {any ? wo / (l * w) : 0.f, wp / w, (top + __builtin_amdgcn_logf(w)) * kLn2};
}

// Combine over the four lanes that hold one query row (lane % 16).
template <class Op>
__device__ inline float over_row(float v, Op op) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = op(__builtin_bit_cast(float, static_cast<uint32_t>(a[0])), __builtin_bit_cast(float, static_cast<uint32_t>(a[1])));
  const uint32_t w = __builtin_bit_cast(uint32_t, v);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return op(__builtin_bit_cast(float, static_cast<uint32_t>(b[0])), __builtin_bit_cast(float, static_cast<uint32_t>(b[1])));
}

}  // namespace mssa
