// Reductions over the 64 lanes of a wave by lane permutations, in a fixed
// order.  Included by the HIP kernels only.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace mssa {

// Value of the lane that DPP control CTRL names (all of them permutations).
template <int CTRL>
__device__ inline uint32_t dpp(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, true));
}

constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E;       // quad_perm [1,0,3,2], [2,3,0,1]
constexpr int kDppHalfMirror = 0x141, kDppMirror = 0x140;  // lane 7 - i of eight, 15 - i of sixteen

// Combine over the wave: every lane gets the result.  After the exchanges
// with 1 and 2 all four lanes of a quad agree, so the mirrors act as
// exchanges with 4 and 8; permlane16/32_swap finish.
template <class Op>
__device__ inline uint32_t wave_reduce(uint32_t v, Op op) {
  v = op(v, dpp<kDppXor1>(v));
  v = op(v, dpp<kDppXor2>(v));
  v = op(v, dpp<kDppHalfMirror>(v));
  v = op(v, dpp<kDppMirror>(v));
  auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = op(a[0], a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return op(b[0], b[1]);
}

__device__ inline float wave_sum(float v) {
  return __builtin_bit_cast(float, wave_reduce(__builtin_bit_cast(uint32_t, v), [](uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
  }));
}

__device__ inline float wave_fmax(float v) {
  return __builtin_bit_cast(float, wave_reduce(__builtin_bit_cast(uint32_t, v), [](uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
  }));
}

__device__ inline uint32_t wave_umax(uint32_t v) {
  return wave_reduce(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

}  // namespace mssa
