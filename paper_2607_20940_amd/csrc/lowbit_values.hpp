// Values of the low-bit formats in registers, and eight neighbouring values of
// a row as they lie in memory.  Included by the HIP kernels only.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace mssa {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A scale byte as the conversion instructions take it.  They read the float's
// exponent field alone, as the format's scale byte: 0 is 2^-127, 255 makes NaNs.
__device__ inline float mx_scale(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

// Eight e2m1 codes under one scale to bf16, in order (exact down to bf16's
// smallest number).
__device__ inline bf16x8 expand_e2m1(uint32_t codes, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight e4m3 codes to bf16, in order (exact).
__device__ inline bf16x8 expand_e4m3(uint32_t lo, uint32_t hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight consecutive values, aligned to the element only (rows cut out of a
// wider tensor, odd widths): global accesses need no more.
template <class T>
struct Vec8;
template <>
struct Vec8<__bf16> {
  typedef __bf16 type __attribute__((ext_vector_type(8), aligned(2)));
};
template <>
struct Vec8<float> {
  typedef float type __attribute__((ext_vector_type(8), aligned(4)));
};

}  // namespace mssa
