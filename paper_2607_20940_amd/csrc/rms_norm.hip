// Root-mean-square norm with the residual's addition (mssa_add_rms_norm) and
// its backward.
//
// s = rnd(x + r), y = s w / sqrt(mean(s^2) + eps).  One read of x and r and
// one write of s and y is all the norm cannot do without, so a row's values
// stay in registers between the sum of squares and the scaling: TPR threads
// own a row, thread t the 8-value pieces t, t + TPR, ... of it.  A memory
// bound kernel: what counts is 16-byte loads, all of a row's in flight at
// once, and enough rows in flight.  12870 x 1536 bf16 to e4m3: 31 us, 4.5 TB/s
// (a large copy: 5.2); one row 5.7 us, most of it the call.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lowbit_args.hpp"
#include "lowbit_values.hpp"
#include "wave_ops.hpp"

namespace mssa {
namespace {

constexpr int kE4M3Max = 448;
constexpr float kTiny = 0x1p-100f;  // smallest row maximum that a scale is made from

template <class T>
__device__ inline void load8(const T* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const auto u = *reinterpret_cast<const typename Vec8<T>::type*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(u[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? static_cast<float>(p[i]) : 0.f;
  }
}

template <class T>
__device__ inline void store8(T* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    typename Vec8<T>::type u;
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = static_cast<T>(v[i]);
    *reinterpret_cast<typename Vec8<T>::type*>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = static_cast<T>(v[i]);
  }
}

// Sum of v (or maximum, of bit patterns) over a row's threads, in a fixed order.
template <int TPR>
__device__ inline float row_sum(float v, float* lds, int tid) {
  v = wave_sum(v);
  if constexpr (TPR > 64) {
    if ((tid & 63) == 0) lds[tid >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) v += lds[i];
  }
  return v;
}

template <int TPR>
__device__ inline uint32_t row_max(uint32_t v, uint32_t* lds, int tid) {
  v = wave_umax(v);
  if constexpr (TPR > 64) {
    if ((tid & 63) == 0) lds[tid >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) v = max(v, lds[i]);
  }
  return v;
}

template <class T, bool RES, bool E4, int TPR, int NV>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_kernel(NormArgs a) {
  constexpr int kThreads = TPR > 256 ? TPR : 256, kRows = kThreads / TPR;
  __shared__ float red[TPR / 64];
  __shared__ uint32_t redm[TPR / 64];
  const int tid = threadIdx.x % TPR;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / TPR;
  if (row >= a.rows) return;  // whole waves: TPR >= 64, and with TPR > 64 whole blocks
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* w = static_cast<const T*>(a.weight);

  float s[NV][8];
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) load8(x + (i * TPR + tid) * 8, a.cols - (i * TPR + tid) * 8, s[i]);
  if constexpr (RES) {
    const T* r = static_cast<const T*>(a.residual) + row * a.residual_stride;
    T* so = static_cast<T*>(a.sum) + row * a.sum_stride;
    float rv[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) load8(r + (i * TPR + tid) * 8, a.cols - (i * TPR + tid) * 8, rv[i]);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] = static_cast<float>(static_cast<T>(s[i][e] + rv[i][e]));
      store8(so + (i * TPR + tid) * 8, a.cols - (i * TPR + tid) * 8, s[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sq = __builtin_fmaf(s[i][e], s[i][e], sq);
  sq = row_sum<TPR>(sq, red, tid);
  const float rstd = 1.f / sqrtf(sq * a.inv_cols + a.eps);
  if (a.rstd && tid == 0) a.rstd[row] = rstd;

  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float wv[8];
    const int c = (i * TPR + tid) * 8;
    load8(w + c, a.cols - c, wv);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[i][e] = s[i][e] * rstd * wv[e];
    if constexpr (E4) {
      // bit patterns of magnitudes order like the magnitudes, NaN on top
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __builtin_bit_cast(uint32_t, s[i][e]) & 0x7fffffffu);
    } else {
      store8(static_cast<T*>(a.y) + row * a.y_pitch + c, a.cols - c, s[i]);
    }
  }
  if constexpr (E4) {
    top = max(row_max<TPR>(top, redm, tid), __builtin_bit_cast(uint32_t, kTiny));
    const float amax = __builtin_bit_cast(float, top);
    if (tid == 0) a.y_scale[row] = amax * (1.f / kE4M3Max);
    const float inv = kE4M3Max / amax;
    uint8_t* y = static_cast<uint8_t*>(a.y) + row * a.y_pitch;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + tid) * 8;
      if (c >= a.y_pitch) continue;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = c + e < a.cols ? s[i][e] * inv : 0.f;
      int2 u;
      u.x = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
      u.x = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], u.x, true);
      u.y = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], 0, false);
      u.y = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], u.y, true);
      *reinterpret_cast<int2*>(y + c) = u;
    }
  }
}

// Eight values as they lie in memory (zeros past n).
template <class T>
__device__ inline typename Vec8<T>::type raw8(const T* p, int n) {
  typename Vec8<T>::type v;
  if (n >= 8) return *reinterpret_cast<const typename Vec8<T>::type*>(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : static_cast<T>(0.f);
  return v;
}

// Gradients.  A block walks over rows blockIdx.x, + blocks, ... (kRows at a
// time) and keeps its share of dweight in registers; the shares are summed
// over the block's rows in LDS and over the blocks by a second launch.  A row
// is held as it lies in memory (half the registers in bf16), and the next one
// is on its way while this one's sum goes round (not with 1024 threads a row,
// which have no registers for two).  512 blocks: with 768 or 1024 the last
// rows leave CUs idle or the shares cost more (27840 x 5120 bf16, forward and
// backward: 428, 457, 435 us; 560 with a row at a time).  Rows of up to 16384
// values run at 5.0 to 5.6 TB/s; above, a row's values and its gradients' shares
// no longer fit a thread's 128 registers and spill (bf16, 24576: 2.0, 32768:
// 1.4 to 1.6 TB/s).
template <class T, bool DSUM, int TPR, int NV>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_bwd_kernel(NormBwdArgs a) {
  constexpr int kThreads = TPR > 256 ? TPR : 256, kRows = kThreads / TPR;
  constexpr bool kAhead = TPR <= 256;
  typedef typename Vec8<T>::type raw_t;
  __shared__ float red[2][TPR / 64];
  __shared__ float share[kRows > 1 ? TPR * NV * 8 : 1];
  const int tid = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  struct Row {
    raw_t s[NV], g[NV], d[DSUM ? NV : 1];
    float rstd;
  };
  raw_t w[NV];
  auto at = [&](int i) { return (i * TPR + tid) * 8; };
#pragma unroll
  for (int i = 0; i < NV; ++i) w[i] = raw8(static_cast<const T*>(a.weight) + at(i), a.cols - at(i));
  auto fetch = [&](Row& r, int64_t row) {
    r.rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = at(i), n = a.cols - c;
      r.s[i] = raw8(static_cast<const T*>(a.sum) + row * a.sum_stride + c, n);
      r.g[i] = raw8(static_cast<const T*>(a.dy) + row * a.cols + c, n);
      if constexpr (DSUM) r.d[i] = raw8(static_cast<const T*>(a.dsum) + row * a.cols + c, n);
    }
  };
  float dw[NV][8] = {};
  const int64_t step = static_cast<int64_t>(a.blocks) * kRows;
  int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + sub;
  Row cur, next;
  if (row < a.rows) fetch(cur, row);
  for (int it = 0; row < a.rows; row += step, ++it) {
    const bool more = row + step < a.rows;
    if (kAhead && more) fetch(next, row + step);
    float inner = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float s = static_cast<float>(cur.s[i][e]), g = static_cast<float>(cur.g[i][e]);
        dw[i][e] = __builtin_fmaf(g * cur.rstd, s, dw[i][e]);
        inner = __builtin_fmaf(g * static_cast<float>(w[i][e]), s, inner);
      }
    // with more than one wave a row, alternating slots save a second barrier
    inner = row_sum<TPR>(inner, red[it & 1], tid) * a.inv_cols;
    const float k = cur.rstd * cur.rstd * inner;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = at(i);
      float d[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float g = static_cast<float>(cur.g[i][e]) * static_cast<float>(w[i][e]);
        d[e] = cur.rstd * (g - static_cast<float>(cur.s[i][e]) * k);
        if constexpr (DSUM) d[e] += static_cast<float>(cur.d[i][e]);
      }
      store8(static_cast<T*>(a.dx) + row * a.cols + c, a.cols - c, d);
    }
    if (more) {
      if constexpr (kAhead)
        cur = next;
      else
        fetch(cur, row + step);
    }
  }
  float* out = a.blocks > 1 ? a.partial + static_cast<int64_t>(blockIdx.x) * a.cols : a.dweight;
  if constexpr (kRows > 1) {
    for (int r = 0; r < kRows; ++r) {
      if (sub == r) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float& t = share[(i * 8 + e) * TPR + tid];
            t = r == 0 ? dw[i][e] : t + dw[i][e];
          }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < a.cols; c += kThreads) {
      const int piece = c / 8, i = piece / TPR, t = piece % TPR;
      out[c] = share[(i * 8 + c % 8) * TPR + t];
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) store8(out + (i * TPR + tid) * 8, a.cols - (i * TPR + tid) * 8, dw[i]);
  }
}

// dweight = sum of the blocks' shares: 32 threads a column, each every 32nd
// share with many of them on their way, joined in order.
__global__ __launch_bounds__(1024) void norm_dweight_kernel(NormBwdArgs a) {
  __shared__ float part[32][33];
  const int x = threadIdx.x % 32, g = threadIdx.x / 32, c = blockIdx.x * 32 + x;
  float s = 0.f;
  if (c < a.cols) {
    const float* p = a.partial + c;
#pragma unroll 16
    for (int b = g; b < a.blocks; b += 32) s += p[static_cast<int64_t>(b) * a.cols];
  }
  part[g][x] = s;
  __syncthreads();
  if (g == 0 && c < a.cols) {
#pragma unroll
    for (int i = 1; i < 32; ++i) s += part[i][x];
    a.dweight[c] = s;
  }
}

template <class T, bool RES, bool E4, int TPR, int NV>
hipError_t norm_go(const NormArgs& a, hipStream_t stream) {
  constexpr int kThreads = TPR > 256 ? TPR : 256, kRows = kThreads / TPR;
  const int64_t blocks = (a.rows + kRows - 1) / kRows;
  if (blocks * kThreads > kLaunchThreads) return hipErrorInvalidValue;
  hipLaunchKernelGGL((norm_kernel<T, RES, E4, TPR, NV>), dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

template <class T, bool RES, bool E4, int TPR>
hipError_t norm_nv(const NormArgs& a, int nv, hipStream_t stream) {
  switch (nv) {
    case 1: return norm_go<T, RES, E4, TPR, 1>(a, stream);
    case 2: return norm_go<T, RES, E4, TPR, 2>(a, stream);
    case 3: return norm_go<T, RES, E4, TPR, 3>(a, stream);
    default: return norm_go<T, RES, E4, TPR, 4>(a, stream);
  }
}

template <class T, bool RES, bool E4>
hipError_t norm_tpr(const NormArgs& a, hipStream_t stream) {
  const NormRowShape s = norm_row_shape(E4 ? a.y_pitch : a.cols);
  if (s.tpr == 64) return norm_nv<T, RES, E4, 64>(a, s.nv, stream);
  if (s.tpr == 256) return norm_nv<T, RES, E4, 256>(a, s.nv, stream);
  return norm_nv<T, RES, E4, 1024>(a, s.nv, stream);
}

template <class T>
hipError_t norm_type(const NormArgs& a, bool e4m3, hipStream_t stream) {
  if (a.residual) return e4m3 ? norm_tpr<T, true, true>(a, stream) : norm_tpr<T, true, false>(a, stream);
  return e4m3 ? norm_tpr<T, false, true>(a, stream) : norm_tpr<T, false, false>(a, stream);
}

template <class T, bool DSUM, int TPR, int NV>
hipError_t bwd_go(const NormBwdArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((norm_bwd_kernel<T, DSUM, TPR, NV>), dim3(a.blocks), dim3(TPR > 256 ? TPR : 256), 0, stream, a);
  return hipGetLastError();
}

template <class T, bool DSUM, int TPR>
hipError_t bwd_nv(const NormBwdArgs& a, int nv, hipStream_t stream) {
  switch (nv) {
    case 1: return bwd_go<T, DSUM, TPR, 1>(a, stream);
    case 2: return bwd_go<T, DSUM, TPR, 2>(a, stream);
    case 3: return bwd_go<T, DSUM, TPR, 3>(a, stream);
    default: return bwd_go<T, DSUM, TPR, 4>(a, stream);
  }
}

template <class T, bool DSUM>
hipError_t bwd_tpr(const NormBwdArgs& a, hipStream_t stream) {
  const NormRowShape s = norm_row_shape(a.cols);
  if (s.tpr == 64) return bwd_nv<T, DSUM, 64>(a, s.nv, stream);
  if (s.tpr == 256) return bwd_nv<T, DSUM, 256>(a, s.nv, stream);
  return bwd_nv<T, DSUM, 1024>(a, s.nv, stream);
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, bool bf16, bool e4m3, hipStream_t stream) {
  return bf16 ? norm_type<__bf16>(a, e4m3, stream) : norm_type<float>(a, e4m3, stream);
}

hipError_t launch_norm_bwd(const NormBwdArgs& a, bool bf16, hipStream_t stream) {
  if (a.blocks > 0) {
    hipError_t e;
    if (bf16)
      e = a.dsum ? bwd_tpr<__bf16, true>(a, stream) : bwd_tpr<__bf16, false>(a, stream);
    else
      e = a.dsum ? bwd_tpr<float, true>(a, stream) : bwd_tpr<float, false>(a, stream);
    if (e != hipSuccess || a.blocks == 1) return e;
  }
  hipLaunchKernelGGL(norm_dweight_kernel, dim3((a.cols + 31) / 32), dim3(1024), 0, stream, a);
  return hipGetLastError();
}

}  // namespace mssa
