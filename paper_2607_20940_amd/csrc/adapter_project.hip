// Shared projection with a low-rank adapter per segment of rows
// (mssa_adapter_project): y = x W^T + bias + scale (x A^T) B^T.
//
// Two launches: the low-rank factor u = scale (x A^T) of every row, rounded to
// bf16 (an operand of the second product; it adds up to 2^-9 of the adapter's
// share, which fp32 operands would spare at a sixteenth of the rate), then the
// product, whose tiles add u B^T of the segments that they hold to the sums in
// their registers before the one rounding of the output.  A tile's rows can belong
// to several segments: each one's product is made apart and added to its own
// rows only, so that an infinity or a NaN of one adapter stays with its rows.
#include <hip/hip_runtime.h>

#include "lds_stage.hpp"
#include "lowbit_values.hpp"
#include "paged_args.hpp"

namespace mssa {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;

// Eight neighbouring values of a row, zeros from the n-th on (none where n <= 0).
__device__ inline bf16x8 eight(const __bf16* p, int n) {
  if (n >= 8) return *reinterpret_cast<const Vec8<__bf16>::type*>(p);
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : static_cast<__bf16>(0.f);
  return v;
}

// Rows [first, end) of segment s and its adapter, -1 for none.
struct Segment {
  int32_t first, end, adapter;
};
__device__ inline Segment segment(const AdapterArgs& a, int32_t s) {
  const ChunkRows c = ChunkRows::of(a.segment_begin, s, 0, a.M);
  const int32_t j = a.adapter[s];
  return {c.first, c.end, j >= 0 && j < a.adapters ? j : -1};
}

// The first segment that ends behind row `row` (segments where none does), for
// a wave: segments are probed 64 at a time.
__device__ inline int32_t first_segment(const AdapterArgs& a, int32_t row) {
  const int lane = threadIdx.x & 63;
  int32_t lo = 0, n = a.segments;
  while (n > 0) {
    const int32_t step = (n + 63) / 64, at = lo + lane * step;
    // a probe's segment ends at or before the row: so do those before it
    const uint64_t gone = __ballot(lane * step < n && a.segment_begin[(at < a.segments ? at : 0) + 1] <= row);
    if (!gone) return lo;
    const int last = 63 - __builtin_clzll(gone);
    const int32_t skip = last * step + 1;
    n = n - skip < step - 1 ? n - skip : step - 1;
    lo += skip;
  }
  return lo;
}

// The low-rank factor of 32 rows of one segment and one part: a wave takes
// every fourth 16 values of the contraction, 32 ranks at a time, and the four
// sums meet in LDS.
__global__ __launch_bounds__(kThreads) void low_kernel(AdapterArgs a) {
  __shared__ float sums[4][32 * 33];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = blockIdx.x % a.parts;
  int32_t tile = blockIdx.x / a.parts;
  // the segment that the tile belongs to, and the tile's place in it
  int32_t s = -1;
  for (int32_t c = 0; c < a.segments && s < 0; c += 64) {
    int32_t mine = 0;
    if (c + lane < a.segments) {
      const Segment g = segment(a, c + lane);
      mine = (g.end - g.first + kLowRows - 1) / kLowRows;
    }
    int32_t pre = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int32_t u = __shfl_up(pre, d);
      if (lane >= d) pre += u;
    }
    const uint64_t past = __ballot(pre > tile);
    if (past) {
      const int i = __builtin_ctzll(past);
      s = c + i;
      tile -= __shfl(pre, i) - __shfl(mine, i);
    } else {
      tile -= __shfl(pre, 63);
    }
  }
  if (s < 0) return;
  s = __builtin_amdgcn_readfirstlane(s);
  tile = __builtin_amdgcn_readfirstlane(tile);
  const Segment g = segment(a, s);
  const int32_t row0 = g.first + tile * kLowRows;
  if (g.adapter < 0 || tile < 0 || row0 >= g.end) return;
  const int32_t row = row0 + n32;
  const bool ok = row < g.end;
  const __bf16* x = static_cast<const __bf16*>(a.x) + static_cast<int64_t>(ok ? row : row0) * a.x_stride;
  const __bf16* A = static_cast<const __bf16*>(a.a) + (static_cast<int64_t>(g.adapter) * a.parts + part) * a.rank * a.K;
  const float scale = a.scale ? a.scale[g.adapter] : 1.f;
  for (int r0 = 0; r0 < a.rank; r0 += 32) {
    const int r = r0 + n32;
    const __bf16* ar = A + static_cast<int64_t>(r < a.rank ? r : 0) * a.K;
    f32x16 acc = f32x16{};
#pragma unroll 4
    for (int k = wave * 16; k < a.K; k += 64) {
      const int at = k + hh * 8;
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(eight(ar + at, a.K - at), eight(x + at, a.K - at), acc, 0, 0, 0);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 16; ++e) sums[wave][n32 * 33 + 8 * (e >> 2) + 4 * hh + (e & 3)] = acc[e];
    __syncthreads();
    __bf16* out = static_cast<__bf16*>(a.low);
    for (int i = tid; i < 32 * 32; i += kThreads) {
      const int q = i >> 5, rr = i & 31, at = q * 33 + rr;
      if (row0 + q >= g.end || r0 + rr >= a.low_rank) continue;
      const float u = (sums[0][at] + sums[1][at]) + (sums[2][at] + sums[3][at]);
      out[(static_cast<int64_t>(row0 + q) * a.parts + part) * a.low_rank + r0 + rr] =
          static_cast<__bf16>(r0 + rr < a.rank ? u * scale : 0.f);
    }
  }
}

// The product in 128 x 128 tiles, a wave 64 x 64 of it (A = W rows, B = X rows,
// so that a lane holds one row's sums), the contraction in 32-deep stages
// through registers and LDS.  Any sizes, strides and alignments.
constexpr int kGM = 128, kGN = 128, kGK = 32, kGStr = kGK + 8;  // LDS row stride: conflict-free 16-byte reads

__global__ __launch_bounds__(kThreads) void any_kernel(AdapterArgs a) {
  __shared__ __attribute__((aligned(16))) __bf16 lds[2][2][kGM * kGStr];  // [stage][X | W]
  const int tiles_m = (a.M + kGM - 1) / kGM;
  const int tm = blockIdx.x % tiles_m, tn = blockIdx.x / tiles_m;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave & 1, wn = wave >> 1;
  const int n32 = lane & 31, hh = lane >> 5;
  const int32_t m0 = tm * kGM, m1 = min(m0 + kGM, a.M), f0 = tn * kGN, f1 = min(f0 + kGN, a.N);

  // Stage loads: 128 rows x 4 pieces of 8 values per matrix, 2 pieces per thread.
  const int lr = tid >> 2, lc = (tid & 3) * 8;
  bf16x8 px[2], pw[2];
  auto load = [&](const __bf16* x, int64_t xs, int32_t xa, int32_t xb, const __bf16* w, int64_t ws, int32_t wa, int32_t wb, int left) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int32_t xr = m0 + lr + i * 64, wr = f0 + lr + i * 64;
      px[i] = xr >= xa && xr < xb ? eight(x + xr * xs + lc, left - lc) : bf16x8{};
      pw[i] = wr >= wa && wr < wb ? eight(w + wr * ws + lc, left - lc) : bf16x8{};
    }
  };
  auto store = [&](int s) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = lr + i * 64;
      *reinterpret_cast<bf16x8*>(&lds[s][0][r * kGStr + lc]) = px[i];
      *reinterpret_cast<bf16x8*>(&lds[s][1][r * kGStr + lc]) = pw[i];
    }
  };
  auto operand = [&](int s, int which, int block, int ks) {
    return *reinterpret_cast<const bf16x8*>(&lds[s][which][((which ? wn : wm) * 64 + block * 32 + n32) * kGStr + ks * 16 + hh * 8]);
  };

  f32x16 acc[2][2];
#pragma unroll
  for (int rb = 0; rb < 2; ++rb)
#pragma unroll
    for (int cb = 0; cb < 2; ++cb) acc[rb][cb] = f32x16{};

  const __bf16* X = static_cast<const __bf16*>(a.x);
  const __bf16* W = static_cast<const __bf16*>(a.w);
  const int nst = (a.K + kGK - 1) / kGK;
  auto load_stage = [&](int st) { load(X + st * kGK, a.x_stride, m0, m1, W + st * kGK, a.K, f0, f1, a.K - st * kGK); };
  load_stage(0);
  store(0);
  __syncthreads();
  for (int st = 0; st < nst; ++st) {
    if (st + 1 < nst) load_stage(st + 1);
#pragma unroll
    for (int ks = 0; ks < kGK / 16; ++ks)
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int cb = 0; cb < 2; ++cb)
          acc[rb][cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(st & 1, 1, cb, ks), operand(st & 1, 0, rb, ks), acc[rb][cb], 0, 0, 0);
    if (st + 1 < nst) store((st + 1) & 1);
    __syncthreads();
  }

  // Element e of acc[rb][cb]: row wm 64 + rb 32 + n32, feature wn 64 + cb 32 + 8 (e / 4) + 4 hh + e % 4 of the tile.
  const int p0 = f0 / a.split, p1 = (f1 - 1) / a.split;
  for (int32_t s = __builtin_amdgcn_readfirstlane(first_segment(a, m0)); s < a.segments; ++s) {
    const Segment g = segment(a, s);
    if (g.first >= m1) break;
    if (g.adapter < 0 || g.first >= g.end) continue;
    for (int p = p0; p <= p1; ++p) {
      const __bf16* u = static_cast<const __bf16*>(a.low) + p * a.low_rank;
      const __bf16* B = static_cast<const __bf16*>(a.b) + static_cast<int64_t>(g.adapter) * a.N * a.rank;
      const int32_t fa = p * a.split, fb = fa + a.split;
      for (int r0 = 0; r0 < a.rank; r0 += kGK) {
        load(u + r0, static_cast<int64_t>(a.parts) * a.low_rank, g.first, g.end, B + r0, a.rank, fa, min(fb, f1), a.rank - r0);
        store(0);
        __syncthreads();
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
          const int32_t row = m0 + wm * 64 + rb * 32 + n32;
          const bool mine = row >= g.first && row < g.end;
#pragma unroll
          for (int cb = 0; cb < 2; ++cb) {
            f32x16 add = f32x16{};
#pragma unroll
            for (int ks = 0; ks < kGK / 16; ++ks)
              add = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(0, 1, cb, ks), operand(0, 0, rb, ks), add, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int32_t f = f0 + wn * 64 + cb * 32 + 8 * (e >> 2) + 4 * hh + (e & 3);
              acc[rb][cb][e] += mine && f >= fa && f < fb ? add[e] : 0.f;
            }
          }
        }
        __syncthreads();
      }
    }
  }

  const __bf16* bias = static_cast<const __bf16*>(a.bias);
#pragma unroll
  for (int rb = 0; rb < 2; ++rb) {
    const int32_t row = m0 + wm * 64 + rb * 32 + n32;
    if (row >= m1) continue;
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int32_t f = f0 + wn * 64 + cb * 32 + 8 * (e >> 2) + 4 * hh + (e & 3);
        if (f >= f1) continue;
        const int part = f / a.split;
        const float v = (acc[rb][cb][e] + (bias ? static_cast<float>(bias[f]) : 0.f)) * (part == 0 ? a.part0_scale : 1.f);
        static_cast<__bf16*>(a.y[part])[static_cast<int64_t>(row) * a.split + (f - part * a.split)] = static_cast<__bf16>(v);
      }
  }
}

}  // namespace

hipError_t launch_adapter_project(const AdapterArgs& a, const AdapterPlan& plan, hipStream_t stream) {
  if (plan.low_blocks) {
    hipLaunchKernelGGL(low_kernel, dim3(static_cast<uint32_t>(plan.low_blocks)), dim3(kThreads), 0, stream, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(any_kernel, dim3(static_cast<uint32_t>(plan.blocks)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace mssa
