// Attention over K/V caches held in MXFP4 (mssa_mx_attention).
//
// The rows that share a key head (n_q queries x group heads) are cut into
// blocks of 32 per wave; the context into tiles of 64 tokens and, where there
// are few rows, into pieces that different blocks take.  A tile's codes are
// expanded to bf16 once per block: one MXFP4 block (16 bytes of codes, one
// scale byte) per thread and pass, by the conversion instructions that take a
// scale, into LDS tiles that both products read.  e2m1 values times a power
// of two are exact in bf16.  The products are S^T = K Q^T (a lane holds one
// query row and 16 tokens of each 32) and O^T += V^T P^T, where P leaves S's
// registers without an exchange: the contraction's token order is the one
// that the lanes already hold.
//
// Softmax in base 2 on fp32 scores with a running maximum that only moves
// when a score passes it by 2^8, sums in fp32, P rounded to bf16 as a matrix
// operand.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lds_stage.hpp"
#include "lowbit_args.hpp"
#include "xcd.hpp"

namespace mssa {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr int kTile = 64;                    // tokens of a tile
constexpr int kTileElems = kTile * 128;      // 256-byte rows, also for head_dim 64
constexpr float kRescaleLog2 = 8.f;
constexpr float kNoMax = -__FLT_MAX__;       // a finite running maximum before the first score
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

__device__ inline float mx_scale(uint32_t e) {
  return __builtin_bit_cast(float, e == 255 ? 0x7fc00000u : e == 0 ? 0x00400000u : e << 23);
}

// 32 codes to bf16, in order.
__device__ inline void expand(i32x4 codes, float scale, bf16x8 (&out)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t c = static_cast<uint32_t>(codes[i]);
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2);
    const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
    out[i] = bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
  }
}

// Where a query row's q, out and lse lie.
struct RowPlace {
  int64_t q, lse;
};
__device__ inline RowPlace row_place(const MxAttnArgs& a, int b, int kvh, int r, int D) {
  const int i = r / a.group, h = kvh * a.group + (r - i * a.group);
  return {((static_cast<int64_t>(b) * a.n_q + i) * a.q_heads + h) * D,
          (static_cast<int64_t>(b) * a.q_heads + h) * a.lse_stride + i};
}

// Shares of this result (sum l with maximum m, base 2) and of the prior in
// the joint softmax, and the joint log sum (natural).
struct Joined {
  float own, prior, lse;
};
__device__ inline Joined join(const MxAttnArgs& a, float m, float l, int64_t at) {
  if (!a.prior_lse) return {l > 0.f || l != l ? 1.f / l : 0.f, 0.f, l > 0.f || l != l ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY};
  const float own = l > 0.f || l != l ? m + __builtin_amdgcn_logf(l) : -INFINITY;
  const float prior = a.prior_lse[at] * kLog2e;
  float top = fmaxf(own, prior);
  if (top == -INFINITY) return {0.f, 0.f, -INFINITY};
  const float wo = __builtin_amdgcn_exp2f(own - top), wp = __builtin_amdgcn_exp2f(prior - top), w = wo + wp;
  return {l > 0.f || l != l ? wo / (l * w) : 0.f, wp / w, (top + __builtin_amdgcn_logf(w)) * kLn2};
}

template <int D, int NW>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2))) void attn_kernel(MxAttnArgs a) {
  constexpr int KS = D / 16, DB = D / 32, kThreads = NW * 64;
  constexpr int kBlocks = kTile * DB * 2;                // MXFP4 blocks of a tile, K then V
  constexpr int NL = (kBlocks + kThreads - 1) / kThreads;  // per thread
  __shared__ __attribute__((aligned(16))) __bf16 lds[2][2][kTileElems];  // [buffer][K | V]

  const int tiles_r = (a.rows + NW * 32 - 1) / (NW * 32);
  const int L = xcd_remap(blockIdx.x, gridDim.x);
  const int rt = L % tiles_r, sp = (L / tiles_r) % a.splits, bh = L / tiles_r / a.splits;
  const int b = bh / a.kv_heads, kvh = bh - b * a.kv_heads;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = (rt * NW + wave) * 32 + n;
  const bool ok = r < a.rows;
  const RowPlace at = row_place(a, b, kvh, ok ? r : 0, D);

  int64_t len = a.kv_len ? a.kv_len[b] : a.cache_tokens;
  len = len < 0 ? 0 : len > a.cache_tokens ? a.cache_tokens : len;
  const int nt = static_cast<int>((len + kTile - 1) / kTile);
  const int t0 = static_cast<int>(static_cast<int64_t>(nt) * sp / a.splits);
  const int t1 = static_cast<int>(static_cast<int64_t>(nt) * (sp + 1) / a.splits);

  bf16x8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(a.q) + at.q + ks * 16 + hh * 8);
    qf[ks] = ok ? v : bf16x8{};
  }

  // A thread's MXFP4 blocks of a tile: block p is token (p / DB) % 64, piece
  // p % DB, of K below kBlocks / 2, else of V.
  i32x4 codes[NL];
  uint32_t se[NL];
  const int64_t base_row = static_cast<int64_t>(b) * a.cache_tokens;
  auto fetch = [&](int t) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int p = tid + i * kThreads;
      if (kBlocks % kThreads != 0 && p >= kBlocks) continue;
      const bool is_v = p >= kBlocks / 2;
      const int tok = (p / DB) % kTile, piece = p % DB;
      const int64_t token = static_cast<int64_t>(t) * kTile + tok;
      codes[i] = i32x4{};
      se[i] = 127;
      if (token < len) {
        const int64_t block = ((base_row + token) * a.kv_heads + kvh) * DB + piece;
        codes[i] = *reinterpret_cast<const i32x4*>(static_cast<const char*>(is_v ? a.vc : a.kc) + block * 16);
        se[i] = static_cast<const uint8_t*>(is_v ? a.vs : a.ks)[block];
      }
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int p = tid + i * kThreads;
      if (kBlocks % kThreads != 0 && p >= kBlocks) continue;
      const bool is_v = p >= kBlocks / 2;
      const int tok = (p / DB) % kTile, piece = p % DB;
      bf16x8 v[4];
      expand(codes[i], mx_scale(se[i]), v);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<bf16x8*>(&lds[buf][is_v ? 1 : 0][swz256(tok, piece * 32 + c * 8)]) = v[c];
    }
  };

  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x16{};
  float m = kNoMax, l = 0.f;  // running maximum (base 2), this lane's share of the sum
  const float c = a.scale_log2e;
  const int k_rd = swz256(n, hh * 8);
  const int t_row = 4 * (lane >> 5) + ((lane & 15) >> 2);
  const int t_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);

  if (t0 < t1) {
    fetch(t0);
    put(0);
  }
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    const bool more = t + 1 < t1;
    if (more) fetch(t + 1);
    const __bf16* Ks = lds[buf][0];
    const __bf16* Vs = lds[buf][1];
    f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      s[kb] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(Ks + kb * 32 * 128 + (k_rd ^ (ks * 16))),
                                                        qf[ks], s[kb], 0, 0, 0);
    }
    const int64_t left = len - static_cast<int64_t>(t) * kTile;
    if (left < kTile) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (kb * 32 + 8 * (e >> 2) + 4 * hh + (e & 3) >= left) s[kb][e] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kb][e]);
    mx = fmaxf(mx, other_half(mx)) * c;  // the scale is positive
    if (__any(mx > m + kRescaleLog2)) {
      const float mn = fmaxf(m, mx);
      const float alpha = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= alpha;
    }
    bf16x8 pb[2][2];
    float ls[2] = {0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][e], c, -m));
        ls[e & 1] += p;
        pb[kb][e >> 3][e & 7] = static_cast<__bf16>(p);
      }
    l += ls[0] + ls[1];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int cc = 0; cc < 2; ++cc)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const __bf16* r0 = Vs + (kb * 32 + cc * 16) * 128;
          const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(r0 + swz256(t_row, db * 32 + t_col)));
          const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(r0 + swz256(t_row + 8, db * 32 + t_col)));
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7),
                                                          pb[kb][cc], o[db], 0, 0, 0);
        }
    if (more) put(buf ^ 1);
    __syncthreads();
  }
  l += other_half(l);
  if (!ok) return;
  // dims 32 db + 8 j + 4 hh .. + 3 of row n
  if (a.splits > 1) {
    // [block of the piece][row][D] sums, then [..][row][2] statistics
    const int64_t slot = (static_cast<int64_t>(bh) * a.splits + sp) * a.rows + r;
    float* P = a.partial + slot * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = o[db][4 * j + i];
        *reinterpret_cast<f32x4*>(P + db * 32 + 8 * j + 4 * hh) = v;
      }
    if (hh == 0) {
      float* st = a.partial + static_cast<int64_t>(a.batch) * a.kv_heads * a.splits * a.rows * D + slot * 2;
      st[0] = m;
      st[1] = l;
    }
    return;
  }
  const Joined w = join(a, m, l, at.lse);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t d = at.q + db * 32 + 8 * j + 4 * hh;
      bf16x4 p = {}, v;
      if (a.prior_out) p = *reinterpret_cast<const bf16x4*>(static_cast<const __bf16*>(a.prior_out) + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f = o[db][4 * j + i] * w.own;
        if (a.prior_out && w.prior != 0.f) f += w.prior * static_cast<float>(p[i]);
        v[i] = static_cast<__bf16>(f);
      }
      *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.out) + d) = v;
    }
  if (a.lse && hh == 0) a.lse[at.lse] = w.lse;
}

// Join the pieces of a row: one wave per row, D / 64 dims per lane.
template <int D>
__global__ __launch_bounds__(256) void combine_kernel(MxAttnArgs a) {
  constexpr int N = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t total = static_cast<int64_t>(a.batch) * a.kv_heads * a.rows;
  if (row >= total) return;
  const int bh = static_cast<int>(row / a.rows), r = static_cast<int>(row % a.rows);
  const int b = bh / a.kv_heads, kvh = bh - b * a.kv_heads;
  const float* st = a.partial + total * a.splits * D;
  float m = kNoMax;
  for (int s = 0; s < a.splits; ++s) m = fmaxf(m, st[((static_cast<int64_t>(bh) * a.splits + s) * a.rows + r) * 2]);
  float l = 0.f, o[N] = {};
  for (int s = 0; s < a.splits; ++s) {
    const int64_t slot = (static_cast<int64_t>(bh) * a.splits + s) * a.rows + r;
    const float ls = st[slot * 2 + 1];
    const float w = ls == 0.f ? 0.f : __builtin_amdgcn_exp2f(st[slot * 2] - m);
    l = __builtin_fmaf(w, ls, l);
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = __builtin_fmaf(w, a.partial[slot * D + lane * N + i], o[i]);
  }
  const RowPlace at = row_place(a, b, kvh, r, D);
  const Joined w = join(a, m, l, at.lse);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t d = at.q + lane * N + i;
    float f = o[i] * w.own;
    if (a.prior_out && w.prior != 0.f) f += w.prior * static_cast<float>(static_cast<const __bf16*>(a.prior_out)[d]);
    static_cast<__bf16*>(a.out)[d] = static_cast<__bf16>(f);
  }
  if (a.lse && lane == 0) a.lse[at.lse] = w.lse;
}

template <int D, int NW>
hipError_t attn_go(const MxAttnArgs& a, const MxAttnPlan& plan, hipStream_t stream) {
  const int64_t blocks = plan.items * plan.splits;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((attn_kernel<D, NW>), dim3(static_cast<uint32_t>(blocks)), dim3(NW * 64), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.splits == 1) return e;
  const int64_t rows = static_cast<int64_t>(a.batch) * a.kv_heads * a.rows;
  hipLaunchKernelGGL((combine_kernel<D>), dim3(static_cast<uint32_t>((rows + 3) / 4)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <int D>
hipError_t attn_waves(const MxAttnArgs& a, const MxAttnPlan& plan, hipStream_t stream) {
  switch (plan.waves) {
    case 1: return attn_go<D, 1>(a, plan, stream);
    case 4: return attn_go<D, 4>(a, plan, stream);
    default: return attn_go<D, 8>(a, plan, stream);
  }
}

}  // namespace

MxAttnPlan plan_mx_attention(int32_t batch, int32_t n_q, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                             int64_t cache_tokens) {
  MxAttnPlan p{};
  const int64_t rows = static_cast<int64_t>(n_q) * (q_heads / kv_heads), bh = static_cast<int64_t>(batch) * kv_heads;
  p.waves = rows <= 32 ? 1 : rows <= 1024 ? 4 : 8;
  p.items = (rows + p.waves * 32 - 1) / (p.waves * 32) * bh;
  const int64_t want = 256 * (8 / p.waves), tiles = (cache_tokens + kTile - 1) / kTile;
  p.splits = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>({want / p.items, tiles / 2, 64})));
  p.workspace_bytes = p.splits > 1 ? bh * p.splits * rows * (head_dim + 2) * 4 : 0;
  return p;
}

hipError_t launch_mx_attention(const MxAttnArgs& a, const MxAttnPlan& plan, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? attn_waves<128>(a, plan, stream) : attn_waves<64>(a, plan, stream);
}

}  // namespace mssa
