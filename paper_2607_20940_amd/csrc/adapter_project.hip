// Shared projection with a low-rank adapter per segment of rows
// (mssa_adapter_project): y = x W^T + bias + scale (x A^T) B^T.
//
// Two launches: the low-rank factor u = scale (x A^T) of every row, rounded to
// bf16 (an operand of the second product; it adds up to 2^-8 of the adapter's
// share, which fp32 operands would spare at a sixteenth of the rate), then the
// product, whose tiles add u B^T of the segments that they hold to the sums in
// their registers before the one rounding of the output.  A tile's rows can belong
// to several segments: each one's product is made apart and added to its own
// rows only, so that an infinity or a NaN of one adapter stays with its rows.
#include <hip/hip_runtime.h>

#include "kernel_args.hpp"
#include "lds_stage.hpp"
#include "lowbit_values.hpp"
#include "paged_args.hpp"
#include "xcd.hpp"
#include "zero_row.hpp"

namespace mssa {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
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

// Eight neighbouring values of an aligned tensor from any of them on.  Loads that are
// no multiples of 4 bytes apart take several times as long: the 16 bytes from the even
// place before and the last value apart, joined once both are there (16 x 577 ->
// 1728, rank 16: 15.7 us for both kernels, 33.7 with one load at any place).
struct Eight {
  uint32_t v __attribute__((ext_vector_type(4)));
  uint32_t last, shift;
  __device__ static Eight at(const __bf16* p) {
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t odd = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p) >> 1) & 1;
    return {*reinterpret_cast<const words*>(p - odd), *reinterpret_cast<const uint16_t*>(p + 7), odd * 16};
  }
  __device__ bf16x8 values() const {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(bf16x8, words{__builtin_amdgcn_alignbit(v[1], v[0], shift), __builtin_amdgcn_alignbit(v[2], v[1], shift),
                                            __builtin_amdgcn_alignbit(v[3], v[2], shift), __builtin_amdgcn_alignbit(last, v[3], shift)});
  }
};

// The values of v from the (8 - n)-th on, then zeros: where a row's last eight values
// were read because only n were left, those.
__device__ inline bf16x8 last_of(bf16x8 v, int n) {
  typedef unsigned __int128 u128;
  const u128 bits = __builtin_bit_cast(u128, v);
  return __builtin_bit_cast(bf16x8, n <= 0 ? u128{0} : n >= 8 ? bits : bits >> (16 * (8 - n)));
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

// The segment that tile `tile` of `rows` rows belongs to (every segment has tiles
// of its own, one after the other) and the tile's first row; adapter -1 where
// the tile has nothing to do.
struct LowTile {
  int32_t first, end, adapter;
};
__device__ inline LowTile low_tile(const AdapterArgs& a, int32_t tile, int32_t rows) {
  const int lane = threadIdx.x & 63;
  for (int32_t c = 0; c < a.segments; c += 64) {
    Segment g{0, 0, -1};
    if (c + lane < a.segments) g = segment(a, c + lane);
    const int32_t mine = (g.end - g.first + rows - 1) / rows;
    int32_t pre = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int32_t u = __shfl_up(pre, d);
      if (lane >= d) pre += u;
    }
    const uint64_t past = __ballot(pre > tile);
    if (past) {
      const int i = __builtin_ctzll(past);
      const int32_t at = tile - (__shfl(pre, i) - __shfl(mine, i)), first = __shfl(g.first, i) + at * rows, end = __shfl(g.end, i);
      const bool ok = at >= 0 && first < end;
      return {__builtin_amdgcn_readfirstlane(first), __builtin_amdgcn_readfirstlane(end),
              __builtin_amdgcn_readfirstlane(ok ? __shfl(g.adapter, i) : -1)};
    }
    tile -= __shfl(pre, 63);
  }
  return {0, 0, -1};
}

// The low-rank factors of 16 rows of one segment, 16 of the parts' rank columns,
// which stand behind one another.  The block's 16 waves share out the
// contraction, 320 values each on their way at once, and their sums meet in LDS,
// in a fixed order.  kWhole: rows of whole, aligned 16-byte chunks; else rows of at
// least 8 values that begin anywhere, whose last eight are read where fewer than
// eight are left and put in place afterwards (no load waits for a branch).
// Bound by latency: a look-up of the segment, one round of loads, a meeting.  16 rows
// of 8 adapters, 5120 values, 48 columns: 9 us.
constexpr int kLowWaves = 16;

template <bool kWhole>
__global__ __launch_bounds__(kLowWaves * 64) void low_kernel(AdapterArgs a) {
  constexpr int kUnroll = kWhole ? 10 : 7;
  __shared__ float sums[kLowWaves][16 * 17];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const LowTile g = low_tile(a, blockIdx.x, kLowRows);
  if (g.adapter < 0) return;
  const int32_t row = min(g.first + n, g.end - 1);
  const int cols = a.parts * a.low_rank, c0 = blockIdx.y * 16;  // columns of one part
  const int part = c0 / a.low_rank, r = min(c0 + n - part * a.low_rank, a.rank - 1);
  const __bf16* x = static_cast<const __bf16*>(a.x) + static_cast<int64_t>(row) * a.x_stride + q * 8;
  const __bf16* A = static_cast<const __bf16*>(a.a) + ((static_cast<int64_t>(g.adapter) * a.parts + part) * a.rank + r) * a.K + q * 8;
  auto get = [&](const __bf16* p, int k) {
    if constexpr (kWhole)
      return k + q * 8 < a.K ? *reinterpret_cast<const bf16x8*>(p + k) : bf16x8{};
    else
      return Eight::at(p + min(k, a.K - 8 - q * 8));
  };
  auto values = [&](const auto& v, int s) -> bf16x8 {
    if constexpr (kWhole)
      return v;
    else
      return s * 32 + 32 > a.K ? last_of(v.values(), a.K - s * 32 - q * 8) : v.values();
  };
  f32x4 acc = f32x4{};
  const int steps = (a.K + 31) / 32, each = (steps + kLowWaves - 1) / kLowWaves, s0 = wave * each, s1 = min(s0 + each, steps);
#pragma unroll 1
  for (int s = s0; s < s1; s += kUnroll) {
    decltype(get(x, 0)) xv[kUnroll], av[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int k = min(s + u, s1 - 1) * 32;
      av[u] = get(A, k);
      xv[u] = get(x, k);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (s + u < s1) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values(av[u], s + u), values(xv[u], s + u), acc, 0, 0, 0);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sums[wave][n * 17 + 4 * q + e] = acc[e];
  __syncthreads();
  const int at = tid >> 4, c = tid & 15;
  if (tid >= 256 || g.first + at >= g.end) return;
  float u = 0.f;
#pragma unroll
  for (int w = 0; w < kLowWaves; ++w) u += sums[w][at * 17 + c];
  const float scale = a.scale ? a.scale[g.adapter] : 1.f;
  // ranks are rounded up with zeros
  static_cast<__bf16*>(a.low)[static_cast<int64_t>(g.first + at) * cols + c0 + c] =
      static_cast<__bf16>(c0 + c - part * a.low_rank < a.rank ? u * scale : 0.f);
}

// The same for many rows: 64 rows of one segment and NB x 32 rank columns a
// block, two by two waves of 32 rows and NB x 16 columns.  The contraction comes
// in 64-deep stages of 128-byte rows through four LDS buffers, three of them on
// their way.  Bound by the latency of that chain and by X's bytes: 12870 rows of
// 1536, 96 columns, 20 us; 27840 of 5120, 192 columns, 130 us: 285 MB, which two
// blocks each read.
constexpr int kLowTileRows = kLowManyRows, kLowStages = 4;

template <int NB>
__global__ __launch_bounds__(256) void low_tile_kernel(AdapterArgs a) {
  constexpr int BN = NB * 32, kX = kLowTileRows * 128, kStage = kX + BN * 128, kMine = 2 + NB;  // kMine: a wave's transfers of a stage
  __shared__ __attribute__((aligned(16))) char lds[kLowStages][kStage];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
  const int cols = a.parts * a.low_rank, across = (cols + BN - 1) / BN;
  const int at = xcd_remap(blockIdx.x, gridDim.x), c0 = at % across * BN;
  const LowTile g = low_tile(a, at / across, kLowTileRows);
  if (g.adapter < 0) return;
  const int32_t rows = min(g.end - g.first, kLowTileRows);

  // A transfer: rows 8 i + lane / 8, physical chunk lane % 8 holding logical chunk unswz128(row, lane % 8).
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&lds[0][0]));
  const uint32_t xrb = static_cast<uint32_t>(a.x_stride) * 2;
  const __bf16* X = static_cast<const __bf16*>(a.x) + static_cast<int64_t>(g.first) * a.x_stride;
  const __bf16* A = static_cast<const __bf16*>(a.a) + static_cast<int64_t>(g.adapter) * a.parts * a.rank * a.K;
  uint32_t xo[2];
  int xc[2], ac[NB];     // logical chunks
  const __bf16* ap[NB];  // columns past the ranks are read as others' and written as zeros
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (wave * 2 + i) * 8 + (lane >> 3);
    xc[i] = unswz128(row, lane & 7);
    xo[i] = row * xrb + xc[i] * 16;
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int row = (wave * NB + i) * 8 + (lane >> 3), c = min(c0 + row, cols - 1), part = c / a.low_rank;
    ac[i] = unswz128(row, lane & 7);
    ap[i] = A + (static_cast<int64_t>(part) * a.rank + min(c - part * a.low_rank, a.rank - 1)) * a.K + ac[i] * 8;
  }
  auto put = [&](int st) {
    const int left = min(a.K - st * 64, 64);  // a multiple of 8; zeros past it
    const i32x4 rx = rsrc_of(X + st * 64, static_cast<uint32_t>(rows - 1) * xrb + left * 2);
    const uint32_t base = lds0 + st % kLowStages * kStage;
#pragma unroll
    for (int i = 0; i < 2; ++i) dma16(rx, xc[i] * 8 < left ? xo[i] : kPastEnd, __builtin_amdgcn_readfirstlane(base + (wave * 2 + i) * 1024));
#pragma unroll
    for (int i = 0; i < NB; ++i) gdma16(ac[i] * 8 < left ? static_cast<const void*>(ap[i] + st * 64) : zero_row, __builtin_amdgcn_readfirstlane(base + kX + (wave * NB + i) * 1024));
  };
  f32x4 acc[2][NB];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[m][b] = f32x4{};
  const int nst = (a.K + 63) / 64;
  for (int st = 0; st < kLowStages - 1 && st < nst; ++st) put(st);
  for (int st = 0; st < nst; ++st) {
    wait_for_stage<kLowStages - 2, kMine>(nst - 1 - st);
    // the stage before has been read by all: its buffer is filled next
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (st + kLowStages - 1 < nst) put(st + kLowStages - 1);
    const char* Xs = lds[st % kLowStages] + wm * 32 * 128;
    const char* As = lds[st % kLowStages] + kX + wn * NB * 16 * 128;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8 xv[2], av[NB];
#pragma unroll
      for (int m = 0; m < 2; ++m) xv[m] = *reinterpret_cast<const bf16x8*>(Xs + swz128(m * 16 + n, ks * 32 + q * 8) * 2);
#pragma unroll
      for (int b = 0; b < NB; ++b) av[b] = *reinterpret_cast<const bf16x8*>(As + swz128(b * 16 + n, ks * 32 + q * 8) * 2);
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[m][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[b], xv[m], acc[m][b], 0, 0, 0);
    }
  }
  // element e of acc[m][b]: row wm 32 + m 16 + n, column (wn NB + b) 16 + 4 q + e
  const float scale = a.scale ? a.scale[g.adapter] : 1.f;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const int32_t row = wm * 32 + m * 16 + n;
    if (row >= rows) continue;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int c = c0 + (wn * NB + b) * 16 + 4 * q;
      if (c >= cols) continue;
      const int r = c % a.low_rank;  // four columns of one part
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = static_cast<__bf16>(r + e < a.rank ? acc[m][b][e] * scale : 0.f);
      *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.low) + static_cast<int64_t>(g.first + row) * cols + c) = v;
    }
  }
}

// ------------------------------------------------------------- few tokens
// Up to 64 tokens: bound by the weights' bytes, each read once.  A block takes
// 32 features; its waves share out the contraction and meet in LDS at the end.
// The adapters' share is a dot product of `rank` values for each output.
constexpr int kFewFeatures = kAdapterFewFeatures;

// A row's adapter in its place of `which`, -1 for none: a thread's segments write
// theirs (a row is in one segment).
template <int kRows, int kBlock>
__device__ inline void adapters_of_rows(const AdapterArgs& a, int32_t* which) {
  const int tid = threadIdx.x;
  if (tid < kRows) which[tid] = -1;
  __syncthreads();
  for (int32_t s = tid; s < a.segments; s += kBlock) {
    const Segment sg = segment(a, s);
    for (int32_t r = sg.first; r < sg.end; ++r) which[r] = sg.adapter;
  }
}

// The block's outputs from its waves' sums [row][feature], rows kFewFeatures + 1 apart.
template <int kRows, int kWaves>
__device__ inline void few_outputs(const AdapterArgs& a, const float* sums, const int32_t* which, int32_t f0) {
  constexpr int kStr = kFewFeatures + 1;
  const __bf16* bias = static_cast<const __bf16*>(a.bias);
  for (int i = threadIdx.x; i < kRows * kFewFeatures; i += kWaves * 64) {
    const int r = i / kFewFeatures, f = f0 + i % kFewFeatures;
    if (r >= a.M || f >= a.N) continue;
    const int part = f / a.split, j = which[r];
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) v += sums[k * kRows * kStr + r * kStr + i % kFewFeatures];
    if (j >= 0) {
      const __bf16* u = static_cast<const __bf16*>(a.low) + (r * a.parts + part) * a.low_rank;
      const __bf16* b = static_cast<const __bf16*>(a.b) + (static_cast<int64_t>(j) * a.N + f) * a.rank;
      float d = 0.f;
      for (int q = 0; q < a.rank; q += 8) {
        const bf16x8 uv = *reinterpret_cast<const bf16x8*>(u + q), bv = eight(b + q, a.rank - q);
#pragma unroll
        for (int e = 0; e < 8; ++e) d = __builtin_fmaf(static_cast<float>(uv[e]), static_cast<float>(bv[e]), d);
      }
      v += d;
    }
    v = (v + (bias ? static_cast<float>(bias[f]) : 0.f)) * (part == 0 ? a.part0_scale : 1.f);
    static_cast<__bf16*>(a.y[part])[static_cast<int64_t>(r) * a.split + (f - part * a.split)] = static_cast<__bf16>(v);
  }
}

// Whole rows: four waves, each with a ring of its own in LDS: 64-deep stages of
// its share, filled by direct transfers of whole cache lines, kRing of them on
// their way (no barriers).  Half lines a request, as the matrix cores' operands
// lie, take 10 us more for 16 tokens of 5120 -> 15360, and streamed (nt) ones are
// fetched twice.  That case: 31 us for 157 MB of weights, 5.1 TB/s.
template <int RT, int kRing>
__global__ __launch_bounds__(256) void few_ring_kernel(AdapterArgs a) {
  constexpr int kWaves = 4, FT = kFewFeatures / 16, kRows = RT * 16, kStr = kFewFeatures + 1;
  constexpr int kW = kFewFeatures * 128, kStage = kW + kRows * 128, kMine = kStage / 1024;  // kMine: transfers of a stage
  __shared__ __attribute__((aligned(16))) char lds[kWaves][kRing][kStage];
  __shared__ int32_t which[kRows];
  static_assert(kWaves * kRows * kStr * 4 <= static_cast<int>(sizeof(lds)), "the sums fit the rings' place");
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t f0 = static_cast<int32_t>(blockIdx.x) * kFewFeatures;
  const int stages = (a.K + 63) / 64, each = (stages + kWaves - 1) / kWaves, s0 = wave * each, s1 = min(s0 + each, stages);

  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&lds[wave][0][0]));
  const uint32_t wrb = static_cast<uint32_t>(a.K) * 2, xrb = static_cast<uint32_t>(a.x_stride) * 2;
  const __bf16* W = static_cast<const __bf16*>(a.w) + static_cast<int64_t>(f0) * a.K;
  const uint32_t wrows = min(kFewFeatures, a.N - f0) - 1, xrows = a.M - 1;
  // A transfer: rows 8 i + lane / 8, physical chunk lane % 8 holding logical chunk unswz128(row, lane % 8).
  auto put = [&](int st) {
    const int left = min(a.K - st * 64, 64);  // a multiple of 8
    const i32x4 rw = rsrc_of(W + st * 64, wrows * wrb + left * 2);
    const i32x4 rx = rsrc_of(static_cast<const __bf16*>(a.x) + st * 64, xrows * xrb + left * 2);
    const uint32_t base = lds0 + (st - s0) % kRing * kStage;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const bool is_x = i >= kW / 1024;
      const int row = (is_x ? i - kW / 1024 : i) * 8 + (lane >> 3), lc = unswz128(row, lane & 7);
      const uint32_t off = lc * 8 < left ? row * (is_x ? xrb : wrb) + lc * 16 : kPastEnd;
      if (is_x)
        dma16(rx, off, __builtin_amdgcn_readfirstlane(base + i * 1024));
      else
        dma16_nt(rw, off, __builtin_amdgcn_readfirstlane(base + i * 1024));
    }
  };
#pragma unroll
  for (int i = 0; i < kRing; ++i)
    if (s0 + i < s1) put(s0 + i);
  f32x4 acc[FT][RT];
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[f][t] = f32x4{};
  for (int st = s0; st < s1; ++st) {
    wait_for_stage<kRing - 1, kMine>(s1 - 1 - st);
    asm volatile("" ::: "memory");
    const char* L = lds[wave][(st - s0) % kRing];
    bf16x8 wv[2][FT], xv[2][RT];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int f = 0; f < FT; ++f) wv[ks][f] = *reinterpret_cast<const bf16x8*>(L + swz128(f * 16 + n, ks * 32 + g * 8) * 2);
#pragma unroll
      for (int t = 0; t < RT; ++t) xv[ks][t] = *reinterpret_cast<const bf16x8*>(L + kW + swz128(t * 16 + n, ks * 32 + g * 8) * 2);
    }
    // the buffer is filled again once it has been read
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (st + kRing < s1) put(st + kRing);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int f = 0; f < FT; ++f)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[ks][f], xv[ks][t], acc[f][t], 0, 0, 0);
  }
  __syncthreads();
  // element e of acc[f][t]: row 16 t + n, feature 16 f + 4 g + e
  float* sums = reinterpret_cast<float*>(&lds[0][0][0]);
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) sums[wave * kRows * kStr + (t * 16 + n) * kStr + f * 16 + 4 * g + e] = acc[f][t][e];
  adapters_of_rows<kRows, 256>(a, which);
  __syncthreads();
  few_outputs<kRows, kWaves>(a, sums, which, f0);
}

// Rows of at least 8 values that begin anywhere: eight waves, W and X from memory to
// registers as the matrix cores take them, kUnroll steps of 32 values on their way.
// Rows' ends as in low_kernel.
template <int RT, int kUnroll>
__global__ __launch_bounds__(512) void few_any_kernel(AdapterArgs a) {
  constexpr int kWaves = 8, FT = kFewFeatures / 16, kRows = RT * 16, kStr = kFewFeatures + 1;
  __shared__ float sums[kWaves * kRows * kStr];
  __shared__ int32_t which[kRows];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t f0 = static_cast<int32_t>(blockIdx.x) * kFewFeatures;
  const __bf16 *w[FT], *x[RT];
#pragma unroll
  for (int f = 0; f < FT; ++f) w[f] = static_cast<const __bf16*>(a.w) + static_cast<int64_t>(min(f0 + f * 16 + n, a.N - 1)) * a.K + g * 8;
#pragma unroll
  for (int t = 0; t < RT; ++t) x[t] = static_cast<const __bf16*>(a.x) + min(t * 16 + n, a.M - 1) * a.x_stride + g * 8;
  f32x4 acc[FT][RT];
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[f][t] = f32x4{};
  const int steps = (a.K + 31) / 32, each = (steps + kWaves - 1) / kWaves, s0 = wave * each, s1 = min(s0 + each, steps);
#pragma unroll 1
  for (int s = s0; s < s1; s += kUnroll) {
    Eight wv[kUnroll][FT], xv[kUnroll][RT];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int k = min(min(s + u, s1 - 1) * 32, a.K - 8 - g * 8);
#pragma unroll
      for (int f = 0; f < FT; ++f) wv[u][f] = Eight::at(w[f] + k);
#pragma unroll
      for (int t = 0; t < RT; ++t) xv[u][t] = Eight::at(x[t] + k);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (s + u >= s1) continue;
      const int left = a.K - (s + u) * 32;
      bf16x8 xs[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) xs[t] = left < 32 ? last_of(xv[u][t].values(), left - g * 8) : xv[u][t].values();
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        const bf16x8 ws = left < 32 ? last_of(wv[u][f].values(), left - g * 8) : wv[u][f].values();
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ws, xs[t], acc[f][t], 0, 0, 0);
      }
    }
  }
  // element e of acc[f][t]: row 16 t + n, feature 16 f + 4 g + e
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) sums[wave * kRows * kStr + (t * 16 + n) * kStr + f * 16 + 4 * g + e] = acc[f][t][e];
  adapters_of_rows<kRows, 512>(a, which);
  __syncthreads();
  few_outputs<kRows, kWaves>(a, sums, which, f0);
}

// ------------------------------------------------------------ many tokens
// Tiles of WM x MB x 32 rows and WN x NB x 32 features, WM x WN waves of
// MB x NB matrix-core tiles each (A = W rows, B = X rows).  The contraction
// comes in 64-deep stages of 128-byte rows (the swizzle of lds_stage.hpp)
// through kStages LDS buffers, filled by direct transfers kStages - 1 stages ahead;
// one barrier a stage.  (Small tiles, of which there are few, wait for their
// transfers' way: four buffers, 200 x 5120 -> 3000 takes 60 us with two, 47 with
// four, 50 with eight.)  KG groups of such waves take KG stages at once, each one
// of its own, and meet in the end.  The adapters follow as further stages: 64 ranks
// of one part of one segment, its rows' low-rank factors against B.
// Tiles are taken in panels of four feature tiles, each XCD a run of them.
// The outputs leave through LDS as whole-row 16-byte stores.
// Bound by the stages' way into LDS and the outputs': 27840 x 5120 -> 15360 takes
// 4.0 ms, 1.1 PFLOP/s (a large product reaches 1.2); 12870 x 1536 -> 4608 takes 205 to 220
// us, 0.85 PFLOP/s, the matrix cores busy 42 % of the time: 918 tiles are 3.6 rounds,
// each with 24 stages, a start and 118 MB / 918 of outputs.
constexpr int kBK = 64, kPanel = 4;

template <int WM, int WN, int MB, int NB, int KG, int kStages>
__global__ __launch_bounds__(WM * WN * KG * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void tile_kernel(AdapterArgs a) {
  constexpr int NW = WM * WN, kThreadsAll = NW * KG * 64, BM = WM * MB * 32, BN = WN * NB * 32;
  constexpr int kX = BM * 128, kW = BN * 128, kStage = kX + kW;  // bytes
  constexpr int TX = BM / 8 / NW, TW = BN / 8 / NW;              // transfers (8 rows) of a wave
  __shared__ __attribute__((aligned(16))) char lds[kStages * KG][kStage];
  __shared__ float biases[BN];
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  const int t = xcd_remap(blockIdx.x, tiles_m * tiles_n);
  const int panel = t / (tiles_m * kPanel), pw = min(kPanel, tiles_n - panel * kPanel);
  const int ip = t - panel * tiles_m * kPanel;
  const int32_t m0 = ip / pw * BM, f0 = (panel * kPanel + ip % pw) * BN;
  const int32_t m1 = min(m0 + BM, a.M), f1 = min(f0 + BN, a.N);

  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, hh = lane >> 5;
  const int kg = __builtin_amdgcn_readfirstlane((tid >> 6) / NW), wave = __builtin_amdgcn_readfirstlane((tid >> 6) % NW);
  const int wm = wave % WM, wn = wave / WM;

  // A transfer: rows 8 i + lane / 8, physical chunk lane % 8 holding logical
  // chunk unswz128(row, lane % 8).  Rows past the matrix read zeros.
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&lds[0][0]));
  auto put = [&](int buf, const __bf16* x, uint32_t xrb, uint32_t xbytes, const __bf16* w, uint32_t wrb, uint32_t wbytes, int chunks) {
    const i32x4 rx = rsrc_of(x, xbytes), rw = rsrc_of(w, wbytes);
    const uint32_t base = lds0 + buf * kStage;
#pragma unroll
    for (int i = 0; i < TX; ++i) {
      const int row = (wave * TX + i) * 8 + (lane >> 3), lc = unswz128(row, lane & 7);
      dma16(rx, lc < chunks ? row * xrb + lc * 16 : kPastEnd, __builtin_amdgcn_readfirstlane(base + (wave * TX + i) * 1024));
    }
#pragma unroll
    for (int i = 0; i < TW; ++i) {
      const int row = (wave * TW + i) * 8 + (lane >> 3), lc = unswz128(row, lane & 7);
      dma16(rw, lc < chunks ? row * wrb + lc * 16 : kPastEnd, __builtin_amdgcn_readfirstlane(base + kX + (wave * TW + i) * 1024));
    }
  };
  const __bf16* X = static_cast<const __bf16*>(a.x) + static_cast<int64_t>(m0) * a.x_stride;
  const __bf16* W = static_cast<const __bf16*>(a.w) + static_cast<int64_t>(f0) * a.K;
  const uint32_t xrb = static_cast<uint32_t>(a.x_stride) * 2, wrb = static_cast<uint32_t>(a.K) * 2;
  auto put_main = [&](int st) {
    const int k = (st * KG + kg) * kBK, left = KG == 1 ? min(a.K - k, kBK) : max(min(a.K - k, kBK), 0);  // a multiple of 8
    put(st % kStages * KG + kg, X + k, xrb, static_cast<uint32_t>(m1 - m0 - 1) * xrb + left * 2, W + k, wrb,
        static_cast<uint32_t>(f1 - f0 - 1) * wrb + left * 2, left / 8);
  };
  const int nst = (a.K + kBK * KG - 1) / (kBK * KG);
#pragma unroll
  for (int st = 0; st < kStages - 1; ++st)
    if (st < nst) put_main(st);

  // The adapters' stages, found one after the other: a segment with an adapter
  // among the tile's rows, a part among its features, 64 ranks.
  const int p0 = f0 / a.split, p1 = (f1 - 1) / a.split;
  struct {
    int32_t s, first, end, adapter, part, r0;
  } next{};
  auto to_segment = [&](int32_t s) {  // s or the next that has an adapter here; first = m1 where none does
    next.first = m1;
    for (; s < a.segments; ++s) {
      const Segment g = segment(a, s);
      const int32_t first = __builtin_amdgcn_readfirstlane(g.first), end = __builtin_amdgcn_readfirstlane(g.end);
      const int32_t adapter = __builtin_amdgcn_readfirstlane(g.adapter);
      if (first >= m1) break;
      if (adapter < 0 || first >= end || end <= m0) continue;
      next = {s, first, end, adapter, p0, 0};
      break;
    }
  };
  auto advance = [&]() {
    if ((next.r0 += kBK) < a.rank) return;
    next.r0 = 0;
    if (++next.part <= p1) return;
    to_segment(next.s + 1);
  };
  const uint32_t urb = static_cast<uint32_t>(a.parts * a.low_rank) * 2, brb = static_cast<uint32_t>(a.rank) * 2;
  auto put_low = [&](int buf) {
    const __bf16* u = static_cast<const __bf16*>(a.low) + static_cast<int64_t>(m0) * a.parts * a.low_rank + next.part * a.low_rank + next.r0;
    const __bf16* b = static_cast<const __bf16*>(a.b) + (static_cast<int64_t>(next.adapter) * a.N + f0) * a.rank + next.r0;
    const int left = min(a.rank - next.r0, kBK), chunks = (left + 7) / 8;
    const uint32_t ubytes = static_cast<uint32_t>(m1 - m0 - 1) * urb + chunks * 16;
    if (a.whole_b) {
      if (kg == 0) put(buf, u, urb, ubytes, b, brb, static_cast<uint32_t>(f1 - f0 - 1) * brb + left * 2, chunks);
    } else {
      // rows that are not whole aligned chunks: through registers
      const i32x4 ru = rsrc_of(u, ubytes);
#pragma unroll
      for (int i = 0; i < TX; ++i) {
        if (kg) break;
        const int row = (wave * TX + i) * 8 + (lane >> 3), lc = unswz128(row, lane & 7);
        dma16(ru, lc < chunks ? row * urb + lc * 16 : kPastEnd,
              __builtin_amdgcn_readfirstlane(lds0 + buf * kStage + (wave * TX + i) * 1024));
      }
      for (int c = tid; c < BN * 8; c += kThreadsAll) {
        const int row = c >> 3, chunk = c & 7;
        const int n = f0 + row < f1 ? left - chunk * 8 : 0;
        *reinterpret_cast<bf16x8*>(lds[buf] + kX + swz128(row, chunk * 8) * 2) = eight(b + static_cast<int64_t>(row) * a.rank + chunk * 8, n);
      }
    }
  };
  const __bf16* bias = static_cast<const __bf16*>(a.bias);
  if (tid < BN) biases[tid] = bias && f0 + tid < a.N ? static_cast<float>(bias[f0 + tid]) : 0.f;
  next.first = m1;
  if (a.segments) to_segment(__builtin_amdgcn_readfirstlane(first_segment(a, m0)));

  f32x16 acc[MB][NB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = f32x16{};
  // Operand reads: row (block base + n32), columns 16 ks + 8 hh; the swizzle
  // of a row depends only on n32 (block bases are multiples of 32).
  int rd[kBK / 16];
#pragma unroll
  for (int ks = 0; ks < kBK / 16; ++ks) rd[ks] = swz128(n32, ks * 16 + hh * 8) * 2;

  for (int st = 0; st < nst; ++st) {
    wait_for_stage<kStages - 2, TX + TW>(nst - 1 - st);
    // the stage before has been read by all: its buffer is filled next
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (st + kStages - 1 < nst) put_main(st + kStages - 1);
    if (st + 1 == nst && next.first < m1) put_low(nst % kStages * KG);
    const char* Xs = lds[st % kStages * KG + kg] + wm * MB * 32 * 128;
    const char* Ws = lds[st % kStages * KG + kg] + kX + wn * NB * 32 * 128;
    // Operands of k step ks in register set ks & 1: the reads of step ks + 1
    // run between the matrix instructions of step ks.
    bf16x8 op[2][NB + MB];
    auto rd_op = [&](int ks, int j) -> bf16x8 {
      return j < NB ? *reinterpret_cast<const bf16x8*>(Ws + j * 32 * 128 + rd[ks])
                    : *reinterpret_cast<const bf16x8*>(Xs + (j - NB) * 32 * 128 + rd[ks]);
    };
#pragma unroll
    for (int j = 0; j < NB + MB; ++j) op[0][j] = rd_op(0, j);
#pragma unroll
    for (int ks = 0; ks < kBK / 16; ++ks) {
      const int c = ks & 1;
#pragma unroll
      for (int i = 0; i < MB * NB; ++i) {
        const int mb = i / NB, nb = i % NB;
        acc[mb][nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[c][nb], op[c][NB + mb], acc[mb][nb], 0, 0, 0);
        if (ks + 1 < kBK / 16 && i < NB + MB) op[c ^ 1][i] = rd_op(ks + 1, i);
      }
      if constexpr (MB * NB < NB + MB)
#pragma unroll
        for (int j = MB * NB; j < NB + MB; ++j)
          if (ks + 1 < kBK / 16) op[c ^ 1][j] = rd_op(ks + 1, j);
    }
    if constexpr (MB * NB < NB + MB) continue;  // fewer matrix instructions than reads: the compiler's order
#pragma unroll
    for (int j = 0; j < NB + MB; ++j) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
    for (int ks = 0; ks < kBK / 16; ++ks)
#pragma unroll
      for (int i = 0; i < MB * NB; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (ks + 1 < kBK / 16 && i < NB + MB) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    __builtin_amdgcn_sched_barrier(0);
  }
  for (int st = nst; next.first < m1; ++st) {
    const int32_t first = next.first, end = next.end, fa = next.part * a.split, fb = fa + a.split;
    const int steps = (min(a.rank - next.r0, kBK) + 15) / 16;
    wait_vmcnt<0>();
    __syncthreads();
    advance();
    if (next.first < m1) put_low((st + 1) % kStages * KG);
    if (kg) continue;
    const char* Xs = lds[st % kStages * KG] + wm * MB * 32 * 128;
    const char* Ws = lds[st % kStages * KG] + kX + wn * NB * 32 * 128;
    const bool all_f = fa <= f0 && f1 <= fb;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int32_t row = m0 + (wm * MB + mb) * 32 + n32;
      const bool mine = row >= first && row < end;
      if (!__any(mine)) continue;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        f32x16 add = f32x16{};
#pragma unroll
        for (int ks = 0; ks < kBK / 16; ++ks)
          if (ks < steps)
            add = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(Ws + nb * 32 * 128 + rd[ks]),
                                                          *reinterpret_cast<const bf16x8*>(Xs + mb * 32 * 128 + rd[ks]), add, 0, 0, 0);
        if (all_f) {
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[mb][nb][e] += mine ? add[e] : 0.f;
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int32_t f = f0 + (wn * NB + nb) * 32 + 8 * (e >> 2) + 4 * hh + (e & 3);
            acc[mb][nb][e] += mine && f >= fa && f < fb ? add[e] : 0.f;
          }
        }
      }
    }
  }

  if constexpr (KG > 1) {
    // the first group takes the others' sums, one after the other
    static_assert(NW * MB * NB * 64 * 16 * 4 <= static_cast<int>(sizeof(lds)), "a group's sums fit the stage buffers");
    f32x4* const S = reinterpret_cast<f32x4*>(&lds[0][0]) + wave * MB * NB * 256 + lane;
#pragma unroll 1
    for (int g = 1; g < KG; ++g) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < MB * NB * 4; ++i) {
        f32x16& c = acc[i / 4 / NB][i / 4 % NB];
        const int e = i % 4 * 4;
        if (kg == g) S[i * 64] = f32x4{c[e], c[e + 1], c[e + 2], c[e + 3]};
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < MB * NB * 4; ++i) {
        f32x16& c = acc[i / 4 / NB][i / 4 % NB];
        if (kg == 0) {
          const f32x4 v = S[i * 64];
#pragma unroll
          for (int e = 0; e < 4; ++e) c[i % 4 * 4 + e] += v[e];
        }
      }
    }
  }

  // Epilogue through LDS, one wave row's rows at a time.
  constexpr int kEStr = BN + 8, kERows = MB * 32;
  static_assert(kERows * kEStr * 2 <= static_cast<int>(sizeof(lds)), "a wave row's outputs fit the stage buffers");
  __bf16* E = reinterpret_cast<__bf16*>(&lds[0][0]);
#pragma unroll 1
  for (int part_m = 0; part_m < WM; ++part_m) {
    __syncthreads();  // the stage buffers, or the rows before, are free
    if (wm == part_m && kg == 0) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          const int at = (wn * NB + nb) * 32 + 8 * jj + 4 * hh;
          const int32_t f = f0 + at;
          float bv[4], factor[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            bv[i] = biases[at + i];
            factor[i] = f + i < a.split ? a.part0_scale : 1.f;
          }
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) {
            bf16x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = static_cast<__bf16>((acc[mb][nb][4 * jj + i] + bv[i]) * factor[i]);
            *reinterpret_cast<bf16x4*>(E + (mb * 32 + n32) * kEStr + at) = v;
          }
        }
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < (kERows * BN / 8 + kThreadsAll - 1) / kThreadsAll; ++p) {
      const int c = p * kThreadsAll + tid, rt = c / (BN / 8), ch = c % (BN / 8);
      const int32_t row = m0 + part_m * kERows + rt, f = f0 + ch * 8;
      if (rt >= kERows || row >= m1 || f >= a.N) continue;
      const bf16x8 v = *reinterpret_cast<const bf16x8*>(E + rt * kEStr + ch * 8);
      if (a.whole_y) {
        const int part = f / a.split;  // 8 features never straddle a part (split % 8 == 0)
        *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(a.y[part]) + static_cast<int64_t>(row) * a.split + (f - part * a.split)) = v;
      } else {
        for (int i = 0; i < 8 && f + i < a.N; ++i) {
          const int part = (f + i) / a.split;
          static_cast<__bf16*>(a.y[part])[static_cast<int64_t>(row) * a.split + (f + i - part * a.split)] = v[i];
        }
      }
    }
  }
}

// -------------------------------------------------------------- odd rows
// Rows that are not whole aligned chunks, copied behind one another with zeros up
// to whole ones: the tiles' transfers take no others, and rows of fewer than 8 values
// none at all.  (With 128 x 128 tiles made
// through registers instead, 27840 x 5120 -> 15360 took 16.7 ms; the copies are 0.2.)
struct PackArgs {
  const __bf16* from[3];
  __bf16* to[3];
  int64_t stride[3], rows[3];  // stride: elements between rows
  int32_t K, K8;
};

__global__ __launch_bounds__(kThreads) void pack_kernel(PackArgs a) {
  const int32_t chunks = a.K8 / 8;
  int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
#pragma unroll
  for (int t = 0; t < 3; ++t) {
    const int64_t n = a.rows[t] * chunks;
    if (i < n) {
      const int64_t row = i / chunks;
      const int32_t k = static_cast<int32_t>(i - row * chunks) * 8;
      *reinterpret_cast<bf16x8*>(a.to[t] + row * a.K8 + k) = eight(a.from[t] + row * a.stride[t] + k, a.K - k);
      return;
    }
    i -= n;
  }
}

template <int RT, int kRing, int kUnroll>
void launch_few(const AdapterArgs& a, const AdapterPlan& plan, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(plan.blocks));
  if constexpr (RT * 16 <= kAdapterFewOdd) {
    if (!a.whole) {
      hipLaunchKernelGGL((few_any_kernel<RT, kUnroll>), grid, dim3(512), 0, stream, a);
      return;
    }
  }
  hipLaunchKernelGGL((few_ring_kernel<RT, kRing>), grid, dim3(256), 0, stream, a);
}

hipError_t launch_low(const AdapterArgs& a, const AdapterPlan& plan, hipStream_t stream) {
  const uint32_t tiles = static_cast<uint32_t>(plan.low_tiles), across = static_cast<uint32_t>(plan.low_across);
  if (plan.low_rows == kLowRows) {
    const dim3 grid(tiles, across), block(kLowWaves * 64);
    if (a.whole)
      hipLaunchKernelGGL(low_kernel<true>, grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL(low_kernel<false>, grid, block, 0, stream, a);
  } else {
    const dim3 grid(tiles * across), block(256);
    if (plan.low_columns == 32)
      hipLaunchKernelGGL((low_tile_kernel<1>), grid, block, 0, stream, a);
    else if (plan.low_columns == 64)
      hipLaunchKernelGGL((low_tile_kernel<2>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((low_tile_kernel<3>), grid, block, 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adapter_project(const AdapterArgs& given, const AdapterPlan& plan, hipStream_t stream) {
  AdapterArgs a = given;
  if (plan.pack_x || plan.pack_w) {
    const int32_t k8 = (a.K + 7) / 8 * 8;
    PackArgs p{};
    p.K = a.K;
    p.K8 = k8;
    char* to = static_cast<char*>(a.low) + plan.low_bytes;
    int64_t chunks = 0;
    auto pack = [&](int t, const void** tensor, int64_t rows, int64_t stride) {
      p.from[t] = static_cast<const __bf16*>(*tensor);
      p.to[t] = reinterpret_cast<__bf16*>(to);
      p.stride[t] = stride;
      p.rows[t] = rows;
      *tensor = to;
      to += rows * k8 * 2;
      chunks += rows * (k8 / 8);
    };
    if (plan.pack_x) {
      pack(0, &a.x, a.M, a.x_stride);
      a.x_stride = k8;
    }
    if (plan.pack_w) {
      pack(1, &a.w, a.N, a.K);
      if (a.segments) pack(2, &a.a, int64_t{a.adapters} * a.parts * a.rank, a.K);
      a.K = k8;
    }
    a.whole = true;
    hipLaunchKernelGGL(pack_kernel, dim3(static_cast<uint32_t>((chunks + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (plan.low_tiles) {
    if (const hipError_t e = launch_low(a, plan, stream); e != hipSuccess) return e;
  }
  const dim3 grid(static_cast<uint32_t>(plan.blocks));
  switch (plan.kernel) {
    case AdapterKernel::kFew:
      if (a.M <= 16)
        launch_few<1, 3, 7>(a, plan, stream);
      else if (a.M <= 32)
        launch_few<2, 2, 0>(a, plan, stream);
      else
        launch_few<4, 3, 0>(a, plan, stream);  // odd rows have been copied
      break;
    case AdapterKernel::kTiles64:
      if (plan.groups == 2)
        hipLaunchKernelGGL((tile_kernel<2, 2, 1, 1, 2, 4>), grid, dim3(512), 0, stream, a);
      else
        hipLaunchKernelGGL((tile_kernel<2, 2, 1, 1, 1, 4>), grid, dim3(256), 0, stream, a);
      break;
    case AdapterKernel::kTiles128:
      if (plan.groups == 2)
        hipLaunchKernelGGL((tile_kernel<2, 2, 2, 2, 2, 2>), grid, dim3(512), 0, stream, a);
      else
        hipLaunchKernelGGL((tile_kernel<2, 2, 2, 2, 1, 2>), grid, dim3(256), 0, stream, a);
      break;
    case AdapterKernel::kTiles256:
      hipLaunchKernelGGL((tile_kernel<2, 4, 4, 2, 1, 2>), grid, dim3(512), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace mssa
