// Y = X W^T + b with MXFP4 weights (mssa_mx_project): tokens in 8 bits with
// one fp32 scale each (applied to the fp32 sum), or in MXFP4.
//
// The block-scaled matrix instructions take both operands as they lie in
// memory: a lane holds the 32 values of one MXFP4 block (16 bytes) and the
// block's scale byte; e4m3 operands are 16-byte pieces of two such blocks.
// The contraction runs over blocks in any order as long as both operands take the same one, so the two lane
// halves take the first and the second half of a stage's blocks and each
// lane's scales of a stage are consecutive bytes.
//
// Bound by waiting for the stages' transfers where there are many tokens
// (27840 x 5120 -> 15360 in MXFP4: 1.20 ms, 3.6 PFLOP/s, matrix cores busy 42 %
// of the time; 12870 x 1536 -> 4608 in e4m3: 104 us, 1.7 PFLOP/s, busy 35 %, an
// eighth of it the 118 MB of outputs), by the weights' bytes where there are
// few (1 x 5120 -> 15360: 12.1 us with 8-bit tokens, 3.5 TB/s, 11.3 with MXFP4
// ones), by 36 to 160 blocks for 256 CUs in between (64 x 5120 -> 15360: 22 and
// 17 us).  Waves of 128 x 128 outputs read a quarter
// fewer LDS bytes but are alone on their SIMD: 1.34 ms and 141 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "lds_stage.hpp"
#include "lowbit_args.hpp"
#include "lowbit_values.hpp"
#include "xcd.hpp"

namespace mssa {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kFmtE4M3 = 0, kFmtE2M1 = 4;  // operand formats of the f8f6f4 instructions
constexpr uint32_t kPastEnd = 0xfffffff0u;  // a buffer offset outside every range

// bf16 outputs take the f8f6f4 instructions for 8-bit tokens too.  Inside one
// of those steps the matrix core aligns e4m3 products to the largest of them
// with fewer bits than fp32 has: up to 2^-12 of the sum of magnitudes was
// measured on codes of every size, 6e-6 of the result's norm on ordinary
// tokens, far below the output's own rounding.  fp32 outputs of 8-bit tokens
// are asked for to be more exact than that: both operands are expanded to
// bf16, which holds them exactly, and multiplied with fp32 sums (12870 x 1536 ->
// 4608: 171-189 us against 104-107 with bf16 outputs, which are half the bytes;
// each wave expands its own copy of both operands).  (e2m1 by e2m1 steps add
// exactly enough for both.)
template <bool XF4, class T>
constexpr bool kWide = !XF4 && std::is_same_v<T, float>;

__device__ inline i32x8 widen(i32x4 v) { return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; }

// n consecutive features' outputs of one token, from feature col on.
template <class T, int N>
__device__ inline void store_features(const ProjectArgs& a, int64_t row, int col, const float (&v)[N]) {
  const T* bias = static_cast<const T*>(a.bias);
  const int part = col / a.split, pc = col - part * a.split;
  if ((a.split & 3) == 0 && col + N <= a.N) {
    typedef T vec __attribute__((ext_vector_type(N)));
    vec u;
    const float f = part == 0 ? a.part0_scale : 1.f;
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = static_cast<T>((v[i] + (bias ? static_cast<float>(bias[col + i]) : 0.f)) * f);
    *reinterpret_cast<vec*>(static_cast<T*>(a.y[part]) + row * a.split + pc) = u;
    return;
  }
  for (int i = 0; i < N && col + i < a.N; ++i) {
    const int p = (col + i) / a.split, c = col + i - p * a.split;
    static_cast<T*>(a.y[p])[row * a.split + c] =
        static_cast<T>((v[i] + (bias ? static_cast<float>(bias[col + i]) : 0.f)) * (p == 0 ? a.part0_scale : 1.f));
  }
}

// Tiles.  A block of WM x WN waves owns BM tokens x BN features; the matrix
// instruction computes the transposed tile (A = W rows, B = X rows), so a
// lane holds one token and runs of four features.  A stage is 128 bytes
// of every token (four blocks of e4m3, eight of MXFP4: whole cache lines) and
// as many blocks of every feature, moved by direct global -> LDS transfers;
// kBufs of them are in LDS or on their way.  Scale bytes come four to a row and
// stage with 8-bit tokens, sixteen for two stages at once with MXFP4 tokens.
template <bool XF4, int BM, int BN, int WM, int WN, int BUFS>
struct TileShape {
  static constexpr int kThreads = WM * WN * 64, kWaves = WM * WN;
  static constexpr int NBK = XF4 ? 8 : 4, NS = NBK / 2;   // blocks and matrix steps a stage
  // stages that share a transfer of scales: 4 bytes of each feature are few
  // beside the stage's 48 KB, 8 of both operands' rows are not
  static constexpr int kSuper = XF4 ? 2 : 1, kSBytes = NBK * kSuper;
  static constexpr int kSBufs = kSuper == 1 ? BUFS : 2;
  static constexpr int XB = 128, WB = NBK * 16;           // bytes of a row a stage
  static constexpr int kBufs = BUFS;
  // LDS: the X tiles of all buffers, the W tiles, two groups' scales
  static constexpr int kXBytes = BM * XB, kWBytes = BN * WB, kStage = kXBytes + kWBytes;
  static constexpr int kWBase = BUFS * kXBytes, kSBase = BUFS * kStage;
  static constexpr int kSRows = (XF4 ? BM : 0) + BN, kScales = kSRows * kSBytes;
  static constexpr int NX = kXBytes / 1024 / kWaves, NW = kWBytes / 1024 / kWaves;  // transfers of a wave a stage
  static_assert(NX * 1024 * kWaves == kXBytes && NW * 1024 * kWaves == kWBytes, "whole transfers");
  static constexpr int NSG = (kSRows / 64 + kWaves - 1) / kWaves;  // groups of 64 scale rows of a wave
  static_assert(kSRows % 64 == 0 && BM % 64 == 0, "whole groups of scale rows");
  static_assert(kBufs * kStage + kSBufs * kScales == tile_lds({BM, BN, WM, WN, BUFS}, XF4), "the tile choice's LDS");
  static_assert(kBufs * kStage + kSBufs * kScales <= kLdsBytes, "LDS of a CU");
};

// Chunk (16 bytes) c of row r lies at chunk c ^ swizzle(r): sixteen rows read
// at one chunk hit distinct banks.
template <int ROW>
__device__ inline int chunk_swizzle(int row) {
  return ROW == 128 ? (row >> 1) & 7 : (row >> 2) & 3;
}

// Order of a run of P matrix instructions and R LDS reads: the reads spread
// evenly behind the products.
template <int P, int R, int K = 0>
__device__ inline void interleave() {
  if constexpr (K < P) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (R * (K + 1) / P > R * K / P) __builtin_amdgcn_sched_group_barrier(0x100, R * (K + 1) / P - R * K / P, 0);
    interleave<P, R, K + 1>();
  }
}

template <bool XF4, class T, int BM, int BN, int WM, int WN, int BUFS>
__global__ __launch_bounds__(WM* WN * 64) __attribute__((amdgpu_waves_per_eu(BM / WM * BN / WN > 128 * 64 ? 1 : 2)))
void tile_kernel(ProjectArgs a) {
  using S = TileShape<XF4, BM, BN, WM, WN, BUFS>;
  constexpr int NBK = S::NBK, NS = S::NS, XB = S::XB, WB = S::WB, NX = S::NX, NW = S::NW;
  constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  // The output's rows, 32 of every wave, take the stages' place at the end.
  constexpr int kPitch = BN * static_cast<int>(sizeof(T)) + 16, kOut = WM * 32 * kPitch, kVec = 16 / sizeof(T);
  constexpr int kIn = S::kBufs * S::kStage + S::kSBufs * S::kScales, kOutBufs = 2 * kOut <= kIn ? 2 : 1;
  static_assert(kIn >= kOut, "the outputs' rows fit the stages' place");
  __shared__ __attribute__((aligned(16))) char lds[kIn];

  // Tiles in panels of four feature tiles: the blocks of an XCD, a run of
  // them, share rows of both operands in its L2.
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  const int L = xcd_remap(blockIdx.x, gridDim.x);
  const int panel = L / (tiles_m * 4), in = L - panel * tiles_m * 4, wide = min(4, tiles_n - panel * 4);
  const int tm = in / wide, tn = panel * 4 + in - tm * wide;
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int mrows = min(BM, a.M - tm * BM), nrows = min(BN, a.N - tn * BN);
  const uint32_t xp = static_cast<uint32_t>(a.NB) * (XF4 ? 16 : 32), wp = static_cast<uint32_t>(a.NB) * 16;
  const char* X = static_cast<const char*>(a.x) + static_cast<int64_t>(tm) * BM * xp;
  const char* W = static_cast<const char*>(a.w) + static_cast<int64_t>(tn) * BN * wp;
  const uint8_t* XS = static_cast<const uint8_t*>(a.xs) + static_cast<int64_t>(tm) * BM * a.NB;
  const uint8_t* WS = static_cast<const uint8_t*>(a.ws) + static_cast<int64_t>(tn) * BN * a.NB;
  // Scales go straight to LDS too where a group of a row's is whole dwords of
  // it; else through registers.
  constexpr int SB = S::kSBytes;
  const ScaleGroups<NBK, S::kSuper> groups{a.NB};
  const bool direct = groups.direct();

  // Transfer i of a wave fills 1 KB of consecutive LDS, XB- or WB-byte rows of
  // it; a lane's 16 bytes are its physical chunk's.  The rows of transfer i
  // are i * (1024 / XB) further on, which moves the swizzle by a fixed pattern.
  constexpr int kXRows = 1024 / XB, kWRows = 1024 / WB;
  auto x_chunk = [&](int i) { return (lane % (XB / 16)) ^ chunk_swizzle<XB>((wave * NX + i) * kXRows + lane / (XB / 16)); };
  auto w_chunk = [&](int i) { return (lane % (WB / 16)) ^ chunk_swizzle<WB>((wave * NW + i) * kWRows + lane / (WB / 16)); };
  const uint32_t x_row = (wave * NX * kXRows + lane / (XB / 16)) * xp, w_row = (wave * NW * kWRows + lane / (WB / 16)) * wp;
  // (1024 / 128 = 8 rows: the swizzle has two values; 16 rows of 64 bytes: one)
  constexpr int kXAlt = XB == 128 ? 2 : 1, kWAlt = WB == 128 ? 2 : 1;
  uint32_t xo[kXAlt], wo[kWAlt];
#pragma unroll
  for (int i = 0; i < kXAlt; ++i) xo[i] = x_row + x_chunk(i) * 16;
#pragma unroll
  for (int i = 0; i < kWAlt; ++i) wo[i] = w_row + w_chunk(i) * 16;
  const i32x4 rx = rsrc_of(X, static_cast<uint32_t>(mrows) * xp);
  const i32x4 rw = rsrc_of(W, static_cast<uint32_t>(nrows) * wp);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&lds[0]));
  // The place in LDS of a stage's group of scales.
  auto scale_place = [&](int st) { return S::kSBase + st / S::kSuper % S::kSBufs * S::kScales; };
  // The scales of stage st's group, straight to LDS.  A wave takes 64 rows
  // (where there are fewer groups than waves, two take the same).
  auto issue_scales = [&](int st) {
    const uint32_t dst = lds0 + scale_place(st);
    const int first = groups.first(st);
#pragma unroll
    for (int i = 0; i < S::NSG; ++i) {
      const int group = (wave + i * S::kWaves) % (S::kSRows / 64);  // rows of X first for MXFP4 tokens
      const bool of_x = XF4 && group * 64 < BM;
      const int row = group * 64 + lane - (XF4 && !of_x ? BM : 0), rows = of_x ? mrows : nrows;
      const i32x4 range = rsrc_of(of_x ? XS : WS, static_cast<uint32_t>(rows) * a.NB);
      const uint32_t off = row < rows ? row * static_cast<uint32_t>(a.NB) + first : kPastEnd;
      const uint32_t to = __builtin_amdgcn_readfirstlane(dst + group * 64 * SB);
      if constexpr (SB == 16)
        dma16(range, off, to);
      else
        dma4(range, off, to);
    }
  };
  // Stage st, all of its blocks inside the rows.
  auto issue_full = [&](int st, int buf) {
    const uint32_t bx = lds0 + buf * S::kXBytes, bw = lds0 + S::kWBase + buf * S::kWBytes;
#pragma unroll
    for (int i = 0; i < NX; ++i)
      dma16(rx, xo[i % kXAlt] + (i * kXRows * xp + st * XB), __builtin_amdgcn_readfirstlane(bx + (wave * NX + i) * 1024));
#pragma unroll
    for (int i = 0; i < NW; ++i)
      dma16(rw, wo[i % kWAlt] + (i * kWRows * wp + st * WB),
            __builtin_amdgcn_readfirstlane(bw + (wave * NW + i) * 1024));
  };
  // Any stage (past the last: zeros, which keep the count of transfers in
  // flight the same), with the scales of its group if it is the group's first.
  auto issue = [&](int st) {
    const int left = a.NB - st * NBK;
    if (st % S::kSuper == 0 && left > 0) {
      if (direct) {
        issue_scales(st);
      } else {
        // rows past the tile and blocks past the row: zeros (their codes are)
        const int first = groups.first(st);
        for (int group = wave; group < S::kSRows / 64; group += S::kWaves) {
          const bool of_x = XF4 && group * 64 < BM;
          const int row = group * 64 + lane - (XF4 && !of_x ? BM : 0);
          uint32_t v[SB / 4] = {};
          if (row < (of_x ? mrows : nrows)) {
            const uint8_t* p = (of_x ? XS : WS) + static_cast<int64_t>(row) * a.NB + first;
#pragma unroll
            for (int k = 0; k < SB; ++k)
              if (first + k < a.NB) v[k >> 2] |= static_cast<uint32_t>(p[k]) << (8 * (k & 3));
          }
#pragma unroll
          for (int k = 0; k < SB / 4; ++k)
            *reinterpret_cast<uint32_t*>(lds + scale_place(st) + (group * 64 + lane) * SB + k * 4) = v[k];
        }
      }
    }
    if (left >= NBK) {
      issue_full(st, st % S::kBufs);
      return;
    }
    const uint32_t bx = lds0 + st % S::kBufs * S::kXBytes, bw = lds0 + S::kWBase + st % S::kBufs * S::kWBytes;
#pragma unroll
    for (int i = 0; i < NX; ++i)
      dma16(rx, x_chunk(i) / (XF4 ? 1 : 2) < left ? xo[i % kXAlt] + (i * kXRows * xp + st * XB) : kPastEnd,
            __builtin_amdgcn_readfirstlane(bx + (wave * NX + i) * 1024));
#pragma unroll
    for (int i = 0; i < NW; ++i)
      dma16(rw, w_chunk(i) < left ? wo[i % kWAlt] + (i * kWRows * wp + st * WB) : kPastEnd,
            __builtin_amdgcn_readfirstlane(bw + (wave * NW + i) * 1024));
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x16{};

  // Scales of a stage: byte j of a row's is matrix step j's (block hh NS + j).
  // Of a short last stage (with 8-bit tokens its group is filled with zeros)
  // a lane half may have none: zeros then, as its codes are.
  int sx[TM], sw[TN];
  using scales_t = std::conditional_t<NS == 4, uint32_t, uint16_t>;
  auto read_scales = [&](int st, auto full) {
    const bool there = !XF4 || decltype(full)::value || groups.there(st, hh);
    const char* P = lds + scale_place(st) + (there ? groups.offset(st, hh) : 0);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      sx[i] = XF4 ? *reinterpret_cast<const scales_t*>(P + ((wm * TM + i) * 32 + n32) * SB) : 0x7f7f;
      if (!there) sx[i] = 0;
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      sw[j] = *reinterpret_cast<const scales_t*>(P + ((XF4 ? BM : 0) + (wn * TN + j) * 32 + n32) * SB);
      if (!there) sw[j] = 0;
    }
  };
  // Operands of step J of the stage in buffer buf: 32 rows further on is a
  // fixed distance, for the swizzle too.
  i32x8 xv[2][TM];
  i32x4 wv[2][TN];
  int xa[NS][XF4 ? 1 : 2], wa[NS];
#pragma unroll
  for (int J = 0; J < NS; ++J) {
    const int xr = wm * TM * 32 + n32, wr = wn * TN * 32 + n32;
    // e4m3: a lane's first 16 bytes are its half's piece of the first lane
    // half's block, its last 16 bytes of the second's; expanded to bf16, a
    // lane takes the block of its own half
    const int c0 = XF4 ? hh * NS + J : kWide<XF4, T> ? 2 * (hh * NS + J) : 2 * J + hh;
    const int c1 = kWide<XF4, T> ? c0 + 1 : 2 * (NS + J) + hh;
    xa[J][0] = xr * XB + ((c0 ^ chunk_swizzle<XB>(xr)) << 4);
    if constexpr (!XF4) xa[J][1] = xr * XB + ((c1 ^ chunk_swizzle<XB>(xr)) << 4);
    wa[J] = S::kWBase + wr * WB + (((hh * NS + J) ^ chunk_swizzle<WB>(wr)) << 4);
  }
  auto read_step = [&](auto js, int buf) {
    constexpr int J = decltype(js)::value;
#pragma unroll
    for (int j = 0; j < TN; ++j)
      wv[J & 1][j] = *reinterpret_cast<const i32x4*>(lds + wa[J] + buf * S::kWBytes + j * 32 * WB);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const char* X0 = lds + xa[J][0] + buf * S::kXBytes + i * 32 * XB;
      if constexpr (XF4) {
        xv[J & 1][i] = widen(*reinterpret_cast<const i32x4*>(X0));
      } else {
        const i32x4 lo = *reinterpret_cast<const i32x4*>(X0);
        const i32x4 hi = *reinterpret_cast<const i32x4*>(lds + xa[J][1] + buf * S::kXBytes + i * 32 * XB);
        xv[J & 1][i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    }
  };
  auto multiply = [&](auto js) {
    constexpr int J = decltype(js)::value;
    if constexpr (kWide<XF4, T>) {
#pragma unroll
      for (int p = 0; p < 4; ++p) {  // eight values at a time
        bf16x8 xw[TM], ww[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) xw[i] = expand_e4m3(xv[J & 1][i][2 * p], xv[J & 1][i][2 * p + 1]);
#pragma unroll
        for (int j = 0; j < TN; ++j) ww[j] = expand_e2m1(wv[J & 1][j][p], mx_scale((static_cast<uint32_t>(sw[j]) >> (8 * J)) & 255u));
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ww[j], xw[i], acc[i][j], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(widen(wv[J & 1][j]), xv[J & 1][i], acc[i][j], kFmtE2M1,
                                                                     XF4 ? kFmtE2M1 : kFmtE4M3, J, sw[j], XF4 ? J : 0, sx[i]);
    }
  };
  constexpr int kReads = TM * (XF4 ? 1 : 2) + TN, kProducts = kWide<XF4, T> ? 0 : TM * TN;

  const int nst = (a.NB + NBK - 1) / NBK;
#pragma unroll
  for (int i = 0; i < S::kBufs; ++i) issue(i);
  // A step's operands are read while the step before is multiplied, across
  // the stages' edges too: before the last step every wave has read the whole
  // stage, and its buffer takes the transfers of stage + kBufs.
  auto arrive = [&](auto later_c) {  // this wave's transfers but those of `later` stages, then everybody's
    wait_vmcnt<decltype(later_c)::value * (NX + NW)>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  arrive(std::integral_constant<int, S::kBufs - 1>{});
  read_scales(0, std::false_type{});
  read_step(std::integral_constant<int, 0>{}, 0);
  auto stage = [&](int buf, int next, int next_buf, auto next_full, auto refill) {
    auto inner = [&](auto js) {
      constexpr int J = decltype(js)::value;
      read_step(std::integral_constant<int, J + 1>{}, buf);
      multiply(js);
      interleave<kProducts, kReads>();
      __builtin_amdgcn_sched_barrier(0);
    };
    inner(std::integral_constant<int, 0>{});
    if constexpr (NS == 4) {
      inner(std::integral_constant<int, 1>{});
      inner(std::integral_constant<int, 2>{});
    }
    arrive(std::integral_constant<int, S::kBufs - 2>{});
    refill();
    __builtin_amdgcn_sched_barrier(0);
    multiply(std::integral_constant<int, NS - 1>{});
    read_step(std::integral_constant<int, 0>{}, next_buf);
    read_scales(next, next_full);
    interleave<kProducts, kReads + (XF4 ? TM : 0) + TN>();
    __builtin_amdgcn_sched_barrier(0);
  };
  // Stages whose refill is a whole one (and the next stage with it), without a branch in the loop (the
  // compiler would move products across it); then the rest.
  int st = 0;
  if (direct)
    for (const int whole = a.NB / NBK; st + S::kSuper - 1 + S::kBufs < whole; st += S::kSuper)
#pragma unroll
      for (int u = 0; u < S::kSuper; ++u) {
        // st is a multiple of kSuper: where that is one of kBufs the buffers are constants
        const int s0 = S::kSuper % S::kBufs == 0 ? 0 : st;
        stage((s0 + u) % S::kBufs, st + u + 1, (s0 + u + 1) % S::kBufs, std::true_type{}, [&] {
          if ((u + S::kBufs) % S::kSuper == 0) issue_scales(st + u + S::kBufs);
          issue_full(st + u + S::kBufs, (s0 + u) % S::kBufs);
        });
      }
  for (; st < nst; ++st) {
    const int next = st + 1 < nst ? st + 1 : st;  // past the last stage: read again, not used
    stage(st % S::kBufs, next, next % S::kBufs, std::false_type{}, [&] { issue(st + S::kBufs); });
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");

  // Outputs leave through LDS, 32 rows of every wave at a time, as whole rows
  // of the tile: a lane's own runs of four features would be 8-byte stores
  // into 32 rows at once (half of the time of a short contraction).
  const T* bias = static_cast<const T*>(a.bias);
  const bool vectors = a.split % kVec == 0;
  // this lane's features: bias and factor, 4 jj + e of feature block j
  float add[TN][16], factor[TN][16];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int col = tn * BN + (wn * TN + j) * 32 + 8 * (e >> 2) + 4 * hh + (e & 3);
      add[j][e] = bias && col < a.N ? static_cast<float>(bias[col]) : 0.f;
      factor[j][e] = col < a.split ? a.part0_scale : 1.f;
    }
  wait_vmcnt<0>();  // the transfers past the last stage
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    char* E = lds + i % kOutBufs * kOut;
    if (kOutBufs == 1 && i > 0) __syncthreads();
    const int r_in = (wm * TM + i) * 32 + n32;
    const float xs = XF4 || r_in >= mrows ? 1.f : static_cast<const float*>(a.xs)[static_cast<int64_t>(tm) * BM + r_in];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const int ct = (wn * TN + j) * 32 + 8 * jj + 4 * hh;
        typedef T vec4 __attribute__((ext_vector_type(4)));
        vec4 u;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          u[e] = static_cast<T>((acc[i][j][4 * jj + e] * xs + add[j][4 * jj + e]) * factor[j][4 * jj + e]);
        *reinterpret_cast<vec4*>(E + (wm * 32 + n32) * kPitch + ct * sizeof(T)) = u;
      }
    __syncthreads();
    for (int p = tid; p < WM * 32 * (BN / kVec); p += S::kThreads) {
      const int er = p / (BN / kVec), ct = p % (BN / kVec) * kVec, col = tn * BN + ct;
      const int row_in = (er / 32 * TM + i) * 32 + er % 32;
      if (row_in >= mrows || col >= a.N) continue;
      const int64_t row = static_cast<int64_t>(tm) * BM + row_in;
      const char* src = E + er * kPitch + ct * sizeof(T);
      if (vectors) {
        const int part = col / a.split;
        // streamed: the outputs are not to push the operands out of L2
        __builtin_nontemporal_store(*reinterpret_cast<const i32x4*>(src),
                                    reinterpret_cast<i32x4*>(static_cast<T*>(a.y[part]) + row * a.split + (col - part * a.split)));
      } else {
        for (int e = 0; e < kVec && col + e < a.N; ++e) {
          const int part = (col + e) / a.split;
          static_cast<T*>(a.y[part])[row * a.split + (col + e - part * a.split)] = reinterpret_cast<const T*>(src)[e];
        }
      }
    }
  }
}

// Few tokens: the weights are read once, from memory straight into the
// matrix instruction's operand (16 features x 128 values, A = W rows); the
// tokens are the 16 columns of B.  Sixteen features a block, whose waves take
// pieces of the contraction and join their sums in LDS.  A lane group (lane /
// 16) takes blocks 4 g .. 4 g + 3 of sixteen, one per matrix step, so its
// codes are 64 consecutive bytes and its scales four.  What counts is bytes on
// their way: each wave has its next piece loading.
constexpr int kFewWaves = kProjectFewWaves;

// Four scale bytes, of which the first n are there.
__device__ inline uint32_t four_scales(const uint8_t* p, int n) {
  typedef uint32_t u32_u __attribute__((aligned(1)));
  if (n >= 4) return *reinterpret_cast<const u32_u*>(p);
  uint32_t v = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < n) v |= static_cast<uint32_t>(p[i]) << (8 * i);
  return v;
}

template <bool XF4, class T, int TT>
__global__ __launch_bounds__(kFewWaves * 64) void few_kernel(ProjectArgs a) {
  __shared__ float red[kFewWaves - 1][TT][4][64];
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * kProjectFewFeatures;
  const int64_t xp = static_cast<int64_t>(a.NB) * (XF4 ? 16 : 32);
  const int feature = min(n0 + m, a.N - 1);
  const char* W = static_cast<const char*>(a.w) + static_cast<int64_t>(feature) * a.NB * 16;
  const uint8_t* WS = static_cast<const uint8_t*>(a.ws) + static_cast<int64_t>(feature) * a.NB;
  f32x4 acc[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[t] = f32x4{};

  const int nsb = (a.NB + 15) / 16;
  struct Weights {
    i32x4 v[4];
    uint32_t s;
  } now, later;
  auto fetch = [&](Weights& w, int sb) {
    const int b0 = sb * 16 + g * 4, left = a.NB - b0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w.v[j] = j < left ? *reinterpret_cast<const i32x4*>(W + (b0 + j) * 16) : i32x4{};
    w.s = four_scales(WS + b0, left);
  };
  if (wave < nsb) fetch(now, wave);
  for (int sb = wave; sb < nsb; sb += kFewWaves) {
    const int b0 = sb * 16 + g * 4, left = a.NB - b0;
    i32x4 xv[TT][4][XF4 ? 1 : 2];
    uint32_t sx[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int64_t tok = t * 16 + m;
      const bool ok = tok < a.M;
      const char* X = static_cast<const char*>(a.x) + (ok ? tok : 0) * xp;
      sx[t] = 0x7f7f7f7fu;
      if constexpr (XF4) sx[t] = ok ? four_scales(static_cast<const uint8_t*>(a.xs) + tok * a.NB + b0, left) : 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (XF4) {
          xv[t][j][0] = ok && j < left ? *reinterpret_cast<const i32x4*>(X + (b0 + j) * 16) : i32x4{};
        } else if constexpr (kWide<XF4, T>) {
          xv[t][j][0] = ok && j < left ? *reinterpret_cast<const i32x4*>(X + (b0 + j) * 32) : i32x4{};
          xv[t][j][1] = ok && j < left ? *reinterpret_cast<const i32x4*>(X + (b0 + j) * 32 + 16) : i32x4{};
        } else {
          // e4m3: 16 bytes of the block of group g / 2, 16 of group 2 + g / 2's
          const int c0 = sb * 16 + (g >> 1) * 4 + j, c1 = c0 + 8;
          xv[t][j][0] = ok && c0 < a.NB ? *reinterpret_cast<const i32x4*>(X + c0 * 32 + (g & 1) * 16) : i32x4{};
          xv[t][j][1] = ok && c1 < a.NB ? *reinterpret_cast<const i32x4*>(X + c1 * 32 + (g & 1) * 16) : i32x4{};
        }
      }
    }
    if (sb + kFewWaves < nsb) fetch(later, sb + kFewWaves);
    auto step = [&](auto js) {
      constexpr int J = decltype(js)::value;
      if constexpr (kWide<XF4, T>) {
        const float f = mx_scale((now.s >> (8 * J)) & 255u);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const bf16x8 wa = expand_e2m1(static_cast<uint32_t>(now.v[J][p]), f);
#pragma unroll
          for (int t = 0; t < TT; ++t) {
            const i32x4 v = xv[t][J][p >> 1];
            const bf16x8 xw = expand_e4m3(static_cast<uint32_t>(v[2 * (p & 1)]), static_cast<uint32_t>(v[2 * (p & 1) + 1]));
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa, xw, acc[t], 0, 0, 0);
          }
        }
        return;
      }
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        i32x8 b;
        if constexpr (XF4)
          b = widen(xv[t][J][0]);
        else
          b = __builtin_shufflevector(xv[t][J][0], xv[t][J][1], 0, 1, 2, 3, 4, 5, 6, 7);
        acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(widen(now.v[J]), b, acc[t], kFmtE2M1,
                                                                  XF4 ? kFmtE2M1 : kFmtE4M3, J, now.s, XF4 ? J : 0, sx[t]);
      }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
    now = later;
  }
  if (wave > 0) {
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[wave - 1][t][e][lane] = acc[t][e];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = acc[t][e];
#pragma unroll
      for (int w = 0; w < kFewWaves - 1; ++w) v[e] += red[w][t][e][lane];
    }
    const int64_t tok = t * 16 + m;
    const int col = n0 + 4 * g;
    if (tok >= a.M || col >= a.N) continue;
    if constexpr (!XF4) {
      const float xs = static_cast<const float*>(a.xs)[tok];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= xs;
    }
    store_features<T, 4>(a, tok, col, v);
  }
}

template <bool XF4, class T, int TT>
hipError_t few_go(const ProjectArgs& a, const ProjectPlan& plan, hipStream_t stream) {
  hipLaunchKernelGGL((few_kernel<XF4, T, TT>), dim3(static_cast<uint32_t>(plan.blocks)), dim3(kFewWaves * 64), 0, stream, a);
  return hipGetLastError();
}

template <bool XF4, class T, bool LARGE>
hipError_t tile_go(const ProjectArgs& a, const ProjectPlan& plan, hipStream_t stream) {
  constexpr TileSize t = tile_size(XF4, LARGE);
  hipLaunchKernelGGL((tile_kernel<XF4, T, t.tokens, t.features, t.waves_m, t.waves_n, t.stages>),
                     dim3(static_cast<uint32_t>(plan.blocks)), dim3(t.threads()), 0, stream, a);
  return hipGetLastError();
}

template <bool XF4, class T>
hipError_t project(const ProjectArgs& a, hipStream_t stream) {
  ProjectPlan plan;
  if (const hipError_t e = plan_mx_project(a.M, a.N, a.NB, XF4, &plan); e != hipSuccess) return e;
  switch (plan.kernel) {
    case ProjectKernel::kFew16: return few_go<XF4, T, 1>(a, plan, stream);
    case ProjectKernel::kFew32: return few_go<XF4, T, 2>(a, plan, stream);
    case ProjectKernel::kSmallTiles: return tile_go<XF4, T, false>(a, plan, stream);
    default: return tile_go<XF4, T, true>(a, plan, stream);
  }
}

}  // namespace

hipError_t launch_mx_project(const ProjectArgs& a, bool x_fp4, bool out_bf16, hipStream_t stream) {
  if (x_fp4) return out_bf16 ? project<true, __bf16>(a, stream) : project<true, float>(a, stream);
  return out_bf16 ? project<false, __bf16>(a, stream) : project<false, float>(a, stream);
}

}  // namespace mssa
