// Attention over K/V caches held in MXFP4 (mssa_mx_attention).
//
// The rows that share a key head (n_q queries x group heads) are cut into
// blocks of 32 per wave, the context into tiles of 64 tokens.  A tile's codes are
// expanded to bf16 once per block: one MXFP4 block (16 bytes of codes, one
// scale byte) per thread and pass, by the conversion instructions that take a
// scale, into LDS tiles that both products read.  e2m1 values times a power
// of two are exact in bf16.  The products are S^T = K Q^T (a lane holds one
// query row and 16 tokens of each 32) and O^T += V^T P^T, where P leaves S's
// registers without an exchange: the contraction's token order is the one
// that the lanes already hold.
//
// Softmax in base 2 on fp32 scores with a running maximum that only moves
// when a score passes it by 2^8, sums in fp32.  P is rounded to bf16 as a
// matrix operand (fp32 products would run at a sixteenth of the rate), the sum
// that divides it is not: an error of up to 2^-8 of each term, on top of the
// output's own rounding.  Where a few keys carry the softmax it shows: against
// 64 bits 0.0023 of the output's norm on single queries and short caches, 0.0017
// without it; 9360 queries joined with other keys 0.0017 either way.
//
// Many rows are bound by the matrix cores and the softmax between them (9360
// queries, 12 heads, 32760 tokens, d 128: 1.74 ms, 1.08 PFLOP/s), few rows by
// the cache's bytes (16 streams of one token, 40 over 8 heads, up to 32760
// tokens: 73 us, 3.9 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attend_parts.hpp"
#include "lds_stage.hpp"
#include "lowbit_args.hpp"
#include "lowbit_values.hpp"
#include "wave_ops.hpp"
#include "xcd.hpp"

namespace mssa {
namespace {

constexpr int kMaxWorkers = kMxAttnMaxWorkers;
// How the work is shared out, whatever the lengths are.  An item is the query
// rows of one block (a.items of them per sequence) against their sequence's
// whole context; all items' tiles stand in a row, sequence by sequence and
// item by item, and each worker takes as many of them as every other (or one
// more).  An item that one worker holds whole is written by it; the sums of
// one that several share go to slots, 2 i for the first item of worker i and
// 2 i + 1 for a later one (which then is its last), and a second launch joins
// them.  (All tiles of a call are fewer than 2^31: the plan's check.)
constexpr int kTile = kMxAttnTile;

__device__ inline int64_t tokens_of(const MxAttnArgs& a, int b) {
  const int64_t len = a.kv_len ? a.kv_len[b] : a.cache_tokens;
  return len < 0 ? 0 : len > a.cache_tokens ? a.cache_tokens : len;
}
__device__ inline int tiles_of(const MxAttnArgs& a, int b) { return static_cast<int>((tokens_of(a, b) + kTile - 1) / kTile); }

// The same for a sequence that the whole wave shares, in scalar registers (the
// loops' bounds and the last tile's mask are branches then, not lane masks).
__device__ inline int len_of(const MxAttnArgs& a, int b) { return __builtin_amdgcn_readfirstlane(static_cast<int>(tokens_of(a, b))); }
__device__ inline int tiles_in(int len) { return static_cast<int>((static_cast<int64_t>(len) + kTile - 1) / kTile); }

// Tokens of tile t below `end`, at most a tile's; none past it.
__device__ inline int left_of(int end, int t) {
  const int64_t left = end - static_cast<int64_t>(t) * kTile;
  return left > kTile ? kTile : left < 0 ? 0 : static_cast<int>(left);
}

// Tiles of the sequences before b, times the items of a sequence, and the
// shares.  Lengths are read 64 at a time: every lane of a wave calls these.
__device__ inline Shares shares_of(const MxAttnArgs& a, int b, uint32_t* before) {
  const int lane = threadIdx.x & 63;
  uint32_t all = 0, pre_b = 0;
  if (!a.kv_len || a.batch == 1) {
    const uint32_t one = tiles_in(len_of(a, 0));
    all = one * a.batch;
    pre_b = one * b;
  } else {
    for (int c = 0; c < a.batch; c += 64) {
      const uint32_t pre = wave_prefix(c + lane < a.batch ? tiles_of(a, c + lane) : 0);
      if (b >= c + 64)
        pre_b = all + __shfl(pre, 63);
      else if (b > c)
        pre_b = all + __shfl(pre, b - c - 1);
      all += __shfl(pre, 63);
    }
    all = uniform(all);
    pre_b = uniform(pre_b);
  }
  if (before) *before = pre_b * a.items;
  all *= a.items;
  return Shares::of(all, static_cast<uint32_t>(a.workers));
}
// The sequence, item and tile that tile x of all is.
struct Spot {
  int b, item, tile;
};
__device__ inline Spot locate(const MxAttnArgs& a, uint32_t x) {
  const int lane = threadIdx.x & 63;
  const uint32_t y = x / a.items;  // sequences' tiles before: the sequence holds tiles items * P .. of all
  uint32_t b = 0, t = tiles_in(len_of(a, 0)), base = 0;
  if (!a.kv_len || a.batch == 1) {
    b = y / t;
    base = t * b;
  } else {
    for (int c = 0; c < a.batch; c += 64) {
      const uint32_t mine = c + lane < a.batch ? tiles_of(a, c + lane) : 0;
      const uint32_t pre = wave_prefix(mine);
      const uint64_t past = __ballot(base + pre > y);
      if (past) {
        const int i = __builtin_ctzll(past);
        b = c + i;
        t = uniform(__shfl(mine, i));
        base = uniform(base + __shfl(pre, i) - t);
        break;
      }
      base += __shfl(pre, 63);
    }
  }
  const uint32_t in = x - base * a.items, item = in / t;
  return {static_cast<int>(uniform(b)), static_cast<int>(uniform(item)), static_cast<int>(uniform(in - item * t))};
}

// Row `row` of slot `slot`: its sums, and its maximum and sum of exponentials
// (behind all slots' sums).
__device__ inline float* slot_sums(const MxAttnArgs& a, int D, int64_t slot, int row) {
  return a.partial + (slot * a.slot_rows + row) * D;
}
__device__ inline float2* slot_stats(const MxAttnArgs& a, int D, int64_t slot, int row) {
  return reinterpret_cast<float2*>(a.partial + 2 * static_cast<int64_t>(a.workers) * a.slot_rows * D) + slot * a.slot_rows + row;
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

// Four dims d .. d + 3 of a row's result from its sums v, maximum m and sum l.
// The row's lse is written by the thread of d = 0: callers read prior_lse,
// which may be the same memory, before any thread of the row gets here (the
// threads of a row belong to one wave).
__device__ inline void write_joined(const MxAttnArgs& a, const RowPlace& at, float m, float l, float prior_lse, f32x4 v,
                                    int d) {
  const Joined w = join(a.prior_lse != nullptr, m, l, prior_lse);
  bf16x4 p = {}, u;
  if (a.prior_out) p = *reinterpret_cast<const bf16x4*>(static_cast<const __bf16*>(a.prior_out) + at.q + d);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float f = v[i] * w.own;
    // a prior without keys adds nothing, whatever it holds; one whose share is too small for fp32 still adds its NaNs
    if (a.prior_out && prior_lse != -INFINITY) f += w.prior * static_cast<float>(p[i]);
    u[i] = static_cast<__bf16>(f);
  }
  *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.out) + at.q + d) = u;
  if (a.lse && d == 0) a.lse[at.lse] = w.lse;
}

// `bytes` bytes from a wave-uniform address, for range-checked loads.
__device__ inline __amdgpu_buffer_rsrc_t range_of(const void* p, uint32_t bytes) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(static_cast<uint64_t>(hi) << 32 | lo), 0,
                                           __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

template <int NS>
__device__ inline auto load_codes(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  if constexpr (NS == 4)
    return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0);
  else
    return __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
}

// Order of a run of NM matrix instructions and their ND LDS reads: LEAD reads
// first, then a matrix instruction and its share of reads in turn.
template <int NM, int ND, int LEAD>
__device__ inline void interleave() {
  __builtin_amdgcn_sched_group_barrier(0x100, LEAD, 0);
#pragma unroll
  for (int i = 0; i < (ND - LEAD) / (ND / NM); ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, ND / NM, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, NM - (ND - LEAD) / (ND / NM), 0);
}

// Many rows.  A wave's tile is two phases: matrix instructions (O += V^T P of
// the tile before, then S = K Q^T), and vector work (softmax, and expanding
// the next tile's codes).  Eight waves are two groups, one wave of each per
// SIMD, and the second group runs one phase behind the first, so that a SIMD's
// matrix core and vector unit both have a wave at work; a barrier ends each
// phase.  The first group expands K, the second V.  Four waves (fewer rows)
// are one group that expands both; two such blocks share a CU.
//
// With phases counted from the first group's S of tile t in 2 t: K of tile t + 1
// is written in 2 t + 1 and read in 2 t + 2 and 2 t + 3, V of tile t + 1 written
// in 2 t + 2 (four waves: 2 t + 1) and read in 2 t + 4 and 2 t + 5, each into the
// buffer whose tile (two before) was last read in 2 t - 1 and 2 t + 1 (2 t).
template <int D, int NW>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2))) void attn_kernel(MxAttnArgs a) {
  constexpr int KS = D / 16, DB = D / 32, NS = D / 32, kTileElems = kTile * 128;  // 256-byte rows for both D
  constexpr int NP = NW == 8 ? 1 : 2;  // operands (K, V) that a thread expands
  typedef uint32_t codes_t __attribute__((ext_vector_type(NS)));
  __shared__ __attribute__((aligned(16))) __bf16 lds[2][2][kTileElems];  // [buffer][K | V]

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), second = NW == 8 ? wave >> 2 : 0;
  const int tiles_r = a.items / a.kv_heads;
  // Workers next to one another share key heads: each XCD takes a run of them.
  const int worker = xcd_remap(blockIdx.x, gridDim.x);
  Spot at{worker / a.items, worker % a.items, 0};
  int todo = 0;  // tiles
  if (a.workers) {
    const Shares sh = shares_of(a, 0, nullptr);
    if (static_cast<uint32_t>(worker) >= sh.workers) return;
    const uint32_t x0 = sh.first(worker);
    todo = static_cast<int>(uniform(sh.first(worker + 1) - x0));
    at = locate(a, x0);
  }

  // 256 threads expand an operand's tile: four neighbours a token, D / 4 values
  // each.  Sixteen lanes take tokens 0, 4, 8, 12 of sixteen, whose swizzles
  // differ where their quarters' chunks agree: no bank conflicts.
  const uint32_t token_rows = static_cast<uint32_t>(a.kv_heads);
  const int tok = (wave & 3) * 16 + ((lane >> 2) & 3) * 4 + (lane >> 4), quarter = lane & 3;
  const uint32_t c_off = tok * token_rows * (D / 2) + quarter * (D / 8);
  const uint32_t e_off = tok * token_rows * DB + quarter * (D / 4) / 32;
  const int dst = swz256(tok, quarter * (D / 4));
  const float c = a.scale_log2e;
  const int k_rd = swz256(n, hh * 8);
  const int t_row = 4 * (lane >> 5) + ((lane & 15) >> 2);
  const int t_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  // The end of a phase.  Codes on their way to registers need not have arrived.
  auto phase_end = [&]() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  for (int seg = 0;; ++seg) {
    const int len = len_of(a, at.b), nt = tiles_in(len);
    const int kvh = at.item / tiles_r, rt = at.item - kvh * tiles_r;
    const int t0 = at.tile, t1 = a.workers && todo < nt - t0 ? t0 + todo : nt;
    const bool whole = t0 == 0 && t1 == nt;
    todo -= t1 - t0;

    // Reads past the sequence's last token return zeros: codes of zeros.
    codes_t codes[NP];
    uint32_t se[NP];
    const int64_t row0 = static_cast<int64_t>(at.b) * a.cache_tokens * a.kv_heads + kvh;
    auto fetch = [&](int t) {
      const int64_t first = row0 + static_cast<int64_t>(t) * kTile * a.kv_heads;
      const int left = left_of(len, t);
      const uint32_t rows = left ? (left - 1) * token_rows + 1 : 0u;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const bool is_v = NW == 8 ? second != 0 : i == 1;
        codes[i] = load_codes<NS>(range_of(static_cast<const char*>(is_v ? a.vc : a.kc) + first * (D / 2), rows * (D / 2)), c_off);
        se[i] = __builtin_amdgcn_raw_buffer_load_b8(
            range_of(static_cast<const char*>(is_v ? a.vs : a.ks) + first * DB, rows * DB), e_off, 0, 0);
      }
    };
    auto put = [&](int buf) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const float f = mx_scale(se[i]);
        __bf16* P = lds[buf][NW == 8 ? second : i];
#pragma unroll
        for (int k = 0; k < NS; ++k) *reinterpret_cast<bf16x8*>(P + (dst ^ (k * 8))) = expand_e2m1(codes[i][k], f);
      }
    };
    if (t0 < t1) fetch(t0);

    const int r_in = wave * 32 + n, r = rt * (NW * 32) + r_in;
    const bool ok = r < a.rows;
    const RowPlace row = row_place(a, at.b, kvh, ok ? r : 0, D);
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 v = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(a.q) + row.q + ks * 16 + hh * 8);
      qf[ks] = ok ? v : bf16x8{};
    }

    f32x16 o[DB], s[2];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x16{};
    float m = kNoMax, l = 0.f;  // running maximum (base 2), this lane's share of the sum
    bf16x8 pb[2][2];
    auto add_pv = [&](int buf) {
      const __bf16* Vs = lds[buf][1];
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
      // operand reads a few products ahead, not all of them at once (registers)
      interleave<DB * 4, DB * 8, DB * 3>();
    };
    auto scores = [&](int buf) {
      const __bf16* Ks = lds[buf][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        s[kb] = f32x16{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(Ks + kb * 32 * 128 + (k_rd ^ (ks * 16))),
                                                          qf[ks], s[kb], 0, 0, 0);
      }
      interleave<KS * 2, KS * 2, 6>();
    };
    auto softmax = [&](int t) {
      const int left = left_of(len, t);
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
    };

    if (t0 < t1) {
      if (seg > 0) phase_end();  // the last item's V has been read by all
      put(0);
      if (t0 + 1 < t1) fetch(t0 + 1);
      phase_end();
      if (second) phase_end();
      for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        // the wave whose turn at the matrix core it is goes first elsewhere too
        __builtin_amdgcn_s_setprio(1);
        if (t > t0) add_pv(buf ^ 1);
        scores(buf);
        __builtin_amdgcn_s_setprio(0);
        phase_end();
        softmax(t);
        if (t + 1 < t1) {
          put(buf ^ 1);
          if (t + 2 < t1) fetch(t + 2);
        }
        phase_end();
      }
      add_pv((t1 - 1 - t0) & 1);
      if (NW == 8 && !second) phase_end();
    }
    l += other_half(l);
    // dims 32 db + 8 j + 4 hh .. + 3 of the row
    if (ok && !whole) {
      const int64_t slot = 2 * static_cast<int64_t>(worker) + (seg > 0);
      float* P = slot_sums(a, D, slot, r_in);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = o[db][4 * j + i];
          *reinterpret_cast<f32x4*>(P + db * 32 + 8 * j + 4 * hh) = v;
        }
      if (hh == 0) *slot_stats(a, D, slot, r_in) = make_float2(m, l);
    } else if (ok) {
      const float prior = a.prior_lse ? a.prior_lse[row.lse] : 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = o[db][4 * j + i];
          write_joined(a, row, m, l, prior, v, db * 32 + 8 * j + 4 * hh);
        }
    }
    if (todo <= 0) return;
    at.tile = 0;
    do {  // the next item that has tiles (there is one: tiles are left to do)
      if (++at.item == a.items) {
        at.item = 0;
        ++at.b;
      }
    } while (len_of(a, at.b) == 0);
  }
}

// Few query rows: single tokens of a stream, or of a group of heads.  Memory
// bound (the cache is read once, 0.53 bytes a value), so a wave works alone on
// tiles of 64 tokens, with the next tile's codes on their way.  RT x 16 rows.
// K needs no LDS: in the 16x16x32 products a lane's share of a token (D / 4
// consecutive values) is read and expanded in place, and the queries' dims are
// permuted alike.  V is expanded into a tile of the wave's own in LDS and read
// transposed.
//
// The heads of a token lie side by side, 64 or 32 bytes of codes each, so a
// block's waves take neighbouring key heads of the same tokens (head_waves of
// them, the rest other tokens): whole cache lines are used at once.  An item is
// a whole sequence, its heads' blocks side by side.
constexpr int kFewWaves = kMxAttnFewWaves;

template <int D, int RT>
__global__ __launch_bounds__(kFewWaves * 64) __attribute__((amdgpu_waves_per_eu(2))) void few_rows_kernel(MxAttnArgs a) {
  constexpr int NS = D / 32, DT = D / 16, kRows = 16 * RT;
  typedef uint32_t codes_t __attribute__((ext_vector_type(NS)));
  __shared__ __attribute__((aligned(16))) __bf16 lds[kFewWaves][32 * 128];
  __shared__ float stat[2][kFewWaves][kRows];

  const int head_blocks = a.kv_heads / a.head_waves;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hw = wave % a.head_waves, tw = wave / a.head_waves, token_waves = kFewWaves / a.head_waves;
  // Blocks go to the 8 XCDs in turn: a worker's head blocks share an XCD and its L2.
  const int j = blockIdx.x / 8, worker = j / head_blocks * 8 + blockIdx.x % 8;
  const int kvh = j % head_blocks * a.head_waves + hw;
  int b = worker;
  int tile = 0;  // the sequence's first tile here
  int todo = 0;  // tiles
  if (a.workers) {
    const Shares sh = shares_of(a, 0, nullptr);
    if (static_cast<uint32_t>(worker) >= sh.workers) return;
    const uint32_t x0 = sh.first(worker);
    todo = static_cast<int>(uniform(sh.first(worker + 1) - x0));
    const Spot at = locate(a, x0);
    b = at.b;
    tile = at.tile;
  } else if (b >= a.batch) {
    return;
  }
  const float c = a.scale_log2e;
  __bf16* V = lds[wave];
  const int t_row = 4 * g + (n >> 2), t_col = 4 * (n & 3);
  const uint32_t token_rows = static_cast<uint32_t>(a.kv_heads);
  const uint32_t c_off = n * token_rows * (D / 2) + g * (D / 8), e_off = lane * token_rows * (D / 32);
  // This lane's scale of token 16 u + n, from the lane that holds the token's.
  const int e_shift = g * (D / 4) / 32 * 8;
  auto scale_of = [&](uint32_t e, int u) {
    const uint32_t all = __builtin_amdgcn_ds_bpermute((u * 16 + n) * 4, static_cast<int>(e));
    return mx_scale((all >> e_shift) & 255u);
  };

  for (int seg = 0;; ++seg) {
    const int len = len_of(a, b), nt = tiles_in(len);
    const int tile1 = a.workers && todo < nt - tile ? tile + todo : nt;
    const bool whole = tile == 0 && tile1 == nt;
    const int end = tile1 < nt ? tile1 * kTile : len;
    todo -= tile1 - tile;

    bf16x8 qf[RT][NS];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = t * 16 + n;
      const RowPlace at = row_place(a, b, kvh, r < a.rows ? r : 0, D);
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const bf16x8 v = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(a.q) + at.q + g * (D / 4) + s * 8);
        qf[t][s] = r < a.rows ? v : bf16x8{};
      }
    }

    // A tile's codes: lane (n, g) holds share g of tokens 16 u + n.  Its scales
    // come as one load: lane i holds all of token i's (bytes), which the lanes
    // exchange when the tile is used.  Reads past the piece's last token return
    // zeros: codes that stand for zeros.
    codes_t kc[kTile / 16], vc[kTile / 16];
    uint32_t ke = 0, ve = 0;
    const int64_t row0 = static_cast<int64_t>(b) * a.cache_tokens * a.kv_heads + kvh;
    auto fetch = [&](codes_t (&codes)[kTile / 16], uint32_t& e, const void* code_base, const void* scale_base, int t) {
      const int left = left_of(end, t);
      const uint32_t rows = left ? (left - 1) * token_rows + 1 : 0u;
      const int64_t row = row0 + static_cast<int64_t>(t) * kTile * a.kv_heads;
      const auto rc = range_of(static_cast<const char*>(code_base) + row * (D / 2), rows * (D / 2));
      const auto re = range_of(static_cast<const char*>(scale_base) + row * (D / 32), rows * (D / 32));
#pragma unroll
      for (int u = 0; u < kTile / 16; ++u) codes[u] = load_codes<NS>(rc, c_off + u * 16 * token_rows * (D / 2));
      if constexpr (NS == 4)
        e = __builtin_amdgcn_raw_buffer_load_b32(re, e_off, 0, 0);
      else
        e = __builtin_amdgcn_raw_buffer_load_b16(re, e_off, 0, 0);
    };
    f32x4 o[RT][DT];
    float m[RT], l[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      m[t] = kNoMax;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[t][d] = f32x4{};
    }
    constexpr int NU = kTile / 16;
    fetch(kc, ke, a.kc, a.ks, tile + tw);
    fetch(vc, ve, a.vc, a.vs, tile + tw);
    for (int t64 = tile + tw; t64 < tile1; t64 += token_waves) {
      f32x4 s[RT][NU];
#pragma unroll
      for (int u = 0; u < NU; ++u) {
#pragma unroll
        for (int t = 0; t < RT; ++t) s[t][u] = f32x4{};
        const float f = scale_of(ke, u);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const bf16x8 kv = expand_e2m1(kc[u][i], f);
#pragma unroll
          for (int t = 0; t < RT; ++t) s[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv, qf[t][i], s[t][u], 0, 0, 0);
        }
      }
      const int left = left_of(end, t64);
      fetch(kc, ke, a.kc, a.ks, t64 + token_waves);  // past the end: nothing is read
      bf16x8 pb[RT][NU / 2];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if (left < kTile) {
#pragma unroll
          for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (u * 16 + 4 * g + i >= left) s[t][u][i] = -INFINITY;
        }
        float mx = s[t][0][0];
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[t][u][i]);
        mx = over_row(mx, [](float x, float y) { return fmaxf(x, y); }) * c;
        if (__any(mx > m[t] + kRescaleLog2)) {
          const float mn = fmaxf(m[t], mx);
          const float alpha = __builtin_amdgcn_exp2f(m[t] - mn);
          m[t] = mn;
          l[t] *= alpha;
#pragma unroll
          for (int d = 0; d < DT; ++d) o[t][d] *= alpha;
        }
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][u][i], c, -m[t]));
            l[t] += p;
            pb[t][u / 2][u % 2 * 4 + i] = static_cast<__bf16>(p);
          }
      }
      // V in halves of 32 tokens through the wave's tile.  A wave's LDS accesses
      // happen in their order; the fences keep the compiler to it.
#pragma unroll
      for (int w = 0; w < NU / 2; ++w) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float f = scale_of(ve, w * 2 + u);
#pragma unroll
          for (int i = 0; i < NS; ++i)
            *reinterpret_cast<bf16x8*>(V + swz256(u * 16 + n, g * (D / 4) + i * 8)) = expand_e2m1(vc[w * 2 + u][i], f);
        }
        if (w == NU / 2 - 1) fetch(vc, ve, a.vc, a.vs, t64 + token_waves);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(V + swz256(t_row, d * 16 + t_col)));
          const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(V + swz256(t_row + 16, d * 16 + t_col)));
          const bf16x8 vt = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
          for (int t = 0; t < RT; ++t) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pb[t][w], o[t][d], 0, 0, 0);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }

    // Join the waves of a head: their maximum, then the scaled sums one by one.
#pragma unroll
    for (int t = 0; t < RT; ++t) l[t] = over_row(l[t], [](float x, float y) { return x + y; });
    if (token_waves > 1) {
#pragma unroll
      for (int t = 0; t < RT; ++t)
        if (g == 0) {
          stat[0][wave][t * 16 + n] = m[t];
          stat[1][wave][t * 16 + n] = l[t];
        }
      __syncthreads();
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float top = m[t];
        for (int w = 0; w < token_waves; ++w) top = fmaxf(top, stat[0][w * a.head_waves + hw][t * 16 + n]);
        const float alpha = __builtin_amdgcn_exp2f(m[t] - top);
        m[t] = top;
        l[t] = 0.f;
        for (int w = 0; w < token_waves; ++w) {
          const int i = w * a.head_waves + hw;
          l[t] = __builtin_fmaf(__builtin_amdgcn_exp2f(stat[0][i][t * 16 + n] - top), stat[1][i][t * 16 + n], l[t]);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) o[t][d] *= alpha;
      }
      f32x4* O = reinterpret_cast<f32x4*>(&lds[0][0]) + hw * (RT * DT * 64) + lane;
      static_assert(2 * RT * DT * 64 * 16 <= static_cast<int>(sizeof(lds)), "two heads' sums fit the V tiles' place");
      for (int w = 1; w < token_waves; ++w) {
        if (tw == w) {
#pragma unroll
          for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int d = 0; d < DT; ++d) O[(t * DT + d) * 64] = o[t][d];
        }
        __syncthreads();
        if (tw == 0) {
#pragma unroll
          for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int d = 0; d < DT; ++d) o[t][d] += O[(t * DT + d) * 64];
        }
        __syncthreads();
      }
    }
    // dims 16 d + 4 g .. + 3 of row 16 t + n
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = t * 16 + n;
      if (r >= a.rows || tw > 0) continue;
      if (!whole) {
        const int64_t slot = 2 * static_cast<int64_t>(worker) + (seg > 0);
        float* P = slot_sums(a, D, slot, kvh * a.rows + r);
#pragma unroll
        for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(P + d * 16 + 4 * g) = o[t][d];
        if (g == 0) *slot_stats(a, D, slot, kvh * a.rows + r) = make_float2(m[t], l[t]);
      } else {
        const RowPlace at = row_place(a, b, kvh, r, D);
        const float prior = a.prior_lse ? a.prior_lse[at.lse] : 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) write_joined(a, at, m[t], l[t], prior, o[t][d], d * 16 + 4 * g);
      }
    }
    if (todo <= 0) return;
    tile = 0;
    do ++b;
    while (len_of(a, b) == 0);  // there is one: tiles are left to do
  }
}

// Join the slots of the items that several workers shared, and write the rows
// of sequences without tokens.  D / 4 threads side by side on a row's dims.
// Items in many slots (few rows, long contexts): a row at a time, the groups
// of threads on different slots; else a row per group.  Fixed orders.
constexpr int kJoinThreads = kMxAttnJoinThreads;

template <int D>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(MxAttnArgs a, int block_rows, int row_groups, int first) {
  constexpr int kSide = D / 4, kGroups = kJoinThreads / kSide;
  __shared__ float weight[kMaxWorkers];
  __shared__ f32x4 part[kGroups][kSide];
  __shared__ float red[2][kJoinThreads / 64];
  const int tid = threadIdx.x, wave = tid >> 6, side = tid % kSide, grp = tid / kSide;
  const int block = first + static_cast<int>(blockIdx.x);
  const int unit = block / row_groups, rg = block - unit * row_groups;
  const int b = unit / a.items, item = unit - b * a.items;
  uint32_t start;
  const Shares sh = shares_of(a, b, &start);
  const uint32_t nt = tiles_in(len_of(a, b));
  start += item * nt;
  // the workers that took the item's first and last tile
  const int64_t w0 = nt ? sh.worker_of(start) : 0, w1 = nt ? sh.worker_of(start + nt - 1) : 0;
  if (nt && w0 == w1) return;
  const int pieces = nt ? static_cast<int>(w1 - w0) + 1 : 0;
  const int64_t slot0 = nt && sh.first(w0) != start ? 2 * w0 + 1 : 2 * w0;
  auto slot = [&](int s) { return s == 0 ? slot0 : 2 * (w0 + s); };
  const int tiles_r = a.items / a.kv_heads;  // 0: an item is a sequence, rows are (key head, row)
  auto place = [&](int in, bool* ok) {
    const int kvh = tiles_r ? item / tiles_r : in / a.rows;
    const int r = tiles_r ? (item - kvh * tiles_r) * a.slot_rows + in : in - kvh * a.rows;
    *ok = r < a.rows && kvh < a.kv_heads;
    return row_place(a, b, kvh, *ok ? r : 0, D);
  };
  const int r0 = rg * block_rows;
  if (pieces <= kSide && block_rows > 1) {
    for (int k = grp; k < block_rows; k += kGroups) {
      bool ok;
      const RowPlace at = place(r0 + k, &ok);
      if (!ok) continue;  // all threads of the row
      // thread `side` holds slot side's statistics, then its weight
      const float2 mine = side < pieces ? *slot_stats(a, D, slot(side), r0 + k) : make_float2(kNoMax, 0.f);
      float m = mine.x;
#pragma unroll
      for (int d = 1; d < kSide; d *= 2) m = fmaxf(m, __shfl_xor(m, d, kSide));
      const float f = __builtin_amdgcn_exp2f(mine.x - m);
      float l = f * mine.y;
#pragma unroll
      for (int d = 1; d < kSide; d *= 2) l += __shfl_xor(l, d, kSide);
      f32x4 v = {};
      for (int s0 = 0; s0 < pieces; s0 += 4) {
        f32x4 part[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int s = min(s0 + u, pieces - 1);
          part[u] = *reinterpret_cast<const f32x4*>(slot_sums(a, D, slot(s), r0 + k) + side * 4);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (s0 + u < pieces) v += part[u] * __shfl(f, s0 + u, kSide);
      }
      write_joined(a, at, m, l, a.prior_lse ? a.prior_lse[at.lse] : 0.f, v, side * 4);
    }
    return;
  }
  for (int k = 0; k < block_rows; ++k) {
    bool ok;
    const RowPlace at = place(r0 + k, &ok);
    if (!ok) continue;  // the whole block
    float2 mine[kMaxWorkers / kJoinThreads];
    float m = kNoMax, l = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxWorkers / kJoinThreads; ++i) {
      const int s = tid + i * kJoinThreads;
      mine[i] = s < pieces ? *slot_stats(a, D, slot(s), r0 + k) : make_float2(kNoMax, 0.f);
      m = fmaxf(m, mine[i].x);
    }
    m = wave_fmax(m);
    if ((tid & 63) == 0) red[0][wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinThreads / 64; ++w) m = fmaxf(m, red[0][w]);
#pragma unroll
    for (int i = 0; i < kMaxWorkers / kJoinThreads; ++i) {
      const float f = __builtin_amdgcn_exp2f(mine[i].x - m);
      weight[tid + i * kJoinThreads] = f;
      l = __builtin_fmaf(f, mine[i].y, l);
    }
    l = wave_sum(l);
    if ((tid & 63) == 0) red[1][wave] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinThreads / 64; ++w) l += red[1][w];
    f32x4 v = {};
#pragma unroll 4
    for (int s = grp; s < pieces; s += kGroups)
      v += *reinterpret_cast<const f32x4*>(slot_sums(a, D, slot(s), r0 + k) + side * 4) * weight[s];
    part[grp][side] = v;
    __syncthreads();
    if (grp == 0) {
#pragma unroll
      for (int i = 1; i < kGroups; ++i) v += part[i][side];
      write_joined(a, at, m, l, a.prior_lse ? a.prior_lse[at.lse] : 0.f, v, side * 4);
    }
    __syncthreads();
  }
}

template <int D>
hipError_t attn_dim(const MxAttnArgs& a, const MxAttnPlan& plan, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(plan.blocks));
  if (plan.waves == 0 && a.rows <= 16)
    hipLaunchKernelGGL((few_rows_kernel<D, 1>), grid, dim3(kFewWaves * 64), 0, stream, a);
  else if (plan.waves == 0)
    hipLaunchKernelGGL((few_rows_kernel<D, 2>), grid, dim3(kFewWaves * 64), 0, stream, a);
  else if (plan.waves == 4)
    hipLaunchKernelGGL((attn_kernel<D, 4>), grid, dim3(4 * 64), 0, stream, a);
  else
    hipLaunchKernelGGL((attn_kernel<D, 8>), grid, dim3(8 * 64), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.workers == 0) return e;
  const int row_groups = plan.slot_rows / plan.join_rows;
  constexpr int64_t kSlice = kLaunchThreads / kJoinThreads;
  for (int64_t first = 0; first < plan.join_blocks; first += kSlice) {
    hipLaunchKernelGGL((join_kernel<D>), dim3(static_cast<uint32_t>(std::min(kSlice, plan.join_blocks - first))),
                       dim3(kJoinThreads), 0, stream, a, plan.join_rows, row_groups, static_cast<int>(first));
    if (const hipError_t joined = hipGetLastError(); joined != hipSuccess) return joined;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_mx_attention(const MxAttnArgs& a, const MxAttnPlan& plan, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? attn_dim<128>(a, plan, stream) : attn_dim<64>(a, plan, stream);
}

}  // namespace mssa
