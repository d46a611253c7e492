// Attention of chunks of new tokens over paged K/V caches
// (mssa_paged_attention).
//
// The query rows of a sequence that share a key head (chunk tokens x heads of
// the group) are cut into items; the cache is read in tiles of 64 tokens,
// whose rows are found one by one in the page table (a page may end anywhere
// inside a tile).  The products are S^T = K Q^T (a lane holds one query row)
// and O^T += V^T P^T, where P leaves S's registers without an exchange: the
// contraction's token order is the one that the lanes already hold.  Softmax in
// base 2 on fp32 scores with a running maximum that only moves when a score
// passes it by 2^8, sums in fp32.  P is rounded to bf16 as a matrix operand (up
// to 2^-8 of each term; fp32 products would run at a sixteenth of the rate),
// the sum that divides it is not.
//
// Tokens past the sequence's last, and those whose page is none, are read from
// a row of zeros and masked.  A token that some rows see and others do not (the
// mask's steps) has P = 0 for the latter, which an infinity or a NaN among its
// values would turn into a NaN: in tiles with such a step the products take
// zeros for them, and they are added apart, to the rows that see them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attend_parts.hpp"
#include "lds_stage.hpp"
#include "paged_args.hpp"
#include "wave_ops.hpp"
#include "xcd.hpp"
#include "zero_row.hpp"

namespace mssa {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = kPagedTile;
constexpr uint64_t kAll = ~uint64_t{0};

// -------------------------------------------------------------- sharing out
// All items stand in a row, sequence by sequence, key head by key head, item by
// item, each as long as it weighs (PagedSeq), and each worker takes as many
// units as every other (or one more).  An item that one worker holds whole is
// written by it; the sums of one that several share go to slots, 2 i for the
// first item of worker i and 2 i + 1 for a later one (which then is its last),
// and a second launch joins them.

__device__ inline uint32_t units_of(const PagedAttnArgs& a, const PagedSeq& s) {
  return s.head_units() * static_cast<uint32_t>(a.kv_heads);
}

// A value of lane i, in a scalar register.
template <class T>
__device__ inline T from_lane(T v, int i) {
  return static_cast<T>(__builtin_amdgcn_readlane(static_cast<int>(v), i));
}
__device__ inline PagedSeq from_lane(const PagedSeq& s, int i) {
  return {from_lane(s.first, i), from_lane(s.n, i),     from_lane(s.len, i),   from_lane(s.start, i),
          from_lane(s.rows, i),  from_lane(s.items, i), from_lane(s.cost0, i), from_lane(s.step, i)};
}
__device__ inline PagedSeq sequence(const PagedAttnArgs& a, int b) { return from_lane(PagedSeq::of(a, b), 0); }

// Unit x of all: its sequence, key head and item, and its place in the item.
// Where chunk_begin decreases somewhere, chunks overlap and sums can pass 32
// bits: what is not found then, or lies past its sequence, is no work (b < 0).
struct Spot {
  int b, kvh, item;
  uint32_t unit;
  PagedSeq seq;
};

// The shares of all units and the spot of the first unit of worker `w` (of no
// share: b < 0).  Sequences are read 64 at a time, a lane each; every lane of a
// wave calls this.
__device__ inline Spot find_share(const PagedAttnArgs& a, uint32_t w, Shares* sh) {
  const int lane = threadIdx.x & 63;
  uint32_t all = 0, mine = 0, pre = 0;
  PagedSeq s{};
  auto read = [&](int c) {
    mine = 0;
    if (c + lane < a.batch) {
      s = PagedSeq::of(a, c + lane);
      mine = units_of(a, s);
    }
    pre = wave_prefix(mine);
  };
  for (int c = 0; c < a.batch; c += 64) {
    read(c);
    all += from_lane(pre, 63);
  }
  if (!a.workers) {
    *sh = Shares::of(all, all);  // a unit an item, an item a block
  } else {
    const uint32_t most = all / static_cast<uint32_t>(a.least), workers = static_cast<uint32_t>(a.workers);
    *sh = Shares::of(all, most < 1 ? 1 : most < workers ? most : workers);
  }
  Spot at{};
  at.b = -1;
  if (w >= sh->workers) return at;
  const uint32_t x = uniform(sh->first(w));
  uint32_t base = 0;
  for (int c = 0; c < a.batch; c += 64) {
    if (a.batch > 64) read(c);  // else read above
    const uint64_t past = __ballot(base + pre > x);
    if (past) {
      const int i = __builtin_ctzll(past);
      const uint32_t units = from_lane(mine, i), y = x - (base + from_lane(pre, i) - units);
      if (y >= units) break;
      at.b = c + i;
      at.seq = from_lane(s, i);
      const uint32_t of_head = at.seq.head_units();
      at.kvh = static_cast<int>(y / of_head);
      const uint32_t z = y - static_cast<uint32_t>(at.kvh) * of_head;
      at.item = at.seq.item_of(z);
      at.unit = z - at.seq.before(at.item);
      break;
    }
    base += from_lane(pre, 63);
  }
  return at;
}
// The item after this one; whether there is one.
__device__ inline bool next_item(const PagedAttnArgs& a, Spot* at) {
  at->unit = 0;
  if (++at->item < at->seq.items) return true;
  at->item = 0;
  if (++at->kvh < a.kv_heads) return true;
  at->kvh = 0;
  do {
    if (++at->b >= a.batch) return false;
    at->seq = sequence(a, at->b);
  } while (at->seq.items == 0);
  return true;
}

// Row `row` of slot `slot`: its sums, and its maximum and sum of exponentials
// (behind all slots' sums).
__device__ inline float* slot_sums(const PagedAttnArgs& a, int D, int64_t slot, int row) {
  return a.partial + (slot * a.slot_rows() + row) * D;
}
__device__ inline float2* slot_stats(const PagedAttnArgs& a, int D, int64_t slot, int row) {
  return reinterpret_cast<float2*>(a.partial + 2 * static_cast<int64_t>(a.workers) * a.slot_rows() * D) + slot * a.slot_rows() + row;
}

// Where query row r of a key head lies, and which cache indices it sees.
struct RowPlace {
  int64_t q, out, lse;
  int32_t seen;
};
__device__ inline RowPlace row_place(const PagedAttnArgs& a, const PagedSeq& s, int kvh, int r, int D) {
  const int i = static_cast<int>(a.by_group.quotient(r)), h = kvh * a.group + (r - i * a.group);
  const int64_t row = static_cast<int64_t>(s.first) + i;
  return {row * a.q_stride + static_cast<int64_t>(h) * D, (row * a.q_heads + h) * D, h * a.lse_stride + row,
          s.seen(i, a)};
}

// Four dims d .. d + 3 of a row's result from its sums v, maximum m and sum l.
// The row's lse is written by the thread of d = 0: callers read prior_lse,
// which may be the same memory, before any thread of the row gets here (the
// threads of a row belong to one wave).
__device__ inline void write_joined(const PagedAttnArgs& a, const RowPlace& at, float m, float l, float prior_lse, f32x4 v,
                                    int d) {
  const Joined w = join(a.prior_lse != nullptr, m, l, prior_lse);
  bf16x4 p = {}, u;
  if (a.prior_out) p = *reinterpret_cast<const bf16x4*>(static_cast<const __bf16*>(a.prior_out) + at.out + d);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float f = v[i] * w.own;
    // a prior without keys adds nothing, whatever it holds; one whose share is too small for fp32 still adds its NaNs
    if (a.prior_out && prior_lse != -INFINITY) f += w.prior * static_cast<float>(p[i]);
    u[i] = static_cast<__bf16>(f);
  }
  *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.out) + at.out + d) = u;
  if (a.lse && d == 0) a.lse[at.lse] = w.lse;
}

// The pages of one sequence.
struct PageWalk {
  const int32_t* table;
  uint32_t len;  // at least 1 where a tile is looked up
  int64_t pages;
  Divisor page;
};
__device__ inline PageWalk walk_of(const PagedAttnArgs& a, int b, int len) {
  return {a.page_table + static_cast<int64_t>(b) * a.table_pages, static_cast<uint32_t>(len), a.pages, a.page};
}

// Lane `from`'s value.
__device__ inline int32_t of_lane(int32_t v, int from) { return __builtin_amdgcn_ds_bpermute(from * 4, v); }

// Infinities and NaN of two bf16 values, zeros elsewhere.
__device__ inline uint32_t wild_of(uint32_t two) {
  return ((two & 0x7f80u) == 0x7f80u ? two & 0xffffu : 0u) | ((two & 0x7f800000u) == 0x7f800000u ? two & 0xffff0000u : 0u);
}

// v without its infinities and NaN; `wild` collects their bits.
__device__ inline bf16x8 tamed(bf16x8 v, uint32_t* wild) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = wild_of(w[i]);
    *wild |= x;
    w[i] ^= x;
  }
  return __builtin_bit_cast(bf16x8, w);
}

// ------------------------------------------------------------------ many rows
// A wave's tile is two phases: matrix instructions (O += V^T P of the tile
// before, then S = K Q^T), and the softmax.  Eight waves are two groups, one
// wave of each per SIMD, and the second group runs one phase behind the first,
// so that a SIMD's matrix core and vector unit both have a wave at work; a
// barrier ends each phase.  Tiles come by direct transfers, issued in the
// softmax phase and waited for at its end: the first group brings K, the second
// V.  Four waves (fewer rows) are one group that brings both; two such blocks
// share a CU.  The first kLead operands of a matrix phase are read at the end of
// the softmax phase before it, the others kLead ahead.
//
// With phases counted from the first group's S of tile t in 2 t: K of tile t + 1
// is brought in 2 t + 1 and read in 2 t + 2 and 2 t + 3, V of tile t + 1 brought
// in 2 t + 2 (four waves: 2 t + 1) and read in 2 t + 3 to 2 t + 5, each into the
// buffer whose tile (two before) was last read in 2 t - 1 and 2 t + 1 (2 t).
//
// Bound by the matrix cores' and the vector unit's phases, which are about as long
// as each other: 32 matrix instructions a wave and tile (a thousand cycles of the
// core) against 32 exponentials a lane with their scaling, sums and packing.  12
// heads of 4680 over 37440 tokens: 1.03 ms, 1.05 PFLOP/s (a large product reaches
// 1.2), the matrix cores busy 58 % of the time; three streams of 12 heads with up
// to 9360 tokens in frames of 1560 over up to 23400: 2.25 ms, 0.95 PFLOP/s, 52 %;
// 16 heads of 8192 over 32768, whose items fill their blocks: 1.1 to 1.15.  Tiles
// of 64 tokens and 32 rows a wave: sums, scores and queries then take the
// registers that two waves a SIMD leave each.
//
// The maximum is taken only where a lane's 32 exponentials against the running
// one pass 2^8 in sum (no single one can have stayed below): most tiles spend
// a fused multiply-add, an exponential and an addition per score.
constexpr int kLead = 4;
constexpr float kRescaleSum = 256.f;  // 2^kRescaleLog2

template <int D, int NW, bool MASK>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_kernel(PagedAttnArgs a) {
  constexpr int KS = D / 16, DB = D / 32, kTileElems = kTile * 128;  // 256-byte rows for both D
  using T_ = std::true_type;
  using F_ = std::false_type;
  __shared__ __attribute__((aligned(16))) __bf16 lds[2][2][kTileElems];  // [K | V][buffer]
  __shared__ const char* where[2][2][NW * kTile];                        // [run & 1][K | V][token]
  __shared__ uint64_t masks[2][NW];
  __shared__ int32_t entries[NW * kTile];

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), second = NW == 8 ? wave >> 2 : 0;
  // Workers next to one another share key heads: each XCD takes a run of them.
  const int worker = xcd_remap(blockIdx.x, gridDim.x);
  Shares sh;
  Spot at = find_share(a, worker, &sh);
  if (at.b < 0) return;
  uint32_t todo = uniform(sh.first(worker + 1) - sh.first(worker));

  // Transfers: wave instruction i fills four rows of 256 bytes, lane l bytes 16 l,
  // i.e. row l / 16, whose chunk l % 16 holds chunk (l % 16) ^ 4 (l / 16) ^ i.
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&lds[0][0][0]));
  const uint32_t entries0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&entries[0]));
  const uint32_t row_bytes = static_cast<uint32_t>(a.kv_heads) * D * 2;
  const float c = a.scale_log2e;
  // Operands: K rows 32 kb + n, columns 16 ks + 8 hh; V rows R + t_row (+ 8 for
  // the upper half), columns 32 db + t_col, R a multiple of 16.
  const int k_rd = swz256(n, hh * 8);
  const int t_row = 4 * (lane >> 5) + ((lane & 15) >> 2);
  const int t_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  int v_rd[DB][2];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int h = 0; h < 2; ++h) v_rd[db][h] = swz256(t_row + 8 * h, db * 32 + t_col);
  auto phase_end = [&]() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  for (int seg = 0;; ++seg) {
    const int tiles = at.seq.tiles(at.item, a);
    const uint32_t cost = at.seq.cost(at.item), take = todo < cost - at.unit ? todo : cost - at.unit;
    const int t0 = __builtin_amdgcn_readfirstlane(PagedSeq::tile_at(at.unit, tiles, cost));
    const int t1 = __builtin_amdgcn_readfirstlane(PagedSeq::tile_at(at.unit + take, tiles, cost));
    const bool whole = take == cost;
    todo -= take;

    const int len = at.seq.len;
    const PageWalk walk = walk_of(a, at.b, len);
    const char* const k_base = static_cast<const char*>(a.k_pages) + static_cast<int64_t>(at.kvh) * D * 2;
    const char* const v_base = static_cast<const char*>(a.v_pages) + static_cast<int64_t>(at.kvh) * D * 2;
    // Where the tokens' rows lie: `where` holds the addresses of K and V for two
    // runs of NW tiles, a thread a token and a wave a tile, of zeros for tokens
    // that are not there; `masks` has a bit for those that are.  The page table's
    // entries of the run after this one come by direct transfers at its first tile,
    // and are turned into addresses at the second: the loop itself, whose vector
    // unit the softmax fills, only reads them.
    auto run_token = [&](int run) { return static_cast<uint32_t>(t0 + run * NW) * kTile + tid; };
    auto ask_run = [&](int run) {
      const uint32_t tok = min(run_token(run), walk.len - 1);
      gdma4(walk.table + walk.page.quotient(tok), __builtin_amdgcn_readfirstlane(entries0 + wave * 256));
    };
    auto make_run = [&](int run) {
      const int32_t found = entries[tid];
      const uint32_t tok = min(run_token(run), walk.len - 1);
      const bool is = run_token(run) < walk.len && found >= 0 && found < walk.pages;
      const uint64_t row = static_cast<uint32_t>(found) * walk.page.d + (tok - walk.page.quotient(tok) * walk.page.d);
      where[run & 1][0][tid] = is ? k_base + row * row_bytes : reinterpret_cast<const char*>(zero_row);
      where[run & 1][1][tid] = is ? v_base + row * row_bytes : reinterpret_cast<const char*>(zero_row);
      const uint64_t mask = __ballot(is);
      if (lane == 0) masks[run & 1][wave] = mask;
    };
    // A wave brings rows 16 (wave & 3) .. + 15 of its group's tiles.  Their addresses
    // and the tile's mask are read before the matrix phase, which has room for
    // it, and used in the softmax phase after it.
    const char* place[NW == 8 ? 4 : 8];
    uint64_t there_next = 0;
    auto look = [&](int t) {
      const int half = (t - t0) / NW & 1, in = (t - t0) % NW;
      int ln = lane;  // the chunks are worked out anew: kept, they would cost more registers than there are
      asm volatile("" : "+v"(ln));
#pragma unroll
      for (int is_v = 0; is_v < 2; ++is_v) {
        if (NW == 8 && is_v) break;
        const char* const* const from = &where[half][NW == 8 ? second : is_v][in * kTile + (wave & 3) * 16 + (ln >> 4)];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // 64-dim rows are half as long: their chunks fill the LDS rows' unused half too
          const int chunk = ((ln & 15) ^ ((ln >> 4) << 2) ^ i) & (D / 8 - 1);
          place[is_v * 4 + i] = from[i * 4] + chunk * 16;
        }
      }
      there_next = masks[half][in];
    };
    auto bring = [&](int buf) {
#pragma unroll
      for (int is_v = 0; is_v < 2; ++is_v) {
        if (NW == 8 && is_v) break;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          gdma16(place[is_v * 4 + i], __builtin_amdgcn_readfirstlane(
              lds0 + (((NW == 8 ? second : is_v) * 2 + buf) * kTile + (wave & 3) * 16 + i * 4) * 256));
      }
    };
    auto scalar_mask = [&]() {
      return static_cast<uint64_t>(uniform(static_cast<uint32_t>(there_next >> 32))) << 32 | uniform(static_cast<uint32_t>(there_next));
    };

    const int r_in = wave * 32 + n, r = at.item * (NW * 32) + r_in;
    const bool ok = r < at.seq.rows;
    int seen = len;
    bf16x8 qf[KS];
    {
      const RowPlace row = row_place(a, at.seq, at.kvh, ok ? r : 0, D);
      if (MASK && ok) seen = row.seen;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 v = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(a.q) + row.q + ks * 16 + hh * 8);
        qf[ks] = ok ? v : bf16x8{};
      }
    }

    f32x16 o[DB], s[2];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x16{};
    float m = kNoMax, l = 0.f;  // running maximum (base 2), this lane's share of the sum
    bf16x8 pb[2][2], ring[kLead];

    // Operand i of a matrix phase: with pv the V^T operands of O += P V (key block
    // kb, 16-key half cc, dims db), then the K operands of S (k-step ks, kb).
    auto operand = [&](auto pv, int i, int vb, int kbuf) -> bf16x8 {
      constexpr int NPV = decltype(pv)::value ? 4 * DB : 0;
      if (i < NPV) {
        const int db = i % DB;
        const __bf16* r0 = &lds[1][vb][(i / DB) * 16 * 128];
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(r0 + v_rd[db][0]));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(r0 + v_rd[db][1]));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
      const int j = i - NPV, ks = j / 2, kb = j % 2;
      return *reinterpret_cast<const bf16x8*>(&lds[0][kbuf][kb * 32 * 128 + (k_rd ^ (ks * 16))]);
    };
    auto prefill = [&](auto pv, int vb, int kbuf) {
#pragma unroll
      for (int i = 0; i < kLead; ++i) ring[i] = operand(pv, i, vb, kbuf);
    };
    auto mstep = [&](auto pv, auto sc, int vb, int kbuf) {
      constexpr int NPV = decltype(pv)::value ? 4 * DB : 0, N = NPV + (decltype(sc)::value ? KS * 2 : 0);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const bf16x8 av = ring[i % kLead];
        if (i < NPV) {
          const int st = i / DB, db = i % DB;
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, pb[st >> 1][st & 1], o[db], 0, 0, 0);
        } else {
          const int j = i - NPV, ks = j / 2, kb = j % 2;
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, qf[ks], ks == 0 ? f32x16{} : s[kb], 0, 0, 0);
        }
        if (i + kLead < N) ring[i % kLead] = operand(pv, i + kLead, vb, kbuf);
      }
      // each read kLead instructions before its use: a V operand is two reads
#pragma unroll
      for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (i + kLead < N) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        if (i + kLead < NPV) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    // O += P V of tile t, which may have a step of the mask: without its infinities
    // and NaN.  Those are noted, token by token, for the rows that see them: a bit
    // for each of the lane's sums that they send up and one for down, both for a
    // NaN.
    uint64_t up = 0, down = 0;
    auto add_pv_step = [&](int vb, int t) {
      uint32_t wild = 0;
      int at_row = t_row;
      asm volatile("" : "+v"(at_row));  // addresses of this path's own: none is kept from outside it
#pragma unroll
      for (int i = 0; i < 4 * DB; ++i) {
        const int db = i % DB, st = i / DB;
        const __bf16* r0 = &lds[1][vb][st * 16 * 128];
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(r0 + swz256(at_row, db * 32 + t_col)));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(r0 + swz256(at_row + 8, db * 32 + t_col)));
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tamed(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), &wild),
                                                        pb[st >> 1][st & 1], o[db], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (!__any(wild != 0)) return;
#pragma unroll 1
      for (int tok = 0; tok < kTile; ++tok) {
        int half = hh;
        asm volatile("" : "+v"(half));
        const __bf16* V = lds[1][vb];
        const uint32_t two = *reinterpret_cast<const uint32_t*>(V + swz256(tok, (lane * 2) & (D - 1)));
        if (!__any(wild_of(two) != 0)) continue;
        // P of the token, from the half wave that holds it
        float p = 0.f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (kb * 32 + 8 * (e >> 2) + (e & 3) == (tok & ~4)) p = static_cast<float>(pb[kb][e >> 3][e & 7]);
        p = __shfl(p, n + 32 * (tok >> 2 & 1));
        const bool sees = t * kTile + tok < seen, some = p > 0.f;
#pragma unroll 1
        for (int q = 0; q < DB * 4; ++q) {
          const uint2 v = *reinterpret_cast<const uint2*>(V + swz256(tok, q * 8 + 4 * half));
          uint32_t u = 0, d = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = (i < 2 ? v.x : v.y) >> (16 * (i & 1)) & 0xffffu;
            const bool is = sees && (x & 0x7f80u) == 0x7f80u, both = (x & 0x7fu) || !some;
            u |= is && (both || !(x & 0x8000u)) ? 1u << i : 0u;
            d |= is && (both || (x & 0x8000u)) ? 1u << i : 0u;
          }
          up |= static_cast<uint64_t>(u) << (4 * q);
          down |= static_cast<uint64_t>(d) << (4 * q);
        }
      }
    };
    // masked: the tile may have a step of the mask
    auto softmax = [&](auto masked, int t, uint64_t there) {
      // token kb * 32 + 8 (e / 4) + 4 hh + e % 4 of the tile in s[kb][e]
      if (there != kAll) {
        const uint64_t mine = there >> (4 * hh);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!(mine >> (kb * 32 + 8 * (e >> 2) + (e & 3)) & 1)) s[kb][e] = -INFINITY;
      }
      if constexpr (decltype(masked)::value) {
        const int left = seen - t * kTile - 4 * hh;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (kb * 32 + 8 * (e >> 2) + (e & 3) >= left) s[kb][e] = -INFINITY;
      }
      auto exps = [&]() {
        float ls[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][e], c, -m));
            const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][e + 1], c, -m));
            ls[(e >> 1) & 3] += p0 + p1;
            pb[kb][e >> 3][e & 7] = static_cast<__bf16>(p0);
            pb[kb][e >> 3][(e & 7) + 1] = static_cast<__bf16>(p1);
          }
        return (ls[0] + ls[1]) + (ls[2] + ls[3]);
      };
      float lt = exps();
      if (__any(!(lt <= kRescaleSum))) {  // also true for infinite and NaN sums
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
        lt = exps();
      }
      l += lt;
      // the exponentials stay in this phase: they are not to sink into the matrix phase
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int h = 0; h < 2; ++h) asm volatile("" : "+v"(pb[kb][h]));
      asm volatile("" : "+v"(l));
    };

    if (t0 < t1) {
      if (seg > 0) phase_end();  // the last item's V has been read by all
      ask_run(0);
      wait_vmcnt<0>();
      asm volatile("" ::: "memory");
      make_run(0);
      phase_end();
      look(t0);
      bring(0);
      uint64_t there = scalar_mask();
      wait_vmcnt<0>();
      phase_end();
      if (second) phase_end();
      // The softmax phase of tile t in buffer buf: the next tile comes, the first
      // operands of the next matrix phase are read.
      auto sphase = [&](auto masked, auto next, int t, int buf) {
        phase_end();
        if (t + 1 < t1) bring(buf ^ 1);
        const int in = (t - t0) % NW;
        if (in == 0 && t + NW < t1)
          ask_run((t - t0) / NW + 1);
        else if (in == 1 && t + NW - 1 < t1)
          make_run((t - t0) / NW + 1);
        softmax(masked, t, there);
        there = scalar_mask();
        if constexpr (decltype(next)::value) prefill(T_{}, buf, buf ^ 1);
        wait_vmcnt<0>();
        phase_end();
      };
      // The matrix phase that makes tile t's scores.
      auto mphase = [&](auto pv, auto sc, int t, int vb, int kbuf) {
        __builtin_amdgcn_s_setprio(2);
        if (decltype(sc)::value && t + 1 < t1) look(t + 1);
        mstep(pv, sc, vb, kbuf);
        __builtin_amdgcn_s_setprio(0);
      };
      // Tiles before `plain` have no step of the mask, for no row of the item.
      int plain = t1;
      if constexpr (MASK) {
        const int low = at.seq.seen(a.by_group.quotient(at.item * (NW * 32)), a);
        if (low < len && low / kTile < plain) plain = low / kTile > t0 ? low / kTile : t0;
      }
      prefill(F_{}, 0, 0);
      mphase(F_{}, T_{}, t0, 0, 0);
      // two tiles at a time: their buffers are constants
      int t = t0, buf = 0;
      for (; t + 2 < plain; t += 2) {
        sphase(F_{}, T_{}, t, 0);
        mphase(T_{}, T_{}, t + 1, 0, 1);
        sphase(F_{}, T_{}, t + 1, 1);
        mphase(T_{}, T_{}, t + 2, 1, 0);
      }
      if constexpr (!MASK) {
        if (t + 1 < t1) {
          sphase(F_{}, T_{}, t, 0);
          mphase(T_{}, T_{}, t + 1, 0, 1);
          buf = 1;
          ++t;
        }
        sphase(F_{}, T_{}, t, buf);
        mphase(T_{}, F_{}, t + 1, buf, buf ^ 1);
      } else {
        for (;; ++t, buf ^= 1) {
          sphase(T_{}, F_{}, t, buf);
          __builtin_amdgcn_s_setprio(2);
          add_pv_step(buf, t);
          if (t + 1 < t1) {
            if (t + 2 < t1) look(t + 2);
            prefill(F_{}, 0, buf ^ 1);
            mstep(F_{}, T_{}, 0, buf ^ 1);
          }
          __builtin_amdgcn_s_setprio(0);
          if (t + 1 == t1) break;
        }
      }
      if (NW == 8 && !second) phase_end();
    }
    l += other_half(l);
    if constexpr (MASK) {
      if (__any((up | down) != 0)) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            if (up >> (db * 16 + e) & 1) o[db][e] += INFINITY;
            if (down >> (db * 16 + e) & 1) o[db][e] -= INFINITY;
          }
      }
    }
    // dims 32 db + 8 j + 4 hh .. + 3 of the row
    if (ok) {
      const RowPlace row = row_place(a, at.seq, at.kvh, r, D);
      const int64_t slot = 2 * static_cast<int64_t>(worker) + (seg > 0);
      float* P = whole ? nullptr : slot_sums(a, D, slot, r_in);
      const float prior = whole && a.prior_lse ? a.prior_lse[row.lse] : 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = o[db][4 * j + i];
          const int d = db * 32 + 8 * j + 4 * hh;
          if (whole)
            write_joined(a, row, m, l, prior, v, d);
          else
            *reinterpret_cast<f32x4*>(P + d) = v;
        }
      if (!whole && hh == 0) *slot_stats(a, D, slot, r_in) = make_float2(m, l);
    }
    if (todo == 0 || !next_item(a, &at)) return;
  }
}

// ------------------------------------------------------------------- few rows
// Single tokens of a stream, or a few: at most RT x 16 rows share a key head.
// Memory bound (the cache is read once), so a wave works alone, without barriers,
// on every kFewWaves-th stage of 32 tokens of the block's.  K, V and the page table's
// entries come by direct transfers into rings of the wave's own in LDS, whole
// cache lines and streamed (nt): two stages of K and V on their way, entries two
// stages ahead of them.  The transfers in order, stage by stage: K, V, entries of
// the stage after the next; what a step needs is there once no more than those
// issued after it are left.  Stages past the last are transfers of zeros.
//
// 16 streams of one token, 8 key heads, 1 to 32760 tokens, 1.07 GB: 186 us, 5.8 TB/s
// (half lines a request: 5.4 at most, streamed ones 4.3; whole lines without nt
// 5.8; whole streamed lines with nothing else to do 6.5).
constexpr int kFewStage = 32;  // tokens

template <int D, int RT, bool MASK, int kFewWaves>
__global__ __launch_bounds__(kFewWaves * 64) void few_rows_kernel(PagedAttnArgs a) {
  constexpr int NS = D / 32, DT = D / 16, kRows = 16 * RT, kHalf = kFewStage * 256, kMoves = kFewStage / 4;
  __shared__ __attribute__((aligned(16))) char lds[kFewWaves][2][2][kHalf];  // [wave][buffer][K | V]
  __shared__ int32_t entries[kFewWaves][4][64];
  __shared__ float stat[2][kFewWaves][kRows];

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int worker = xcd_remap(blockIdx.x, gridDim.x);
  Shares sh;
  Spot at = find_share(a, worker, &sh);
  if (at.b < 0) return;
  uint32_t todo = uniform(sh.first(worker + 1) - sh.first(worker));

  const int64_t row_bytes = static_cast<int64_t>(a.kv_heads) * D * 2;
  const float c = a.scale_log2e;
  const int t_row = 4 * g + (n >> 2), t_col = 4 * (n & 3);
  const int t_lc = (lane & 15) ^ ((lane >> 4) << 2);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&lds[wave][0][0][0]));
  const uint32_t ent0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&entries[wave][0][0]));

  for (int seg = 0;; ++seg) {
    const int tiles = at.seq.tiles(at.item, a);
    const uint32_t cost = at.seq.cost(at.item), take = todo < cost - at.unit ? todo : cost - at.unit;
    const int t0 = __builtin_amdgcn_readfirstlane(PagedSeq::tile_at(at.unit, tiles, cost));
    const int t1 = __builtin_amdgcn_readfirstlane(PagedSeq::tile_at(at.unit + take, tiles, cost));
    const bool whole = take == cost;
    todo -= take;
    const int len = at.seq.len;
    const int32_t* const table = a.page_table + static_cast<int64_t>(at.b) * a.table_pages;
    const char* const k_base = static_cast<const char*>(a.k_pages) + static_cast<int64_t>(at.kvh) * D * 2;
    const char* const v_base = static_cast<const char*>(a.v_pages) + static_cast<int64_t>(at.kvh) * D * 2;
    // This wave's stages: first, first + kFewWaves, .. below last (of the context's).
    constexpr int kPer = kTile / kFewStage;
    const int first = t0 * kPer + wave, last = t1 * kPer;
    const int count = first < last ? (last - first + kFewWaves - 1) / kFewWaves : 0;

    // Lane i (and i + 32) looks token i of a stage up; past the last stage the
    // sequence's last token, whose place is not used.
    auto token = [&](int st) {
      const uint32_t tok = static_cast<uint32_t>(first + st * kFewWaves) * kFewStage + (lane & 31);
      return tok < static_cast<uint32_t>(len) ? tok : static_cast<uint32_t>(len) - 1;
    };
    auto ask = [&](int st) {
      gdma4(table + a.page.quotient(token(st)), __builtin_amdgcn_readfirstlane(ent0 + (st & 3) * 256));
    };
    auto row_of = [&](int st, uint32_t* there) {
      const int32_t found = entries[wave][st & 3][lane];
      const uint32_t tok = token(st);
      const bool ok = st < count && static_cast<uint32_t>(first + st * kFewWaves) * kFewStage + (lane & 31) < static_cast<uint32_t>(len) &&
                      found >= 0 && found < a.pages;
      *there = static_cast<uint32_t>(__ballot(ok));
      return ok ? found * static_cast<int32_t>(a.page.d) + static_cast<int32_t>(tok - a.page.quotient(tok) * a.page.d) : -1;
    };
    auto bring = [&](int32_t row, int buf, int is_v) {
#pragma unroll
      for (int i = 0; i < kMoves; ++i) {
        const int chunk = t_lc ^ (i & 3);
        const int32_t r = of_lane(row, i * 4 + (lane >> 4));
        const bool there = r >= 0 && (D == 128 || chunk < D / 8);
        const char* p = (is_v ? v_base : k_base) + static_cast<int64_t>(r) * row_bytes + chunk * 16;
        gdma16_nt(there ? p : reinterpret_cast<const char*>(zero_row) + chunk * 16,
                  __builtin_amdgcn_readfirstlane(lds0 + (buf * 2 + is_v) * kHalf + i * 1024));
      }
    };

    bool ok[RT];
    int seen[RT];
    bf16x8 qf[RT][NS];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = at.item * kRows + t * 16 + n;
      ok[t] = r < at.seq.rows;
      const RowPlace place = row_place(a, at.seq, at.kvh, ok[t] ? r : 0, D);
      seen[t] = MASK && ok[t] ? place.seen : len;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const bf16x8 v = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(a.q) + place.q + i * 32 + g * 8);
        qf[t][i] = ok[t] ? v : bf16x8{};
      }
    }
    f32x4 o[RT][DT];
    float m[RT], l[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      m[t] = kNoMax;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[t][d] = f32x4{};
    }
    uint32_t there[3];  // of this stage and the two after it
    if (count) {
      ask(0);
      ask(1);
      wait_vmcnt<0>();
      asm volatile("" ::: "memory");
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const int32_t row = row_of(st, &there[st]);
        bring(row, st, 0);
        bring(row, st, 1);
        ask(st + 2);
      }
    }
    for (int st = 0; st < count; ++st) {
      const __bf16* K = reinterpret_cast<const __bf16*>(lds[wave][st & 1][0]);
      const __bf16* V = reinterpret_cast<const __bf16*>(lds[wave][st & 1][1]);
      const int64_t tok0 = static_cast<int64_t>(first + st * kFewWaves) * kFewStage;
      // K is there: after it come V, entries, K, V, entries
      wait_vmcnt<3 * kMoves + 2>();
      asm volatile("" ::: "memory");
      f32x4 s[RT][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int t = 0; t < RT; ++t) s[t][u] = f32x4{};
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const bf16x8 k = *reinterpret_cast<const bf16x8*>(K + swz256(u * 16 + n, i * 32 + g * 8));
#pragma unroll
          for (int t = 0; t < RT; ++t) s[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[t][i], s[t][u], 0, 0, 0);
        }
      }
      // V and the entries of stage st + 2 are there, K has been read: after them come K, V, entries
      wait_vmcnt<2 * kMoves + 1>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      const int32_t row = row_of(st + 2, &there[2]);
      bring(row, st & 1, 0);
      bool step = false;
      bf16x8 pb[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        // token 16 u + 4 g + i of the stage in s[t][u][i]
        if (there[0] != ~0u) {
          const uint32_t mine = there[0] >> (4 * g);
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!(mine >> (u * 16 + i) & 1)) s[t][u][i] = -INFINITY;
        }
        if constexpr (MASK) {
          const int64_t left = seen[t] - tok0;
          if (__any(seen[t] < len && left < kFewStage)) {
            step = true;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (u * 16 + 4 * g + i >= left) s[t][u][i] = -INFINITY;
          }
        }
        float mx = s[t][0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
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
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][u][i], c, -m[t]));
            l[t] += p;
            pb[t][u * 4 + i] = static_cast<__bf16>(p);
          }
      }
      uint32_t wild = 0;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(V + swz256(t_row, d * 16 + t_col)));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(V + swz256(t_row + 16, d * 16 + t_col)));
        bf16x8 vt = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        if (MASK && step) vt = tamed(vt, &wild);
#pragma unroll
        for (int t = 0; t < RT; ++t) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pb[t], o[t][d], 0, 0, 0);
      }
      if (MASK && __any(wild != 0)) {
        // the infinities and NaN of the values, token by token, to the rows that see them
#pragma unroll 1
        for (int tok = 0; tok < kFewStage; ++tok) {
          const uint32_t two = *reinterpret_cast<const uint32_t*>(V + swz256(tok, (lane * 2) & (D - 1)));
          if (!__any(wild_of(two) != 0)) continue;
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            float p = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) p = (e >> 2) * 16 + 4 * g + (e & 3) == tok ? static_cast<float>(pb[t][e]) : p;
            p = __shfl(p, n + 16 * (tok >> 2 & 3));
            const bool sees = tok0 + tok < seen[t];
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              const bf16x4 v = *reinterpret_cast<const bf16x4*>(V + swz256(tok, d * 16 + 4 * g));
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float f = static_cast<float>(v[e]);
                o[t][d][e] += sees && !(__builtin_fabsf(f) < INFINITY) ? p * f : 0.f;
              }
            }
          }
        }
      }
      // V has been read
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      bring(row, st & 1, 1);
      ask(st + 4);
      there[0] = there[1];
      there[1] = there[2];
    }
    wait_vmcnt<0>();
    asm volatile("" ::: "memory");

    // Join the waves: their maximum, then the scaled sums one by one.
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      l[t] = over_row(l[t], [](float x, float y) { return x + y; });
      if (g == 0) {
        stat[0][wave][t * 16 + n] = m[t];
        stat[1][wave][t * 16 + n] = l[t];
      }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float top = m[t];
      for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, stat[0][w][t * 16 + n]);
      const float alpha = __builtin_amdgcn_exp2f(m[t] - top);
      m[t] = top;
      l[t] = 0.f;
      for (int w = 0; w < kFewWaves; ++w)
        l[t] = __builtin_fmaf(__builtin_amdgcn_exp2f(stat[0][w][t * 16 + n] - top), stat[1][w][t * 16 + n], l[t]);
#pragma unroll
      for (int d = 0; d < DT; ++d) o[t][d] *= alpha;
    }
    f32x4* O = reinterpret_cast<f32x4*>(&lds[0][0][0][0]) + lane;
    static_assert(RT * DT * 64 * 16 <= static_cast<int>(sizeof(lds)), "a wave's sums fit the V tiles' place");
    for (int w = 1; w < kFewWaves; ++w) {
      if (wave == w) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int d = 0; d < DT; ++d) O[(t * DT + d) * 64] = o[t][d];
      }
      __syncthreads();
      if (wave == 0) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int d = 0; d < DT; ++d) o[t][d] += O[(t * DT + d) * 64];
      }
      __syncthreads();
    }
    // dims 16 d + 4 g .. + 3 of row 16 t + n
    if (wave == 0) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if (!ok[t]) continue;
        const RowPlace place = row_place(a, at.seq, at.kvh, at.item * kRows + t * 16 + n, D);
        if (!whole) {
          const int64_t slot = 2 * static_cast<int64_t>(worker) + (seg > 0);
          float* P = slot_sums(a, D, slot, t * 16 + n);
#pragma unroll
          for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(P + d * 16 + 4 * g) = o[t][d];
          if (g == 0) *slot_stats(a, D, slot, t * 16 + n) = make_float2(m[t], l[t]);
        } else {
          const float prior = a.prior_lse ? a.prior_lse[place.lse] : 0.f;
#pragma unroll
          for (int d = 0; d < DT; ++d) write_joined(a, place, m[t], l[t], prior, o[t][d], d * 16 + 4 * g);
        }
      }
    }
    if (todo == 0 || !next_item(a, &at)) return;
  }
}

// ------------------------------------------------------------------- joining
// Blocks of worker boundary j (between workers j and j + 1) join the slots of
// the item that the boundary cuts, if worker j holds the item's first piece.
// D / 4 threads side by side on a row's dims.  Items in many slots (few rows,
// long contexts): a row at a time, the groups of threads on different slots;
// else a row per group.  Fixed orders.  Bound by the way from memory: 5.4 us for 255
// boundaries of single rows, 30 us for 255 boundaries of 256 rows, 67 MB of sums.
constexpr int kJoinThreads = kPagedJoinThreads;

template <int D>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(PagedAttnArgs a, int join_rows, int row_groups) {
  constexpr int kSide = D / 4, kGroups = kJoinThreads / kSide;
  __shared__ float weight[kPagedMaxWorkers];
  __shared__ f32x4 part[kGroups][kSide];
  __shared__ float red[2][kJoinThreads / 64];
  const int tid = threadIdx.x, wave = tid >> 6, side = tid % kSide, grp = tid / kSide;
  const int j = static_cast<int>(blockIdx.x) / row_groups, r0 = (static_cast<int>(blockIdx.x) - j * row_groups) * join_rows;
  Shares sh;
  const Spot at = find_share(a, j + 1, &sh);
  const uint32_t start = sh.first(j + 1) - at.unit;
  if (at.b < 0 || at.unit == 0 || sh.first(j) > start) return;
  const int w1 = static_cast<int>(min(sh.worker_of(start + at.seq.cost(at.item) - 1), sh.workers - 1));
  const int pieces = w1 - j + 1;
  const int64_t slot0 = sh.first(j) != start ? 2 * static_cast<int64_t>(j) + 1 : 2 * static_cast<int64_t>(j);
  auto slot = [&](int s) { return s == 0 ? slot0 : 2 * static_cast<int64_t>(j + s); };
  const int rows = min(a.slot_rows(), at.seq.rows - at.item * a.slot_rows()), r1 = min(r0 + join_rows, rows);
  auto place = [&](int in) { return row_place(a, at.seq, at.kvh, at.item * a.slot_rows() + in, D); };
  if (pieces <= kSide && join_rows > 1) {
    for (int k = r0 + grp; k < r1; k += kGroups) {
      const RowPlace to = place(k);
      // thread `side` holds slot side's statistics, then its weight
      const float2 mine = side < pieces ? *slot_stats(a, D, slot(side), k) : make_float2(kNoMax, 0.f);
      float m = mine.x;
#pragma unroll
      for (int d = 1; d < kSide; d *= 2) m = fmaxf(m, __shfl_xor(m, d, kSide));
      const float f = __builtin_amdgcn_exp2f(mine.x - m);
      float l = f * mine.y;
#pragma unroll
      for (int d = 1; d < kSide; d *= 2) l += __shfl_xor(l, d, kSide);
      f32x4 v = {};
      for (int s0 = 0; s0 < pieces; s0 += 4) {
        f32x4 some[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) some[u] = *reinterpret_cast<const f32x4*>(slot_sums(a, D, slot(min(s0 + u, pieces - 1)), k) + side * 4);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (s0 + u < pieces) v += some[u] * __shfl(f, s0 + u, kSide);
      }
      write_joined(a, to, m, l, a.prior_lse ? a.prior_lse[to.lse] : 0.f, v, side * 4);
    }
    return;
  }
  for (int k = r0; k < r1; ++k) {
    const RowPlace to = place(k);
    float2 mine[kPagedMaxWorkers / kJoinThreads];
    float m = kNoMax, l = 0.f;
#pragma unroll
    for (int i = 0; i < kPagedMaxWorkers / kJoinThreads; ++i) {
      const int s = tid + i * kJoinThreads;
      mine[i] = s < pieces ? *slot_stats(a, D, slot(s), k) : make_float2(kNoMax, 0.f);
      m = fmaxf(m, mine[i].x);
    }
    m = wave_fmax(m);
    if ((tid & 63) == 0) red[0][wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinThreads / 64; ++w) m = fmaxf(m, red[0][w]);
#pragma unroll
    for (int i = 0; i < kPagedMaxWorkers / kJoinThreads; ++i) {
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
      v += *reinterpret_cast<const f32x4*>(slot_sums(a, D, slot(s), k) + side * 4) * weight[s];
    part[grp][side] = v;
    __syncthreads();
    if (grp == 0) {
#pragma unroll
      for (int i = 1; i < kGroups; ++i) v += part[i][side];
      write_joined(a, to, m, l, a.prior_lse ? a.prior_lse[to.lse] : 0.f, v, side * 4);
    }
    __syncthreads();
  }
}

template <int D, bool MASK>
hipError_t attend(const PagedAttnArgs& a, const PagedAttnPlan& plan, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(plan.blocks)), block(plan.threads());
  if (plan.waves == 0 && plan.slot_rows == 16 && plan.few_waves == 4)
    hipLaunchKernelGGL((few_rows_kernel<D, 1, MASK, 4>), grid, block, 0, stream, a);
  else if (plan.waves == 0 && plan.slot_rows == 16)
    hipLaunchKernelGGL((few_rows_kernel<D, 1, MASK, 2>), grid, block, 0, stream, a);
  else if (plan.waves == 0 && plan.few_waves == 4)
    hipLaunchKernelGGL((few_rows_kernel<D, 2, MASK, 4>), grid, block, 0, stream, a);
  else if (plan.waves == 0)
    hipLaunchKernelGGL((few_rows_kernel<D, 2, MASK, 2>), grid, block, 0, stream, a);
  else if (plan.waves == 4)
    hipLaunchKernelGGL((attn_kernel<D, 4, MASK>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((attn_kernel<D, 8, MASK>), grid, block, 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.workers < 2) return e;
  const int row_groups = plan.slot_rows / plan.join_rows;
  hipLaunchKernelGGL((join_kernel<D>), dim3(static_cast<uint32_t>((plan.workers - 1) * row_groups)), dim3(kJoinThreads), 0,
                     stream, a, plan.join_rows, row_groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attention(const PagedAttnArgs& a, const PagedAttnPlan& plan, int head_dim, hipStream_t stream) {
  if (head_dim == 128) return a.mask_block ? attend<128, true>(a, plan, stream) : attend<128, false>(a, plan, stream);
  return a.mask_block ? attend<64, true>(a, plan, stream) : attend<64, false>(a, plan, stream);
}

}  // namespace mssa
