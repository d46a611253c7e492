// Kernel arguments and launchers of the operators for streams served together
// (projection with adapters, append to a paged cache, attention over it), and
// the rules on sizes that need no device.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "lowbit_args.hpp"

namespace mssa {

// n / d for n < 2^31, by a multiplication: with 2^(l-1) < d <= 2^l and
// m = floor(2^(31+l) / d) + 1, m d exceeds 2^(31+l) by at most 2^l, too little
// to reach the next quotient.
struct Divisor {
  uint32_t d, m;
  int32_t shift;
  static Divisor of(uint32_t d) {
    int l = 0;
    while ((uint64_t{1} << l) < d) ++l;
    return {d, static_cast<uint32_t>((uint64_t{1} << (31 + l)) / d + 1), 31 + l};
  }
  MSSA_HOST_DEVICE uint32_t quotient(uint32_t n) const { return static_cast<uint32_t>(static_cast<uint64_t>(n) * m >> shift); }
};

// Row `first` of sequence b's chunk and the row behind its last, whatever
// chunk_begin holds: inside [0, tokens], none where it decreases.
struct ChunkRows {
  int32_t first, end;
  MSSA_HOST_DEVICE static ChunkRows of(const int32_t* begin, int32_t b, int32_t each, int32_t tokens) {
    if (!begin) return {b * each, (b + 1) * each};
    auto in = [&](int32_t r) { return r < 0 ? 0 : r > tokens ? tokens : r; };
    const int32_t first = in(begin[b]), end = in(begin[b + 1]);
    return {first, end < first ? first : end};
  }
};

// ----------------------------------------------------------------- append
constexpr int kAppendThreads = 256;
constexpr int kAppendMaxTokens = 16;  // tokens of a block
constexpr int kAppendMaxPairs = 128;  // rotated pairs of a head

struct AppendArgs {
  const void *q, *k, *v;
  const int32_t *chunk_begin, *kv_len, *page_table, *positions;
  const float* freqs;
  void *q_out, *k_pages, *v_pages;
  int64_t q_stride, k_stride, v_stride, pages;
  int32_t tokens, token0, token1;  // rows in all; rows of this launch
  int32_t batch, each;             // each: rows of a sequence without chunk_begin
  int32_t q_heads, kv_heads, head_dim, table_pages;
  int32_t pairs, halves, axis_end[2];  // rotated pairs; first pair of the second and third axis
  int32_t block_tokens;
  Divisor page, units, head_units;  // units: pieces of 16 values of a token's heads (q, k, v); of a head
};

// Tokens of a block: a static rule on the sizes.
int32_t append_block_tokens(int64_t tokens, int32_t units);
hipError_t launch_paged_append(const AppendArgs& a, hipStream_t stream);

// -------------------------------------------------------------- attention
constexpr int kPagedTile = 64;  // tokens of a tile
constexpr int kPagedMaxWorkers = 512;
constexpr int kPagedJoinThreads = 256;

struct PagedAttnArgs {
  const void *q, *k_pages, *v_pages, *prior_out;
  const int32_t *chunk_begin, *kv_len, *page_table;
  const float* prior_lse;
  void* out;
  float *lse, *partial;
  int64_t q_stride, lse_stride, pages, capacity;  // capacity: tokens that a row of the table can name
  int32_t tokens, batch, each, max_chunk;
  int32_t q_heads, kv_heads, group, table_pages;
  int32_t mask_block;  // at most 2^30: no chunk is longer
  int32_t slot_shift;  // an item has 2^slot_shift query rows
  int32_t workers;     // shares of all items' contexts, 0: an item a block and no joining launch
  int32_t unit_shift;  // a tile weighs 2^unit_shift units
  int32_t extra;       // tiles that an item weighs besides its own: what beginning and ending one takes
  int32_t least;       // units of a share at least
  Divisor page, by_group, by_mask;
  float scale_log2e;
  MSSA_HOST_DEVICE int32_t slot_rows() const { return 1 << slot_shift; }
};

// One sequence's work.  Its query rows (chunk token, head of the group) that
// share a key head are cut into items of slot_rows rows; an item reads the
// tiles up to the last index that its last row sees.  Items are weighed in
// units of a fraction of a tile, linear in their number so that sums have a
// closed form: their tiles where there is no mask, and where there is one, up to
// its steps.  Every item has units, also one without keys, whose rows are
// written all the same: beginning and ending an item takes as long as some tiles.
struct PagedSeq {
  int32_t first, n;  // chunk: first row, tokens (at most max_chunk)
  int32_t len;       // cache indices in use
  int32_t start;     // cache index of the chunk's first token (negative where the cache is shorter than the chunk)
  int32_t rows, items;
  uint32_t cost0, step;  // item i weighs cost0 + i step

  // Cache indices below this one are seen by chunk token i.
  MSSA_HOST_DEVICE int32_t seen(int32_t i, const PagedAttnArgs& a) const {
    if (!a.mask_block) return len;
    const int64_t end = static_cast<int64_t>(start) + (a.by_mask.quotient(i) + 1) * static_cast<uint32_t>(a.mask_block);
    return end < 0 ? 0 : end < len ? static_cast<int32_t>(end) : len;
  }
  MSSA_HOST_DEVICE int32_t tiles(int32_t item, const PagedAttnArgs& a) const {
    const int32_t past = (item + 1) << a.slot_shift, last = (past < rows ? past : rows) - 1;
    const uint32_t end = a.mask_block ? seen(a.by_group.quotient(last), a) : len;
    return static_cast<int32_t>((end + (kPagedTile - 1)) / kPagedTile);
  }
  MSSA_HOST_DEVICE uint32_t cost(int32_t item) const { return cost0 + static_cast<uint32_t>(item) * step; }
  // Units of a key head's items before this one (all of a call's are fewer than
  // 2^31, so that the items' pairs are where step is not 0).
  MSSA_HOST_DEVICE uint32_t before(int32_t item) const {
    const uint32_t i = static_cast<uint32_t>(item);
    return i * cost0 + (step ? i * (i - 1) / 2 * step : 0);
  }
  // The item that unit x of a key head belongs to.
  MSSA_HOST_DEVICE int32_t item_of(uint32_t x) const {
    if (!step) return static_cast<int32_t>(x / cost0);
    int32_t lo = 0, hi = items - 1;
    while (lo < hi) {
      const int32_t mid = lo + (hi - lo + 1) / 2;
      if (before(mid) <= x)
        lo = mid;
      else
        hi = mid - 1;
    }
    return lo;
  }
  MSSA_HOST_DEVICE static PagedSeq of(const PagedAttnArgs& a, int32_t b) {
    PagedSeq s;
    const ChunkRows c = ChunkRows::of(a.chunk_begin, b, a.each, a.tokens);
    const int32_t held = a.kv_len[b], all = held < 0 ? 0 : held, n = c.end - c.first;  // an empty cache is seen by none
    s.first = c.first;
    s.start = all - n;
    s.n = n < a.max_chunk ? n : a.max_chunk;
    s.len = all < a.capacity ? all : static_cast<int32_t>(a.capacity);
    s.rows = s.n * a.group;
    s.items = (s.rows + a.slot_rows() - 1) >> a.slot_shift;
    s.cost0 = 1;
    s.step = 0;
    if (a.workers && s.items) {
      s.cost0 = static_cast<uint32_t>(s.tiles(0, a) + a.extra) << a.unit_shift;
      if (a.mask_block && s.items > 1) {
        const uint32_t high = static_cast<uint32_t>(s.tiles(s.items - 1, a) + a.extra) << a.unit_shift;
        if (high > s.cost0) s.step = (high - s.cost0) / static_cast<uint32_t>(s.items - 1);
      }
    }
    return s;
  }
  MSSA_HOST_DEVICE uint32_t head_units() const { return before(items); }
  // First tile of unit u (of cost) of an item with `tiles` tiles: u tiles / cost,
  // rounded the same way wherever it is asked for; all of them at u = cost.
  MSSA_HOST_DEVICE static int32_t tile_at(uint32_t u, int32_t tiles, uint32_t cost) {
    return static_cast<int32_t>(static_cast<double>(u) * static_cast<double>(tiles) / static_cast<double>(cost));
  }
};

struct PagedAttnPlan {
  int32_t waves;      // 32 rows each in a block; 0: the kernel for few rows
  int32_t few_waves;  // of a block of that one
  int32_t slot_rows, workers, unit_shift, extra, least;
  int64_t blocks, workspace_bytes;
  int32_t join_rows;  // rows of a block of the joining launch
  int32_t threads() const { return (waves ? waves : few_waves) * 64; }
};
// Sizes whose launch would have 2^32 threads, or 2^31 units, are refused.
hipError_t plan_paged_attention(int64_t tokens, int32_t batch, int32_t max_chunk, int32_t q_heads, int32_t kv_heads,
                                int32_t head_dim, int64_t capacity, PagedAttnPlan* plan);
hipError_t launch_paged_attention(const PagedAttnArgs& a, const PagedAttnPlan& plan, int head_dim, hipStream_t stream);

// ---------------------------------------------------------------- project
struct AdapterArgs {
  const void *x, *w, *bias, *a, *b;
  const int32_t *segment_begin, *adapter;
  const float* scale;
  void* low;  // [M, parts, low_rank] bf16: the rows' low-rank factors, times scale
  void* y[kMaxParts];
  int64_t x_stride;
  int32_t M, N, K;
  int32_t parts, split;  // split: features of a part
  int32_t segments, adapters, rank, low_rank;
  float part0_scale;
  // whole, aligned chunks of 16 bytes: the rows of x, w and a; of b; of the outputs
  bool whole, whole_b, whole_y;
};

// Which kernel makes a product: the one for few tokens, or one of three tile
// sizes (tokens and features).
enum class AdapterKernel { kFew, kTiles64, kTiles128, kTiles256 };
constexpr int kAdapterFewTokens = 64, kAdapterFewFeatures = 32;
constexpr int kAdapterFewOdd = 16;  // tokens whose odd rows are read where they lie

constexpr int kLowRows = 16, kLowManyRows = 64;  // rows of a tile of the low-rank factor
struct AdapterPlan {
  AdapterKernel kernel;
  int32_t groups;       // of waves of a small tile, which share out the contraction
  bool pack_x, pack_w;  // rows of x, and of w and a, are copied to whole chunks first (for few tokens only rows of fewer than 8 values)
  int32_t low_rows;     // of a tile of the low-rank factor's launch
  int32_t low_rank;     // rank rounded up to whole 16 values
  int64_t low_tiles;    // its row tiles, 0: none
  int32_t low_columns;  // rank columns of a block: 16 beside 16 rows; 32, 64 or 96 beside 64
  int32_t low_across;   // blocks of a row tile: the grid's second axis with 16 rows, along the first with 64
  int64_t blocks;       // of the product
  int64_t low_bytes, workspace_bytes;  // the low-rank factors, then the copies
};
hipError_t plan_adapter_project(int64_t rows, int32_t in_features, int64_t x_stride, int32_t out_features, int32_t parts,
                                int32_t segments, int32_t adapters, int32_t rank, AdapterPlan* plan);
hipError_t launch_adapter_project(const AdapterArgs& a, const AdapterPlan& plan, hipStream_t stream);

}  // namespace mssa
