// How the operators for streams served together cut their work: static rules
// on sizes, no device code.
#include <algorithm>

#include "paged_args.hpp"

namespace mssa {

// A block's threads take four pieces of 16 values each at most; while there are
// blocks enough for two on every CU, several tokens share a block, its sines and
// its look-ups (4680 tokens of 12 heads: 19.1 us, 21.1 with two pieces a thread,
// 21.4 with ten).
int32_t append_block_tokens(int64_t tokens, int32_t units) {
  const int64_t most = std::min<int64_t>(std::max(1, 4 * kAppendThreads / units), kAppendMaxTokens);
  return static_cast<int32_t>(std::max<int64_t>(1, std::min(most, tokens / 512)));
}

hipError_t plan_paged_attention(int64_t tokens, int32_t batch, int32_t max_chunk, int32_t q_heads, int32_t kv_heads,
                                int32_t head_dim, int64_t capacity, PagedAttnPlan* plan) {
  PagedAttnPlan p{};
  const int64_t group = q_heads / kv_heads, rows = std::min<int64_t>(max_chunk, std::max<int64_t>(tokens, 1)) * group;
  // Up to 1536 rows blocks of four waves, two on a CU: an item's rows fit better
  // (391 causal tokens of 3 heads a key head, three streams: 35 us, 37 with eight
  // waves); above, eight waves share each tile (1800 tokens of 4 heads over 10800
  // tokens 70 us, 78 with four).
  p.waves = rows <= 32 ? 0 : rows <= 1536 ? 4 : 8;
  p.slot_rows = p.waves ? p.waves * 32 : rows <= 16 ? 16 : 32;
  // every sequence's items: whole ones, and one that is not full
  const int64_t items = kv_heads * std::min(batch * ((rows + p.slot_rows - 1) / p.slot_rows), batch + tokens * group / p.slot_rows);
  const int64_t tiles = (capacity + kPagedTile - 1) / kPagedTile;
  p.extra = p.waves ? 8 : 6;
  if (items > 0x7fffffff || items * (tiles + p.extra) > 0x7fffffff) return hipErrorInvalidValue;
  // Few rows: blocks of four waves, one on a CU; with several items a CU two of
  // two waves, one of which begins or ends an item while the other reads (256
  // streams of 8 key heads and 500 tokens 137 -> 87 us; one stream of 8 heads and
  // 32760 tokens 39.5 us, 49.5 with them, whose pieces are twice as many to join).
  p.few_waves = items >= 1024 ? 2 : 4;
  const int64_t slots = p.waves == 8 || (!p.waves && p.few_waves == 4) ? 256 : 512;  // blocks resident at once
  const int64_t least = p.waves ? 6 : 2 * p.few_waves;  // tiles of a share at least
  if (tiles > least) p.workers = static_cast<int32_t>(std::max<int64_t>(1, std::min(slots, items * tiles / least)));
  // units as small as 31 bits of them allow
  while (p.unit_shift < 4 && items * (tiles + p.extra) << (p.unit_shift + 1) <= 0x7fffffff) ++p.unit_shift;
  p.least = static_cast<int32_t>(least << p.unit_shift);
  p.blocks = p.workers ? p.workers : items;
  if (!launchable(p.blocks, p.threads())) return hipErrorInvalidValue;
  // few items are in many slots each: a block takes one row of them, else 16
  p.join_rows = p.waves || p.workers <= 16 * items ? 16 : 1;
  p.workspace_bytes = int64_t{2} * p.workers * p.slot_rows * (head_dim + 2) * 4;
  *plan = p;
  return hipSuccess;
}

hipError_t plan_adapter_project(int64_t rows, int32_t in_features, int64_t x_stride, int32_t out_features, int32_t parts,
                                int32_t segments, int32_t adapters, int32_t rank, AdapterPlan* plan) {
  AdapterPlan p{};
  auto tiles = [&](int64_t m, int64_t n) { return (rows + m - 1) / m * ((out_features + n - 1) / n); };
  if (rows <= kAdapterFewTokens) {
    p.kernel = AdapterKernel::kFew;
    p.blocks = tiles(kAdapterFewTokens, kAdapterFewFeatures);
  } else if (tiles(64, 64) <= 512) {
    // The smallest tiles that are all on the CUs at once, two of 64 or 128 on each (5120
    // deep: 1300 x 1152, 378 tiles of 64: 51 us, 76 with 128; 1900 x 1728, 810: 86 and 65;
    // 2500 x 3000, 480 of 128: 94 us, 124 with 256; 2500 x 4200, 660: 159 and 139).
    p.kernel = AdapterKernel::kTiles64;
    p.blocks = tiles(64, 64);
    // Two groups need a whole CU's LDS: where there is a CU for every tile (200 x 5120
    // -> 3000, 188 tiles: 48 us with one, 42 with two; 400 x 1536 -> 4608, 504 tiles: 30 and 36).
    p.groups = p.blocks <= 256 ? 2 : 1;
  } else if (tiles(128, 128) <= 512) {
    p.kernel = AdapterKernel::kTiles128;
    p.blocks = tiles(128, 128);
    p.groups = p.blocks <= 256 ? 2 : 1;  // (2500 x 5120 -> 1536, 240 tiles: 77 us with one, 66 with two)
  } else {
    p.kernel = AdapterKernel::kTiles256;
    p.blocks = tiles(256, 256);
  }
  if (!launchable(p.blocks, 512)) return hipErrorInvalidValue;
  const bool low = segments > 0 && adapters > 0;
  if (low) {
    p.low_rank = (rank + 15) / 16 * 16;
    // Tiles of 64 rows where segments fill them, unless their walk through the stages
    // takes longer than the rounds that blocks of 16 rows make, one a CU: about 5 us and
    // a third a stage against 10 to 15 a round (both launches, rank 64, three parts: 3000 x
    // 1536 49 us, 128 with blocks of 16 rows; 1300 x 576 26 and 45; 500 x 5120 58 and 48).
    const int64_t small = std::min<int64_t>(rows, segments + rows / kLowRows) * (parts * p.low_rank / 16);
    const bool walks = 45 * ((small + 255) / 256) > 17 + (in_features + 63) / 64;
    p.low_rows = p.kernel != AdapterKernel::kFew && rows / segments >= kLowManyRows && walks ? kLowManyRows : kLowRows;
    // every segment's tiles: whole ones, and one that is not full
    p.low_tiles = std::min<int64_t>(rows, segments + rows / p.low_rows);
    const int32_t cols = parts * p.low_rank;
    p.low_columns = p.low_rows == kLowRows ? 16 : cols <= 32 ? 32 : cols <= 64 ? 64 : 96;
    p.low_across = (cols + p.low_columns - 1) / p.low_columns;
    if (p.low_rows == kLowRows ? !launchable(p.low_tiles, 1024) : !launchable(p.low_tiles * p.low_across, 256)) return hipErrorInvalidValue;
    p.low_bytes = (rows * parts * p.low_rank * 2 + 255) / 256 * 256;
  }
  p.workspace_bytes = p.low_bytes;
  // Odd rows are copied for more than 16 tokens (60 x 4733 -> 12000: 83 us, 123 read where
  // they lie; 20 tokens: 76 and 82); for fewer the weights' bytes count, which the copy
  // moves three times (one token: 71 and 57).
  if (rows > kAdapterFewOdd || in_features < 8) {
    const int64_t k8 = (in_features + 7) / 8 * 8;
    p.pack_w = in_features % 8 != 0;
    // the tiles' byte offsets have 32 bits: 256 rows of x
    p.pack_x = p.pack_w || x_stride % 8 != 0 || x_stride > (1 << 21);
    const int64_t copied = (p.pack_x ? rows : 0) + (p.pack_w ? out_features + (low ? int64_t{adapters} * parts * rank : 0) : 0);
    if (copied * (k8 / 8) > kLaunchThreads) return hipErrorInvalidValue;
    p.workspace_bytes += copied * k8 * 2;
  }
  *plan = p;
  return hipSuccess;
}

}  // namespace mssa
