// How the low-bit kernels cut their work: static rules on sizes, no device code.
#include <algorithm>

#include "lowbit_args.hpp"

namespace mssa {

// A wave a row up to 2048 values (no barrier), four waves up to 8192, sixteen
// above: a thread holds at most 32 values of a row.
NormRowShape norm_row_shape(int cols) {
  const int pieces = (cols + 7) / 8;
  if (pieces <= 256) return {64, (pieces + 63) / 64};
  if (pieces <= 1024) return {256, (pieces + 255) / 256};
  return {1024, (pieces + 1023) / 1024};
}

int64_t norm_launch_rows(int y_pitch) { return kLaunchThreads / norm_row_shape(y_pitch).tpr; }

int32_t norm_bwd_blocks(int64_t rows, int32_t cols) {
  const NormRowShape s = norm_row_shape(cols);
  const int64_t per = s.tpr >= 256 ? 1 : 256 / s.tpr, want = (rows + per - 1) / per;
  return static_cast<int32_t>(std::min<int64_t>(want, 512));
}

int64_t mx_launch_rows(int32_t blocks) { return kLaunchThreads / (int64_t{4} * blocks); }

namespace {

// Microseconds that `tiles` tiles take: whole rounds of `share` blocks a CU,
// then a rest with fewer.  A round of n blocks a CU takes p0 + p1 n a stage and
// q0 + q1 n besides.
struct ShapeCost {
  double p0, p1, q0, q1;
  double operator()(int64_t tiles, int share, int stages) const {
    auto round = [&](int64_t n) { return (p0 + p1 * static_cast<double>(n)) * stages + q0 + q1 * static_cast<double>(n); };
    const int64_t slots = 256 * share, rest = tiles % slots;
    return static_cast<double>(tiles / slots) * round(share) + (rest ? round((rest + 255) / 256) : 0.0);
  }
};

int64_t tiles_of(const TileSize& t, int64_t tokens, int64_t features) {
  return (tokens + t.tokens - 1) / t.tokens * ((features + t.features - 1) / t.features);
}

}  // namespace

// Up to 32 tokens the weights' bytes are all that counts.  Above, large tiles
// need the fewest LDS bytes a product and small tiles fill the CUs sooner.
// 8-bit tokens: 128 x 256 tiles, two blocks a CU, one's outputs leaving while
// the other multiplies (12870 x 1536 -> 4608: 104 us, 64 x 128 tiles 131; at 119
// us one 256 x 256 block a CU took 123 and 128 x 128 tiles 148), or 64 x 128
// (600 x 608 -> 1000: 8.4 us against 14.7).  MXFP4 tokens, whose products are
// done twice as fast from LDS: 256 x 256 (8000 x 5120 -> 15360: 352 us, 64 x 128
// tiles 537; 27840 tokens 1.20 ms, 128 x 256 tiles 1.54), or 64 x 128
// (600 x 608 -> 1000: 8.1 us against 16.7).  The costs are fitted to both tile
// sizes' times of bf16 products of 33 to 12870 tokens, 608 to 5120 values and
// 1000 to 15360 features (58 of each format, each within 40 %): the tiles that
// they choose are the faster ones, or within 3 % of them.  With fp32 outputs
// of 8-bit tokens, which take another path, within 11 %.
hipError_t plan_mx_project(int32_t tokens, int32_t features, int32_t blocks, bool x_fp4, ProjectPlan* plan) {
  if (tokens <= 32) {
    *plan = {tokens <= 16 ? ProjectKernel::kFew16 : ProjectKernel::kFew32,
             (int64_t{features} + kProjectFewFeatures - 1) / kProjectFewFeatures};
    return hipSuccess;
  }
  const ShapeCost small = x_fp4 ? ShapeCost{0.35, 0.15, 5.3, 0.} : ShapeCost{0.06, 0.29, 5.6, 0.};
  const ShapeCost large = x_fp4 ? ShapeCost{0., 1.36, 0., 11.5} : ShapeCost{0., 0.75, 9.5, 0.5};
  const int stages = (blocks + (x_fp4 ? 7 : 3)) / (x_fp4 ? 8 : 4);
  const TileSize ts = tile_size(x_fp4, false), tl = tile_size(x_fp4, true);
  const int64_t n_small = tiles_of(ts, tokens, features), n_large = tiles_of(tl, tokens, features);
  if (launchable(n_small, ts.threads()) &&
      small(n_small, tile_share(ts, x_fp4), stages) < large(n_large, tile_share(tl, x_fp4), stages))
    *plan = {ProjectKernel::kSmallTiles, n_small};
  else if (launchable(n_large, tl.threads()))
    *plan = {ProjectKernel::kLargeTiles, n_large};
  else
    return hipErrorInvalidValue;
  return hipSuccess;
}

hipError_t plan_mx_attention(int32_t batch, int32_t n_q, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                             int64_t cache_tokens, MxAttnPlan* plan) {
  MxAttnPlan p{};
  const int64_t rows = static_cast<int64_t>(n_q) * (q_heads / kv_heads), tiles = (cache_tokens + kMxAttnTile - 1) / kMxAttnTile;
  // Up to 2048 rows blocks of four waves, two on a CU: an item's rows fit
  // better and one block starts while the other works (1173 rows over 1955
  // tokens 25.2 -> 23.0 us, 1800 rows over 9000 tokens 46.0 and 46.2); above,
  // eight waves share each expanded tile.
  p.waves = rows <= 32 ? 0 : rows <= 2048 ? 4 : 8;
  p.head_waves = kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1;
  const int64_t side = p.waves ? 1 : kv_heads / p.head_waves;  // blocks of one worker
  const int64_t items = p.waves ? (rows + p.waves * 32 - 1) / (p.waves * 32) * kv_heads : 1;
  const int64_t slot_rows = p.waves ? p.waves * 32 : rows * kv_heads;
  const int64_t slots = p.waves == 8 ? 256 : 512;  // blocks resident at once
  // Work for more than one block per item: at least this many tiles a worker.
  const int64_t least = p.waves ? 4 : 2 * kMxAttnFewWaves / p.head_waves;
  if (items * batch > 0x7fffffff || items * batch * tiles > 0x7fffffff) return hipErrorInvalidValue;  // 31 bits of tiles
  const int64_t all = items * batch * tiles;
  // A second worker a CU only where each has 8 tiles: with fewer the slots that
  // the joining launch reads cost more (1173 rows over 1955 tokens 23.0 -> 21.8
  // us; with 8 tiles a worker at least everywhere, 100 rows over 1500 tokens
  // 13.8 -> 17.5).
  int64_t most = all / least;
  if (p.waves == 4) most = std::min(most, std::max<int64_t>(256, all / 8));
  if (tiles > least) p.workers = static_cast<int32_t>(std::max<int64_t>(1, std::min({int64_t{kMxAttnMaxWorkers}, slots / side, most})));
  p.blocks = p.workers ? (p.waves ? p.workers : (p.workers + 7) / 8 * 8 * side)
                       : (p.waves ? items * batch : (batch + int64_t{7}) / 8 * 8 * side);
  p.join_rows = p.waves ? 8 : 1;
  p.join_blocks = p.workers ? items * batch * (slot_rows / p.join_rows) : 0;
  if (slot_rows > 0x7fffffff || !launchable(p.blocks, p.threads()) || p.join_blocks > 0x7fffffff) return hipErrorInvalidValue;
  p.items = static_cast<int32_t>(items);
  p.slot_rows = static_cast<int32_t>(slot_rows);
  p.workspace_bytes = int64_t{2} * p.workers * slot_rows * (head_dim + 2) * 4;
  *plan = p;
  return hipSuccess;
}

}  // namespace mssa
