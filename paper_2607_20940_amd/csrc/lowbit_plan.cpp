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
  if (slot_rows > 0x7fffffff || p.blocks > 0x7fffffff ||
      items * batch * (slot_rows / (p.waves ? 8 : 1)) > 0x7fffffff)
    return hipErrorInvalidValue;
  p.items = static_cast<int32_t>(items);
  p.slot_rows = static_cast<int32_t>(slot_rows);
  p.workspace_bytes = int64_t{2} * p.workers * slot_rows * (head_dim + 2) * 4;
  *plan = p;
  return hipSuccess;
}

}  // namespace mssa
