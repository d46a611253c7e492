// Kernel arguments and launchers of the low-bit layers (norm, MXFP4
// quantisation, product with MXFP4 weights, attention over an MXFP4 cache).
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#ifdef __HIPCC__
#define MSSA_HOST_DEVICE __host__ __device__
#else
#define MSSA_HOST_DEVICE
#endif

namespace mssa {

constexpr int kMxBlock = 32;  // values under one MXFP4 scale

inline int64_t mx_blocks(int64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }

// Threads of a launch.  A grid's axis has to have fewer than 2^32 of them;
// calls with more rows are made in slices of at most kLaunchThreads.
constexpr int64_t kLaunchThreads = int64_t{1} << 31;
inline bool launchable(int64_t blocks, int threads) { return blocks < ((int64_t{1} << 32) + threads - 1) / threads; }

// ------------------------------------------------------------------- norm
constexpr int kNormMaxCols = 32768;

struct NormArgs {
  const void *x, *residual, *weight;
  void *sum, *y;
  float *y_scale, *rstd;
  int64_t rows, x_stride, residual_stride, sum_stride;
  int32_t cols, y_pitch;  // y_pitch: elements between rows of y
  float eps, inv_cols;
};

struct NormBwdArgs {
  const void *sum, *weight, *dy, *dsum;
  const float* rstd;
  void* dx;
  float *dweight, *partial;  // partial: [blocks, cols], null with one block
  int64_t rows, sum_stride;
  int32_t cols, blocks;
  float inv_cols;
};

// Threads of a row of `cols` values and 8-value pieces of a thread
// (lowbit_plan.cpp, as every rule on sizes that needs no device).
struct NormRowShape {
  int tpr, nv;
};
NormRowShape norm_row_shape(int cols);
// Rows of one launch of the norm, whose output rows have y_pitch elements.
int64_t norm_launch_rows(int y_pitch);

// At most norm_launch_rows rows.
hipError_t launch_norm(const NormArgs& a, bool bf16, bool e4m3, hipStream_t stream);
// Blocks of the backward's first launch: a static rule on the sizes.
int32_t norm_bwd_blocks(int64_t rows, int32_t cols);
hipError_t launch_norm_bwd(const NormBwdArgs& a, bool bf16, hipStream_t stream);

// ------------------------------------------------------------- conversion
struct MxArgs {
  const void* in;
  void *codes, *scales, *out;
  int64_t rows, stride;  // stride: elements between rows of the values
  int32_t cols, blocks;  // blocks of 32 a row
};

// Rows of one launch, of `blocks` blocks each: a thread takes eight values.
int64_t mx_launch_rows(int32_t blocks);

// At most mx_launch_rows rows.
hipError_t launch_mx_quantize(const MxArgs& a, bool bf16, hipStream_t stream);    // in -> codes, scales
hipError_t launch_mx_dequantize(const MxArgs& a, bool bf16, hipStream_t stream);  // codes, scales -> out

// ---------------------------------------------------------------- product
constexpr int kMaxParts = 8;

struct ProjectArgs {
  const void *x, *xs, *w, *ws, *bias;
  void* y[kMaxParts];
  int32_t M, N, NB;  // tokens, features, blocks of 32 along the contraction
  int32_t split;     // features of a part
  float part0_scale;
};

// Scale bytes of the product's tiles.  The bytes of SUPER stages of NBK blocks
// are moved to LDS as one group of kBytes for each row.  Where a row's bytes go
// there straight from memory the last group ends at the row's end, else it is
// filled up with zeros.  A lane half takes one half of a stage's blocks.
template <int NBK, int SUPER>
struct ScaleGroups {
  static constexpr int kBytes = NBK * SUPER, kHalf = NBK / 2;
  int blocks;  // of a row
  MSSA_HOST_DEVICE bool direct() const { return blocks % 4 == 0 && blocks >= kBytes; }  // whole dwords of a row
  // First block of stage st's group.
  MSSA_HOST_DEVICE int first(int st) const {
    const int at = st / SUPER * kBytes;
    return direct() && at > blocks - kBytes ? blocks - kBytes : at;
  }
  // The group's byte with the scale of a lane half's first block.
  MSSA_HOST_DEVICE int offset(int st, int half) const { return st * NBK - first(st) + kHalf * half; }
  // Whether the row has blocks for a lane half at all.  If not, a group that
  // ends at the row's end has no bytes for it: what follows there belongs to
  // the next row, whose NaN scales are not to meet this row's zeros.
  MSSA_HOST_DEVICE bool there(int st, int half) const { return st * NBK + kHalf * half < blocks; }
};

// Which kernel makes a product: one of the two for few tokens, whose blocks
// take kProjectFewFeatures features each, or one of the two tile sizes.
enum class ProjectKernel { kFew16, kFew32, kSmallTiles, kLargeTiles };
constexpr int kProjectFewFeatures = 16, kProjectFewWaves = 4;

// A block's tile: tokens x features, its waves, its stages in LDS.
struct TileSize {
  int tokens, features, waves_m, waves_n, stages;
  constexpr int threads() const { return waves_m * waves_n * 64; }
};
constexpr TileSize tile_size(bool x_fp4, bool large) {
  if (x_fp4) return large ? TileSize{256, 256, 2, 4, 2} : TileSize{64, 128, 1, 4, 2};
  return large ? TileSize{128, 256, 1, 4, 2} : TileSize{64, 128, 1, 4, 3};
}

// LDS bytes of a block: 128 bytes of every token and as many blocks of every
// feature a stage, and groups of scales (ScaleGroups) of both operands' rows
// for two pairs of stages (MXFP4 tokens), or of the features for every stage.
constexpr int tile_lds(const TileSize& t, bool x_fp4) {
  return x_fp4 ? t.stages * (t.tokens + t.features) * 128 + 2 * (t.tokens + t.features) * 16
               : t.stages * (t.tokens * 128 + t.features * 64 + t.features * 4);
}
// Blocks that share a CU: its LDS decides (the kernels' registers allow as many).
constexpr int kLdsBytes = 160 * 1024;
constexpr int tile_share(const TileSize& t, bool x_fp4) { return kLdsBytes / tile_lds(t, x_fp4); }

struct ProjectPlan {
  ProjectKernel kernel;
  int64_t blocks;
};
// Sizes whose launch would have 2^32 threads are refused.
hipError_t plan_mx_project(int32_t tokens, int32_t features, int32_t blocks, bool x_fp4, ProjectPlan* plan);

hipError_t launch_mx_project(const ProjectArgs& a, bool x_fp4, bool out_bf16, hipStream_t stream);

// -------------------------------------------------------------- attention
constexpr int kMxAttnTile = 64;          // tokens of a tile
constexpr int kMxAttnMaxWorkers = 512;
constexpr int kMxAttnFewWaves = 4;       // waves of a block of the kernel for few rows

// `all` tiles in a row, shared out to at most `most` workers: the first `more`
// workers take each + 1 tiles, the others `each`; none is without.
struct Shares {
  uint32_t all, workers, each, more;
  MSSA_HOST_DEVICE static Shares of(uint32_t all, uint32_t most) {
    const uint32_t workers = all < most ? all : most, each = workers ? all / workers : 0;
    return {all, workers, each, all - each * workers};
  }
  MSSA_HOST_DEVICE uint32_t first(uint32_t i) const { return i * each + (i < more ? i : more); }
  MSSA_HOST_DEVICE uint32_t worker_of(uint32_t x) const {
    const uint32_t big = more * (each + 1);
    return x < big ? x / (each + 1) : more + (x - big) / each;
  }
};

struct MxAttnArgs {
  const void *q, *kc, *ks, *vc, *vs, *prior_out;
  const int32_t* kv_len;
  const float* prior_lse;
  void* out;
  float *lse, *partial;
  int64_t cache_tokens, lse_stride;
  int32_t batch, n_q, q_heads, kv_heads, group;  // group = q_heads / kv_heads
  int32_t rows;                                  // n_q * group: query rows that share a key head
  int32_t items, workers, slot_rows, head_waves;  // of the plan
  float scale_log2e;
};

// How a call is cut (a static rule on the sizes).
struct MxAttnPlan {
  int32_t waves;       // 32 rows each in a block; 0: the kernel for few rows
  int32_t items;       // pieces of work of a sequence that one block at a time takes
  int32_t workers;     // shares of all items' contexts, 0: a block per item and no joining launch
  int32_t slot_rows;   // query rows of an item
  int32_t head_waves;  // few rows: waves of a block on neighbouring key heads
  int64_t blocks, workspace_bytes;
  int32_t join_rows;   // rows of a block of the joining launch
  int64_t join_blocks;  // blocks of the joining launch (made in slices), 0 without workers
  int32_t threads() const { return (waves ? waves : kMxAttnFewWaves) * 64; }
};
constexpr int kMxAttnJoinThreads = 256;
// Sizes whose first launch would have 2^32 threads are refused.
hipError_t plan_mx_attention(int32_t batch, int32_t n_q, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                             int64_t cache_tokens, MxAttnPlan* plan);
hipError_t launch_mx_attention(const MxAttnArgs& a, const MxAttnPlan& plan, int head_dim, hipStream_t stream);

}  // namespace mssa
