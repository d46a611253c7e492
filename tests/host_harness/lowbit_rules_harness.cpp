// Host harness of the low-bit kernels' rules on sizes, built without any GPU
// code (under AddressSanitizer and UndefinedBehaviorSanitizer by
// tests/test_lowbit_rules.py).  The harness walks each rule the way its kernel
// does and checks what the kernel relies on.  Launchers are stubs that record
// what they are asked for; device addresses are never dereferenced.  Exit
// status 0 iff every check passed.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>
#include <vector>

#include "../../include/libmssa.h"
#include "../../paper_2607_20940_amd/csrc/abi_status.hpp"
#include "../../paper_2607_20940_amd/csrc/lowbit_args.hpp"

namespace {

int g_failures = 0, g_checks = 0;

void check(bool ok, const std::string& what) {
  ++g_checks;
  if (!ok && ++g_failures <= 40) std::fprintf(stderr, "FAIL %s\n", what.c_str());
}

constexpr int64_t kAxis = int64_t{1} << 32;  // threads along a grid's axis: fewer than this

std::vector<mssa::NormArgs> g_norms;
std::vector<mssa::MxArgs> g_conversions;

// An address that stands for a large device array.
char* dev(int i) { return reinterpret_cast<char*>(uintptr_t{1} << 50) + (int64_t{i} << 54); }

}  // namespace

extern "C" const char* hipGetErrorString(hipError_t) { return "stub"; }

namespace mssa {

mssa_status fail(mssa_status s, const char*) noexcept { return s; }
mssa_status fail(mssa_status s, const char*, const char*) noexcept { return s; }

hipError_t launch_norm(const NormArgs& a, bool, bool, hipStream_t) {
  const int tpr = norm_row_shape(a.y_pitch).tpr, threads = std::max(256, tpr), rows = threads / tpr;
  check((a.rows + rows - 1) / rows * threads < kAxis, "a norm launch of 2^32 threads");
  g_norms.push_back(a);
  return hipSuccess;
}
hipError_t launch_norm_bwd(const NormBwdArgs&, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_mx_quantize(const MxArgs& a, bool, hipStream_t) {
  check((a.rows * a.blocks * 4 + 255) / 256 * 256 < kAxis, "a conversion launch of 2^32 threads");
  g_conversions.push_back(a);
  return hipSuccess;
}
hipError_t launch_mx_dequantize(const MxArgs& a, bool bf16, hipStream_t stream) { return launch_mx_quantize(a, bf16, stream); }
hipError_t launch_mx_project(const ProjectArgs& a, bool x_fp4, bool, hipStream_t) {
  ProjectPlan plan;
  check(plan_mx_project(a.M, a.N, a.NB, x_fp4, &plan) == hipSuccess, "the plan of a product that was let through");
  const bool few = plan.kernel == ProjectKernel::kFew16 || plan.kernel == ProjectKernel::kFew32;
  const TileSize t = tile_size(x_fp4, plan.kernel == ProjectKernel::kLargeTiles);
  const int64_t want = few ? (a.N + kProjectFewFeatures - 1) / kProjectFewFeatures
                           : (int64_t{a.M} + t.tokens - 1) / t.tokens * ((a.N + t.features - 1) / t.features);
  check(plan.blocks == want, "a product's blocks");
  check(plan.blocks * (few ? kProjectFewWaves * 64 : t.threads()) < kAxis, "a product launch of 2^32 threads");
  return hipSuccess;
}
hipError_t launch_mx_attention(const MxAttnArgs& a, const MxAttnPlan& p, int, hipStream_t) {
  check(p.blocks * p.threads() < kAxis, "an attention launch of 2^32 threads");
  // the joining launch is made in slices: all rows of all items, in 31 bits
  check(p.join_blocks == (p.workers ? int64_t{a.items} * a.batch * p.slot_rows / p.join_rows : 0) &&
            p.slot_rows % p.join_rows == 0 && p.join_blocks <= 0x7fffffff,
        "the joining launch's blocks");
  return hipSuccess;
}

}  // namespace mssa

namespace {

// The slices of a norm of many rows: together all rows, each in its place.
void norm_slices() {
  for (int32_t cols : {1, 64, 2048, 2049, 8192, 8193, 32768})
    for (int64_t rows : {int64_t{1}, int64_t{1} << 21, (int64_t{1} << 25) + 1, (int64_t{1} << 26) + 3, int64_t{1} << 32})
      for (int e4m3 : {0, 1}) {
        const std::string what = "norm " + std::to_string(rows) + " x " + std::to_string(cols);
        mssa_norm_desc d{};
        d.rows = rows;
        d.cols = cols;
        d.dtype = MSSA_BF16;
        d.out_dtype = e4m3 ? int32_t{MSSA_E4M3} : int32_t{MSSA_BF16};
        d.x_stride = cols + 3;
        g_norms.clear();
        char *x = dev(0), *r = dev(1), *w = dev(2), *s = dev(3), *y = dev(4), *ys = dev(5), *rstd = dev(6);
        check(mssa_add_rms_norm(&d, x, r, w, s, y, e4m3 ? reinterpret_cast<float*>(ys) : nullptr,
                                reinterpret_cast<float*>(rstd), nullptr) == MSSA_OK,
              what);
        int64_t row = 0;
        for (const mssa::NormArgs& a : g_norms) {
          check(a.rows > 0 && a.weight == w && a.cols == cols, what + ": a slice");
          check(a.x == x + row * (cols + 3) * 2 && a.residual == r + row * cols * 2 && a.sum == s + row * cols * 2 &&
                    a.y == y + row * (e4m3 ? a.y_pitch : cols * 2) &&
                    reinterpret_cast<char*>(a.rstd) == rstd + row * 4 &&
                    reinterpret_cast<char*>(a.y_scale) == (e4m3 ? ys + row * 4 : nullptr),
                what + ": a slice's place");
          row += a.rows;
        }
        check(row == rows, what + ": the slices' rows");
      }
}

void conversion_slices() {
  for (int32_t cols : {1, 64, 5120, 1 << 20})
    for (int64_t rows : {int64_t{1}, int64_t{1} << 16, (int64_t{1} << 20) + 7, (int64_t{1} << 30) + 1, int64_t{1} << 35})
      for (int back : {0, 1}) {
        const int64_t blocks = mssa::mx_blocks(cols), stride = cols + 5;
        if (rows * blocks > int64_t{1} << 36) continue;  // refused
        const std::string what = "conversion " + std::to_string(rows) + " x " + std::to_string(cols);
        g_conversions.clear();
        char *v = dev(0), *c = dev(1), *s = dev(2);
        check((back ? mssa_mx_dequantize(rows, cols, MSSA_F32, c, s, v, stride, nullptr)
                    : mssa_mx_quantize(rows, cols, MSSA_F32, v, stride, c, s, nullptr)) == MSSA_OK,
              what);
        int64_t row = 0;
        for (const mssa::MxArgs& a : g_conversions) {
          check(a.rows > 0 && (back ? a.out : a.in) == v + row * stride * 4 && (back ? a.in : a.out) == nullptr &&
                    a.codes == c + row * blocks * 16 && a.scales == s + row * blocks,
                what + ": a slice's place");
          row += a.rows;
        }
        check(row == rows, what + ": the slices' rows");
      }
}

// Products at the limits: made in one launch, or refused where the outputs are 2^38 and more.
void product_launches() {
  for (int64_t rows : {int64_t{1}, int64_t{33}, int64_t{1} << 20, (int64_t{1} << 30) - 64, (int64_t{1} << 30) - 63, int64_t{1} << 30})
    for (int32_t in : {1, 32, 5120, 1 << 20})
      for (int32_t features : {1, 128, 129, 256, 257, 15360, 1 << 20})
        for (int32_t format : {MSSA_E4M3, MSSA_MXFP4}) {
          mssa_mx_project_desc d{};
          d.rows = rows;
          d.in_features = in;
          d.out_features = features;
          d.parts = 1;
          d.x_format = format;
          d.out_dtype = MSSA_BF16;
          d.part0_scale = 1.f;
          void* y = dev(4);
          const mssa_status s = mssa_mx_project(&d, dev(0), dev(1), dev(2), dev(3), nullptr, &y, nullptr);
          check(s == MSSA_OK || (s == MSSA_ERR_UNSUPPORTED && rows * features >= int64_t{1} << 38),
                "product " + std::to_string(rows) + " x " + std::to_string(in) + " -> " + std::to_string(features));
        }
}

// The tile choice's model of a CU: as many blocks as its LDS holds, and no more.  The choices of some sizes, by
// both tiles' measured times, and of the GPU tests that are to
// reach one or the other.
void tile_choices() {
  for (bool x_fp4 : {false, true})
    for (bool large : {false, true}) {
      const mssa::TileSize t = mssa::tile_size(x_fp4, large);
      const int stage = t.tokens * 128 + t.features * (x_fp4 ? 128 : 64);
      // 16 bytes a row and operand for two pairs of stages, or 4 a feature and stage
      const int lds = t.stages * stage + (x_fp4 ? 2 * 16 * (t.tokens + t.features) : t.stages * 4 * t.features);
      const int share = mssa::tile_share(t, x_fp4);
      check(mssa::tile_lds(t, x_fp4) == lds && share * lds <= 163840 && (share + 1) * lds > 163840, "blocks of a CU");
    }
  const struct {
    int32_t tokens, cols, features;
    bool x_fp4, large;
  } cases[] = {{600, 608, 1000, false, false},     {600, 608, 1000, true, false},   {12870, 1536, 4608, false, true},
               {12870, 1536, 4608, true, true},    {400, 5120, 15360, false, true}, {256, 5120, 15360, true, false},
               {1200, 5120, 5120, false, true},    {1200, 5120, 5120, true, false}, {2000, 5120, 5120, true, true},
               {27840, 5120, 15360, true, true},   {70, 1152, 260, true, false},    {4090, 640, 4090, true, true},
               {4090, 1152, 4090, true, true},     {4096, 1536, 4608, false, true}, {4096, 1536, 4608, true, true},
               {2050, 1120, 8001, false, true},    {2050, 1120, 8001, true, true}};
  for (const auto& c : cases) {
    mssa::ProjectPlan p;
    const hipError_t e = mssa::plan_mx_project(c.tokens, c.features, static_cast<int32_t>(mssa::mx_blocks(c.cols)), c.x_fp4, &p);
    check(e == hipSuccess && p.kernel == (c.large ? mssa::ProjectKernel::kLargeTiles : mssa::ProjectKernel::kSmallTiles),
          "tiles of " + std::to_string(c.tokens) + " x " + std::to_string(c.cols) + " -> " + std::to_string(c.features));
  }
}

// Attentions at the limits: made, or refused where they have 2^24 blocks and more (the sizes of single calls).
void attention_launches() {
  for (int32_t batch : {1, 4096, 1 << 20, (1 << 24) - 8, 1 << 24})
    for (int32_t n_q : {1, 32, 33, 2048, 2049, 1 << 20})
      for (int32_t heads : {1, 5, 128})
        for (int64_t tokens : {1, 192, 32760}) {
          mssa_mx_attention_desc d{};
          d.batch = batch;
          d.n_q = n_q;
          d.q_heads = d.kv_heads = heads;
          d.head_dim = 64;
          d.cache_tokens = tokens;
          int64_t bytes = 0;
          const mssa_status sized = mssa_mx_attention_workspace_size(&d, &bytes);
          const mssa_status s = mssa_mx_attention(&d, dev(0), dev(1), dev(2), dev(3), dev(4), nullptr, nullptr, nullptr,
                                                  dev(5), bytes, dev(6), nullptr, nullptr);
          const std::string what = "attention " + std::to_string(batch) + " x " + std::to_string(n_q) + " x " +
                                   std::to_string(heads) + ", " + std::to_string(tokens);
          check(s == sized && (s == MSSA_OK || s == MSSA_ERR_UNSUPPORTED), what);
          if (int64_t{batch} * n_q * heads <= 1 << 24 && int64_t{batch} * heads < 1 << 23) check(s == MSSA_OK, what + ": refused");
        }
}

// Every scale that a tile of the product reads is its own row's: the group as
// the kernel fills it (from memory where it is direct, else with zeros past
// the row), and the bytes that a lane half takes of it.
template <int NBK, int SUPER>
void scale_groups() {
  using G = mssa::ScaleGroups<NBK, SUPER>;
  for (int blocks = 1; blocks <= 200; ++blocks) {
    const G g{blocks};
    for (int st = 0; st * NBK < blocks; ++st) {
      const std::string what = std::to_string(blocks) + " blocks, stage " + std::to_string(st);
      const int first = g.first(st);
      check(first >= 0 && (!g.direct() || (first % 4 == 0 && first + G::kBytes <= blocks)), what + ": the group's place");
      for (int half = 0; half < 2; ++half) {
        const int block0 = st * NBK + G::kHalf * half;  // the half's blocks are block0 .. + kHalf - 1
        check(g.there(st, half) == (block0 < blocks), what + ": there");
        if (!g.there(st, half)) continue;  // the kernel takes zeros
        const int at = g.offset(st, half);
        check(at >= 0 && at + G::kHalf <= G::kBytes, what + ": a half's bytes lie outside its row's");
        for (int k = 0; k < G::kHalf; ++k) {
          const int block = first + at + k;  // whose scale byte k is, if the row has it
          check(block == block0 + k, what + ": another block's scale");
          check(block < blocks || !g.direct(), what + ": past the row in a group that is not filled up");
        }
      }
    }
  }
}

}  // namespace

// With arguments "attention" and a size (batch, n_q, q_heads, kv_heads,
// head_dim, tokens) prints the plan's waves a block, items of a sequence and workers.
int main(int argc, char** argv) {
  if (argc == 8 && std::strcmp(argv[1], "attention") == 0) {
    const auto n = [&](int i) { return static_cast<int32_t>(std::atoi(argv[i])); };
    mssa::MxAttnPlan p;
    if (mssa::plan_mx_attention(n(2), n(3), n(4), n(5), n(6), n(7), &p) != hipSuccess) return 1;
    std::printf("%d %d %d\n", p.waves, p.items, p.workers);
    return 0;
  }
  scale_groups<8, 2>();  // MXFP4 tokens
  scale_groups<4, 1>();  // 8-bit tokens
  norm_slices();
  conversion_slices();
  product_launches();
  tile_choices();
  attention_launches();
  std::printf("%d checks, %d failures\n", g_checks, g_failures);
  return g_failures ? 1 : 0;
}
