// Host harness of the low-bit layers' C ABI and of the rules that cut their
// work, built without any GPU code (under AddressSanitizer and
// UndefinedBehaviorSanitizer by tests/test_lowbit_host_sanitized.py).  The
// kernel launchers are replaced by stubs that check every address range the
// kernel would read or write, derived from its argument struct, against the
// buffers passed; device buffers are address ranges that are never
// dereferenced.  For attention the stub also walks the shares of the tiles as
// the workers and the joining launch do, for random sequence lengths: every
// tile is taken once, and the slots that the join reads of an item are the
// slots that its workers write.
//
// Calls: fixed corner sizes and 400 seeded random descriptors of every entry
// point, and descriptors at the limits.  Exit status 0 iff every check passed.
// With the argument "plant" every workspace is 256 bytes shorter than the
// size the harness passes, a mistake the range checks must report.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cinttypes>
#include <cstdio>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "../../include/libmssa.h"
#include "../../paper_2607_20940_amd/csrc/abi_status.hpp"
#include "../../paper_2607_20940_amd/csrc/lowbit_args.hpp"

namespace {

int g_failures = 0, g_checks = 0;
bool g_plant = false;
std::string g_case;
std::string g_error;

void failure(const char* what) {
  if (++g_failures <= 40) std::fprintf(stderr, "FAIL [%s]: %s\n", g_case.c_str(), what);
}

void check(bool ok, const char* what) {
  ++g_checks;
  if (!ok) failure(what);
}

struct Range {
  uintptr_t b, e;
};
std::vector<Range> g_bufs;
uintptr_t g_next = uintptr_t{1} << 44;
bool g_ranges = true;  // off: descriptors at the limits, whose buffers are a few bytes

void* dev_alloc(int64_t bytes) {
  if (bytes <= 0) return nullptr;
  const uintptr_t b = g_next;
  g_next += uintptr_t{1} << 40;
  g_bufs.push_back({b, b + static_cast<uintptr_t>(bytes)});
  return reinterpret_cast<void*>(b);
}

void* workspace(int64_t bytes) { return dev_alloc(g_plant ? bytes - 256 : bytes); }

void dev_reset() {
  g_bufs.clear();
  g_next = uintptr_t{1} << 44;
}

void check_range(const void* p, int64_t bytes, const char* what) {
  ++g_checks;
  if (bytes <= 0 || !g_ranges) return;
  const uintptr_t b = reinterpret_cast<uintptr_t>(p);
  for (const Range& r : g_bufs)
    if (b >= r.b && b < r.e) {
      if (b + static_cast<uintptr_t>(bytes) > r.e) {
        char msg[256];
        std::snprintf(msg, sizeof msg, "%s: %" PRId64 " bytes from buffer offset %" PRIuPTR " overrun its %" PRIuPTR,
                      what, bytes, b - r.b, r.e - r.b);
        failure(msg);
      }
      return;
    }
  failure((std::string(what) + ": address outside every buffer").c_str());
}

uint64_t g_seed = 88172645463325252ull;
uint64_t rnd() {
  g_seed ^= g_seed << 13;
  g_seed ^= g_seed >> 7;
  g_seed ^= g_seed << 17;
  return g_seed;
}
int64_t pick(int64_t lo, int64_t hi) { return lo + static_cast<int64_t>(rnd() % static_cast<uint64_t>(hi - lo + 1)); }

// Bytes of `rows` rows of `cols` elements, `stride` elements apart.
int64_t span(int64_t rows, int64_t cols, int64_t stride, int64_t eb) {
  return rows ? ((rows - 1) * stride + cols) * eb : 0;
}

int g_launches = 0;

}  // namespace

extern "C" const char* hipGetErrorString(hipError_t) { return "stub"; }

namespace mssa {

mssa_status fail(mssa_status s, const char* msg) noexcept {
  g_error = msg;
  return s;
}
mssa_status fail(mssa_status s, const char* what, const char* detail) noexcept {
  g_error = std::string(what) + ": " + detail;
  return s;
}

hipError_t launch_norm(const NormArgs& a, bool bf16, bool e4m3, hipStream_t) {
  ++g_launches;
  const int64_t eb = bf16 ? 2 : 4;
  const NormRowShape s = norm_row_shape(a.cols);
  check(s.nv >= 1 && s.nv <= 4 && int64_t{s.tpr} * s.nv * 8 >= a.cols, "the threads of a row hold all of it");
  check(a.y_pitch >= a.cols && a.y_pitch <= s.tpr * s.nv * 8, "the threads of a row write all of its output");
  check_range(a.x, span(a.rows, a.cols, a.x_stride, eb), "x");
  check_range(a.weight, a.cols * eb, "weight");
  if (a.residual) {
    check_range(a.residual, span(a.rows, a.cols, a.residual_stride, eb), "residual");
    check_range(a.sum, span(a.rows, a.cols, a.sum_stride, eb), "sum");
  }
  check_range(a.y, a.rows * a.y_pitch * (e4m3 ? 1 : eb), "y");
  if (e4m3) check_range(a.y_scale, a.rows * 4, "y_scale");
  if (a.rstd) check_range(a.rstd, a.rows * 4, "rstd");
  return hipSuccess;
}

hipError_t launch_norm_bwd(const NormBwdArgs& a, bool bf16, hipStream_t) {
  ++g_launches;
  const int64_t eb = bf16 ? 2 : 4;
  check(a.blocks == norm_bwd_blocks(a.rows, a.cols), "the backward's blocks");
  check_range(a.sum, span(a.rows, a.cols, a.sum_stride, eb), "sum");
  check_range(a.dy, a.rows * a.cols * eb, "dy");
  if (a.dsum) check_range(a.dsum, a.rows * a.cols * eb, "dsum");
  check_range(a.dx, a.rows * a.cols * eb, "dx");
  check_range(a.rstd, a.rows * 4, "rstd");
  if (a.rows) check_range(a.weight, a.cols * eb, "weight");
  if (a.blocks > 1) check_range(a.partial, int64_t{a.blocks} * a.cols * 4, "partial");
  check_range(a.dweight, int64_t{a.cols} * 4, "dweight");
  return hipSuccess;
}

void convert_ranges(const MxArgs& a, bool bf16, const void* values) {
  ++g_launches;
  check(int64_t{a.blocks} * kMxBlock >= a.cols && int64_t{a.blocks - 1} * kMxBlock < a.cols, "blocks of a row");
  check_range(values, span(a.rows, a.cols, a.stride, bf16 ? 2 : 4), "values");
  check_range(a.codes, a.rows * a.blocks * 16, "codes");
  check_range(a.scales, a.rows * a.blocks, "scales");
}
hipError_t launch_mx_quantize(const MxArgs& a, bool bf16, hipStream_t) {
  convert_ranges(a, bf16, a.in);
  return hipSuccess;
}
hipError_t launch_mx_dequantize(const MxArgs& a, bool bf16, hipStream_t) {
  convert_ranges(a, bf16, a.out);
  return hipSuccess;
}

hipError_t launch_mx_project(const ProjectArgs& a, bool x_fp4, bool out_bf16, hipStream_t) {
  ++g_launches;
  check_range(a.x, int64_t{a.M} * a.NB * (x_fp4 ? 16 : 32), "x");
  check_range(a.xs, int64_t{a.M} * (x_fp4 ? a.NB : 4), "x_scales");
  check_range(a.w, int64_t{a.N} * a.NB * 16, "w");
  check_range(a.ws, int64_t{a.N} * a.NB, "w_scales");
  if (a.bias) check_range(a.bias, int64_t{a.N} * 4, "bias");
  check(a.N % a.split == 0 && a.N / a.split <= kMaxParts, "parts");
  for (int p = 0; p < a.N / a.split; ++p) check_range(a.y[p], int64_t{a.M} * a.split * (out_bf16 ? 2 : 4), "y");
  return hipSuccess;
}

// The shares of one call: the sequences' tiles, item by item, in a row.
void check_shares(const MxAttnArgs& a, const std::vector<int64_t>& len) {
  std::vector<uint32_t> first;  // first tile of every item, and the end of the last
  uint32_t all = 0;
  for (int64_t n : len)
    for (int i = 0; i < a.items; ++i) {
      first.push_back(all);
      all += static_cast<uint32_t>((n + kMxAttnTile - 1) / kMxAttnTile);
    }
  first.push_back(all);
  const Shares sh = Shares::of(all, static_cast<uint32_t>(a.workers));
  std::vector<int> taken(all, 0);
  std::map<uint32_t, std::vector<uint32_t>> written;  // item -> slots, in the workers' order
  for (uint32_t w = 0; w < sh.workers; ++w) {
    const uint32_t x0 = sh.first(w), x1 = sh.first(w + 1);
    check(x1 > x0 && x1 <= all, "a worker's share");
    uint32_t item = static_cast<uint32_t>(std::upper_bound(first.begin(), first.end(), x0) - first.begin()) - 1;
    int seg = 0;
    for (uint32_t x = x0; x < x1; ++seg, ++item) {
      while (first[item + 1] == first[item]) ++item;
      const uint32_t end = std::min(first[item + 1], x1);
      const bool whole = x == first[item] && end == first[item + 1];
      if (!whole) {
        check(seg == 0 || end == x1, "a shared item is a worker's first or last");
        written[item].push_back(2 * w + (seg > 0));
      }
      for (; x < end; ++x) {
        check(sh.worker_of(x) == w, "worker_of");
        ++taken[x];
      }
    }
  }
  check(std::all_of(taken.begin(), taken.end(), [](int n) { return n == 1; }), "every tile is taken once");
  for (size_t item = 0; item + 1 < first.size(); ++item) {
    const uint32_t start = first[item], nt = first[item + 1] - start;
    const uint32_t w0 = nt ? sh.worker_of(start) : 0, w1 = nt ? sh.worker_of(start + nt - 1) : 0;
    std::vector<uint32_t> read;
    if (nt && w1 > w0)
      for (uint32_t s = 0; s <= w1 - w0; ++s)
        read.push_back(s ? 2 * (w0 + s) : sh.first(w0) != start ? 2 * w0 + 1 : 2 * w0);
    const auto it = written.find(static_cast<uint32_t>(item));
    check(read == (it == written.end() ? std::vector<uint32_t>{} : it->second), "the join reads what was written");
    for (uint32_t s : read) check(s < 2 * static_cast<uint32_t>(a.workers), "a slot of the workspace");
  }
}

hipError_t launch_mx_attention(const MxAttnArgs& a, const MxAttnPlan& plan, int D, hipStream_t) {
  ++g_launches;
  const int64_t tokens = a.batch * a.cache_tokens * a.kv_heads, rows = int64_t{a.batch} * a.n_q * a.q_heads;
  check(a.rows == int64_t{a.n_q} * a.group && a.workers <= kMxAttnMaxWorkers, "plan");
  if (plan.waves == 0) {
    check(a.rows <= 32 && a.kv_heads % a.head_waves == 0 && kMxAttnFewWaves % a.head_waves == 0, "few rows");
    check(plan.blocks >= int64_t{plan.workers ? plan.workers : a.batch} * (a.kv_heads / a.head_waves), "blocks");
  } else {
    check(int64_t{a.items} * plan.waves * 32 >= int64_t{a.rows} * a.kv_heads, "the items hold all rows");
    check(plan.blocks == (plan.workers ? plan.workers : int64_t{a.items} * a.batch), "blocks");
  }
  check_range(a.q, rows * D * 2, "q");
  check_range(a.out, rows * D * 2, "out");
  check_range(a.kc, tokens * D / 2, "k_codes");
  check_range(a.vc, tokens * D / 2, "v_codes");
  check_range(a.ks, tokens * D / 32, "k_scales");
  check_range(a.vs, tokens * D / 32, "v_scales");
  if (a.kv_len) check_range(a.kv_len, int64_t{a.batch} * 4, "kv_len");
  const int64_t lse_bytes = ((int64_t{a.batch} * a.q_heads - 1) * a.lse_stride + a.n_q) * 4;
  if (a.lse) check_range(a.lse, lse_bytes, "lse");
  if (a.prior_out) {
    check_range(a.prior_out, rows * D * 2, "prior_out");
    check_range(a.prior_lse, lse_bytes, "prior_lse");
  }
  if (a.workers) {
    const int64_t slots = int64_t{2} * a.workers * a.slot_rows;
    check_range(a.partial, slots * D * 4, "slot sums");
    check_range(a.partial + slots * D, slots * 8, "slot statistics");
    if (g_ranges) {
      std::vector<int64_t> len(static_cast<size_t>(a.batch), a.cache_tokens);
      check_shares(a, len);
      for (int turn = 0; turn < 3; ++turn) {
        for (int64_t& n : len) n = pick(0, 3) ? pick(0, a.cache_tokens) : 0;
        check_shares(a, len);
      }
      check_shares(a, std::vector<int64_t>(static_cast<size_t>(a.batch), 0));
    }
  }
  return hipSuccess;
}

}  // namespace mssa

namespace {

void expect(mssa_status got, mssa_status want, const char* what) {
  ++g_checks;
  if (got != want) failure((std::string(what) + ": status " + std::to_string(got) + " (" + g_error + ")").c_str());
}

int64_t padded(int64_t cols) { return mssa::mx_blocks(cols) * mssa::kMxBlock; }

void norm_case(int64_t rows, int32_t cols, bool bf16, bool e4m3, bool residual, bool wide, bool dsum) {
  g_case = "norm " + std::to_string(rows) + " x " + std::to_string(cols);
  dev_reset();
  mssa_norm_desc d{};
  d.rows = rows;
  d.cols = cols;
  d.dtype = bf16 ? MSSA_BF16 : MSSA_F32;
  d.out_dtype = e4m3 ? MSSA_E4M3 : d.dtype;
  d.eps = 1e-6f;
  if (wide) {
    d.x_stride = cols + pick(0, 64);
    d.residual_stride = cols + pick(1, 64);
    d.sum_stride = cols + pick(1, 64);
  }
  const int64_t eb = bf16 ? 2 : 4;
  const auto stride = [&](int64_t s) { return s ? s : cols; };
  void* x = dev_alloc(span(rows, cols, stride(d.x_stride), eb));
  void* r = residual ? dev_alloc(span(rows, cols, stride(d.residual_stride), eb)) : nullptr;
  void* sum = residual ? dev_alloc(span(rows, cols, stride(d.sum_stride), eb)) : nullptr;
  void* w = dev_alloc(cols * eb);
  void* y = dev_alloc(rows * (e4m3 ? padded(cols) : cols * eb));
  float* ys = e4m3 ? static_cast<float*>(dev_alloc(rows * 4)) : nullptr;
  float* rstd = static_cast<float*>(dev_alloc(rows * 4));
  const int before = g_launches;
  expect(mssa_add_rms_norm(&d, x, r, w, sum, y, ys, rstd, nullptr), MSSA_OK, "norm");
  check(g_launches == before + (rows > 0), "one launch, none without rows");
  if (e4m3) return;
  int64_t bytes = -1;
  expect(mssa_add_rms_norm_workspace_size(&d, &bytes), MSSA_OK, "workspace size");
  const void* s = residual ? sum : x;
  if (!residual) d.sum_stride = d.x_stride;
  void* dy = dev_alloc(rows * cols * eb);
  void* ds = dsum ? dev_alloc(rows * cols * eb) : nullptr;
  void* dx = dev_alloc(rows * cols * eb);
  float* dw = static_cast<float*>(dev_alloc(cols * 4));
  void* ws = workspace(bytes);
  if (bytes > 0)
    expect(mssa_add_rms_norm_backward(&d, s, w, rstd, dy, ds, ws, bytes - 1, dx, dw, nullptr), MSSA_ERR_WORKSPACE,
           "a short workspace");
  expect(mssa_add_rms_norm_backward(&d, s, w, rstd, dy, ds, ws, bytes, dx, dw, nullptr), MSSA_OK, "norm backward");
}

void convert_case(int64_t rows, int32_t cols, bool bf16, bool wide) {
  g_case = "convert " + std::to_string(rows) + " x " + std::to_string(cols);
  dev_reset();
  const int64_t stride = wide ? cols + pick(0, 64) : 0;
  void* v = dev_alloc(span(rows, cols, stride ? stride : cols, bf16 ? 2 : 4));
  void* codes = dev_alloc(rows * mssa::mx_blocks(cols) * 16);
  void* scales = dev_alloc(rows * mssa::mx_blocks(cols));
  const int32_t dtype = bf16 ? MSSA_BF16 : MSSA_F32;
  expect(mssa_mx_quantize(rows, cols, dtype, v, stride, codes, scales, nullptr), MSSA_OK, "quantize");
  expect(mssa_mx_dequantize(rows, cols, dtype, codes, scales, v, stride, nullptr), MSSA_OK, "dequantize");
}

void project_case(int64_t rows, int32_t in, int32_t part, int32_t parts, bool x_fp4, bool bf16, bool bias) {
  g_case = "project " + std::to_string(rows) + " x " + std::to_string(in) + " -> " + std::to_string(parts) + " x " +
           std::to_string(part);
  dev_reset();
  mssa_mx_project_desc d{};
  d.rows = static_cast<decltype(d.rows)>(rows);
  d.in_features = in;
  d.out_features = part * parts;
  d.parts = parts;
  d.x_format = x_fp4 ? MSSA_MXFP4 : MSSA_E4M3;
  d.out_dtype = bf16 ? MSSA_BF16 : MSSA_F32;
  d.part0_scale = 1.f;
  const int64_t nb = mssa::mx_blocks(in);
  void* x = dev_alloc(rows * nb * (x_fp4 ? 16 : 32));
  void* xs = dev_alloc(rows * (x_fp4 ? nb : 4));
  void* w = dev_alloc(d.out_features * nb * 16);
  void* ws = dev_alloc(d.out_features * nb);
  void* b = bias ? dev_alloc(int64_t{d.out_features} * 4) : nullptr;
  void* y[8] = {};
  for (int p = 0; p < parts; ++p) y[p] = dev_alloc(rows * part * (bf16 ? 2 : 4));
  expect(mssa_mx_project(&d, x, xs, w, ws, b, y, nullptr), MSSA_OK, "project");
}

mssa_mx_attention_desc attention_desc(int32_t batch, int32_t n_q, int32_t kv_heads, int32_t group, int32_t D,
                                      int64_t tokens) {
  mssa_mx_attention_desc d{};
  d.batch = batch;
  d.n_q = n_q;
  d.kv_heads = kv_heads;
  d.q_heads = kv_heads * group;
  d.head_dim = D;
  d.cache_tokens = tokens;
  return d;
}

void attention_case(int32_t batch, int32_t n_q, int32_t kv_heads, int32_t group, int32_t D, int64_t tokens,
                    int32_t extra, bool lengths, bool prior, bool want_lse) {
  g_case = "attention " + std::to_string(batch) + " x " + std::to_string(n_q) + ", heads " + std::to_string(kv_heads) +
           " x " + std::to_string(group) + " of " + std::to_string(D) + ", " + std::to_string(tokens) + " tokens";
  dev_reset();
  mssa_mx_attention_desc d = attention_desc(batch, n_q, kv_heads, group, D, tokens);
  if (extra) d.lse_stride = n_q + extra;
  const int64_t rows = int64_t{batch} * n_q * d.q_heads, all = batch * tokens * kv_heads;
  const int64_t lse_bytes = ((int64_t{batch} * d.q_heads - 1) * (n_q + extra) + n_q) * 4;
  void* q = dev_alloc(rows * D * 2);
  void *kc = dev_alloc(all * D / 2), *ks = dev_alloc(all * D / 32), *vc = dev_alloc(all * D / 2),
       *vs = dev_alloc(all * D / 32);
  auto* len = lengths ? static_cast<int32_t*>(dev_alloc(int64_t{batch} * 4)) : nullptr;
  void* po = prior ? dev_alloc(rows * D * 2) : nullptr;
  auto* pl = prior ? static_cast<float*>(dev_alloc(lse_bytes)) : nullptr;
  void* out = dev_alloc(rows * D * 2);
  auto* lse = want_lse ? static_cast<float*>(dev_alloc(lse_bytes)) : nullptr;
  int64_t bytes = -1;
  expect(mssa_mx_attention_workspace_size(&d, &bytes), MSSA_OK, "workspace size");
  void* ws = workspace(bytes);
  if (bytes > 0)
    expect(mssa_mx_attention(&d, q, kc, ks, vc, vs, len, po, pl, ws, bytes - 1, out, lse, nullptr), MSSA_ERR_WORKSPACE,
           "a short workspace");
  expect(mssa_mx_attention(&d, q, kc, ks, vc, vs, len, po, pl, ws, bytes, out, lse, nullptr), MSSA_OK, "attention");
}

// Descriptors at the limits: answered or refused, without an overflow.
void limit_cases() {
  g_ranges = false;
  g_case = "limits";
  dev_reset();
  void* p = dev_alloc(1024);
  void* q = dev_alloc(1024);
  auto* f = static_cast<float*>(dev_alloc(1024));
  const int32_t top = 0x7fffffff;
  for (int32_t batch : {1, 65536, 0x3fffffff, top})
    for (int32_t n_q : {1, 33, 1025, 0x3fffffff, top})
      for (int32_t heads : {1, 8, 4096, 0x3fffffff})
        for (int32_t group : {1, 2})
          for (int64_t tokens : {int64_t{1}, int64_t{32760}, int64_t{top}}) {
            mssa_mx_attention_desc d = attention_desc(batch, n_q, heads, group, 128, tokens);
            int64_t bytes = -1;
            const mssa_status s = mssa_mx_attention_workspace_size(&d, &bytes);
            check(s == MSSA_ERR_UNSUPPORTED || (s == MSSA_OK && bytes >= 0), "attention at the limits");
            if (s != MSSA_OK) continue;
            mssa::MxAttnPlan plan;
            mssa::plan_mx_attention(batch, n_q, heads * group, heads, 128, tokens, &plan);
            check(plan.blocks >= 1 && plan.blocks <= top, "a launch's blocks");
            // every tile number of the call in 31 bits
            check(int64_t{plan.items} * batch * ((tokens + 63) / 64) <= top, "tiles");
          }
  for (int64_t rows : {int64_t{0}, int64_t{1}, int64_t{1} << 40})
    for (int32_t cols : {1, 32768})
      for (int64_t stride : {int64_t{0}, int64_t{32768}, int64_t{1} << 20, int64_t{1} << 62}) {
        mssa_norm_desc d{};
        d.rows = rows;
        d.cols = cols;
        d.dtype = d.out_dtype = MSSA_F32;
        d.x_stride = stride;
        const mssa_status s = mssa_add_rms_norm(&d, p, nullptr, p, nullptr, q, nullptr, f, nullptr);
        check(s == MSSA_OK || s == MSSA_ERR_INVALID_ARG, "norm at the limits");
        check(s == MSSA_OK || stride > (int64_t{1} << 20) / (rows > 1 ? 2 : 1), "a norm within the limits is refused");
        mssa_mx_quantize(rows, cols, MSSA_F32, p, stride, q, q, nullptr);
        mssa_mx_dequantize(rows, cols, MSSA_F32, p, p, q, stride, nullptr);
      }
  g_ranges = true;
}

}  // namespace

int main(int argc, char** argv) {
  g_plant = argc > 1 && std::strcmp(argv[1], "plant") == 0;
  for (int32_t cols : {1, 8, 31, 33, 2047, 2048, 2049, 8192, 8193, 16385, 32768})
    for (int64_t rows : {0, 1, 5, 2050}) {
      norm_case(rows, cols, true, false, true, false, true);
      norm_case(rows, cols, false, true, false, true, false);
      convert_case(rows, cols, true, false);
    }
  for (int32_t n_q : {1, 2, 4, 5, 127, 129, 1023, 1025})
    for (int64_t tokens : {1, 64, 65, 500, 4097, 32760}) {
      attention_case(1, n_q, 1, 1, 64, tokens, 0, false, false, true);
      attention_case(3, n_q, 4, 8, 128, tokens, 3, true, true, true);
      attention_case(2, n_q, 6, 2, 64, tokens, 0, true, false, false);
    }
  for (int i = 0; i < 400; ++i) {
    norm_case(pick(0, 3) ? pick(1, 5000) : pick(0, 3), static_cast<int32_t>(pick(0, 3) ? pick(1, 6000) : pick(1, 32768)),
              rnd() & 1, rnd() & 1, rnd() & 1, rnd() & 1, rnd() & 1);
    convert_case(pick(0, 4000), static_cast<int32_t>(pick(1, 4000)), rnd() & 1, rnd() & 1);
    project_case(pick(0, 3) ? pick(1, 4000) : pick(0, 33), static_cast<int32_t>(pick(1, 3000)),
                 static_cast<int32_t>(pick(1, 900)), static_cast<int32_t>(pick(1, 8)), rnd() & 1, rnd() & 1, rnd() & 1);
    attention_case(static_cast<int32_t>(pick(1, 9)), static_cast<int32_t>(pick(0, 1) ? pick(1, 16) : pick(17, 3000)),
                   static_cast<int32_t>(pick(1, 9)), static_cast<int32_t>(pick(1, 9)), rnd() & 1 ? 64 : 128,
                   pick(0, 3) ? pick(1, 3000) : pick(1, 100000), static_cast<int32_t>(pick(0, 1) * pick(0, 9)), rnd() & 1,
                   rnd() & 1, rnd() & 1);
  }
  limit_cases();
  std::printf("%d checks, %d launches, %d failures\n", g_checks, g_launches, g_failures);
  return g_failures ? 1 : 0;
}
