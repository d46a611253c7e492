// C ABI of the low-bit layers (declared in include/libmssa.h): every call is
// checked before anything is enqueued.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "abi_status.hpp"
#include "lowbit_args.hpp"

namespace {

using mssa::aligned16;
using mssa::check_device;
using mssa::fail;
using mssa::guarded;

int elem_bytes(int32_t dtype) { return dtype == MSSA_BF16 ? 2 : 4; }

bool aligned_to(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }

// `bytes` further on; null stays null.
const void* at_byte(const void* p, int64_t bytes) { return p ? static_cast<const char*>(p) + bytes : nullptr; }
void* at_byte(void* p, int64_t bytes) { return p ? static_cast<char*>(p) + bytes : nullptr; }

hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }

// rows x stride elements stay addressable in 63 bits.
bool stride_ok(int64_t stride, int64_t cols, int64_t rows) {
  return stride == 0 || (stride >= cols && (rows == 0 || stride <= (int64_t{1} << 60) / rows));
}

mssa_status norm_check(const mssa_norm_desc* d) {
  if (!d) return fail(MSSA_ERR_INVALID_ARG, "null argument");
  if (d->rows < 0 || d->rows > (int64_t{1} << 40)) return fail(MSSA_ERR_INVALID_ARG, "rows must be in [0, 2^40]");
  if (d->cols < 1) return fail(MSSA_ERR_INVALID_ARG, "cols must be positive");
  if (d->cols > mssa::kNormMaxCols) return fail(MSSA_ERR_UNSUPPORTED, "cols above 32768");
  if (d->dtype != MSSA_BF16 && d->dtype != MSSA_F32) return fail(MSSA_ERR_INVALID_ARG, "dtype must be bf16 or fp32");
  if (d->out_dtype != d->dtype && d->out_dtype != MSSA_E4M3)
    return fail(MSSA_ERR_INVALID_ARG, "out_dtype must be dtype or MSSA_E4M3");
  if (!std::isfinite(d->eps) || d->eps < 0.f) return fail(MSSA_ERR_INVALID_ARG, "eps must be finite and not negative");
  for (int64_t s : {d->x_stride, d->residual_stride, d->sum_stride})
    if (!stride_ok(s, d->cols, d->rows)) return fail(MSSA_ERR_INVALID_ARG, "a row stride is shorter than cols, or too long");
  return MSSA_OK;
}

int64_t stride_or(int64_t stride, int64_t cols) { return stride ? stride : cols; }

mssa_status mx_check(int64_t rows, int32_t cols, int32_t dtype, int64_t stride) {
  if (rows < 0 || rows > (int64_t{1} << 40)) return fail(MSSA_ERR_INVALID_ARG, "rows must be in [0, 2^40]");
  if (cols < 1 || cols > (1 << 20)) return fail(MSSA_ERR_INVALID_ARG, "cols must be in [1, 2^20]");
  if (dtype != MSSA_BF16 && dtype != MSSA_F32) return fail(MSSA_ERR_INVALID_ARG, "dtype must be bf16 or fp32");
  if (!stride_ok(stride, cols, rows)) return fail(MSSA_ERR_INVALID_ARG, "the row stride is shorter than cols, or too long");
  if (rows * mssa::mx_blocks(cols) > (int64_t{1} << 36)) return fail(MSSA_ERR_UNSUPPORTED, "more than 2^36 blocks");
  return MSSA_OK;
}

mssa_status mx_convert(const char* who, bool quantize, int64_t rows, int32_t cols, int32_t dtype, const void* values,
                       int64_t stride, const void* codes, const void* scales, void* stream) {
  return guarded(who, [&]() -> mssa_status {
    const mssa_status s = mx_check(rows, cols, dtype, stride);
    if (s != MSSA_OK) return s;
    if (rows == 0) return MSSA_OK;
    if (!values || !codes || !scales) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    if (!aligned_to(values, elem_bytes(dtype))) return fail(MSSA_ERR_INVALID_ARG, "values must be aligned to their type");
    if (!aligned_to(codes, 4)) return fail(MSSA_ERR_INVALID_ARG, "codes must be 4-byte aligned");
    mssa::MxArgs a{};
    a.stride = stride_or(stride, cols);
    a.cols = cols;
    a.blocks = static_cast<int32_t>(mssa::mx_blocks(cols));
    const bool bf16 = dtype == MSSA_BF16;
    const int64_t step = mssa::mx_launch_rows(a.blocks);
    for (int64_t row = 0; row < rows; row += step) {
      const void* v = at_byte(values, row * a.stride * elem_bytes(dtype));
      a.in = quantize ? v : nullptr;
      a.out = quantize ? nullptr : const_cast<void*>(v);
      a.codes = const_cast<void*>(at_byte(codes, row * a.blocks * 16));
      a.scales = const_cast<void*>(at_byte(scales, row * a.blocks));
      a.rows = std::min(step, rows - row);
      const mssa_status launched = check_device(quantize ? mssa::launch_mx_quantize(a, bf16, stream_of(stream))
                                                         : mssa::launch_mx_dequantize(a, bf16, stream_of(stream)),
                                                who);
      if (launched != MSSA_OK) return launched;
    }
    return MSSA_OK;
  });
}

mssa_status attention_check(const mssa_mx_attention_desc* d) {
  if (!d) return fail(MSSA_ERR_INVALID_ARG, "null argument");
  if (d->batch < 1 || d->n_q < 1 || d->q_heads < 1 || d->kv_heads < 1)
    return fail(MSSA_ERR_INVALID_ARG, "batch, n_q and head counts must be positive");
  if (d->q_heads % d->kv_heads != 0) return fail(MSSA_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads");
  if (d->head_dim != 64 && d->head_dim != 128) return fail(MSSA_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (d->cache_tokens < 1 || d->cache_tokens > 0x7fffffff)
    return fail(MSSA_ERR_INVALID_ARG, "cache_tokens must be in [1, 2^31)");
  if (d->lse_stride != 0 && (d->lse_stride < d->n_q || d->lse_stride > (int64_t{1} << 40)))
    return fail(MSSA_ERR_INVALID_ARG, "lse_stride is shorter than n_q, or too long");
  if (!std::isfinite(d->softmax_scale)) return fail(MSSA_ERR_INVALID_ARG, "softmax_scale must be finite");
  if (static_cast<int64_t>(d->n_q) * (d->q_heads / d->kv_heads) > 0x3fffffff ||
      static_cast<int64_t>(d->batch) * d->q_heads > 0x3fffffff)
    return fail(MSSA_ERR_UNSUPPORTED, "too many query rows or heads");
  // the kernels' byte offsets inside a tile of 64 tokens have 32 bits: 2^16 heads x 64 bytes x 64 tokens
  if (d->kv_heads > (1 << 16)) return fail(MSSA_ERR_UNSUPPORTED, "more than 65536 key heads");
  return MSSA_OK;
}

mssa_status plan_of(const mssa_mx_attention_desc* d, mssa::MxAttnPlan* plan) {
  if (mssa::plan_mx_attention(d->batch, d->n_q, d->q_heads, d->kv_heads, d->head_dim, d->cache_tokens, plan) != hipSuccess)
    return fail(MSSA_ERR_UNSUPPORTED, "too many query rows or heads");
  return MSSA_OK;
}

}  // namespace

extern "C" {

mssa_status mssa_add_rms_norm(const mssa_norm_desc* desc, const void* x, const void* residual, const void* weight,
                              void* sum, void* y, float* y_scale, float* rstd, void* stream) {
  return guarded("mssa_add_rms_norm", [&]() -> mssa_status {
    const mssa_status s = norm_check(desc);
    if (s != MSSA_OK) return s;
    const bool e4m3 = desc->out_dtype == MSSA_E4M3;
    if (e4m3 != (y_scale != nullptr) && desc->rows > 0)
      return fail(MSSA_ERR_INVALID_ARG, "y_scale belongs to MSSA_E4M3 outputs and only to them");
    if ((residual != nullptr) != (sum != nullptr) && desc->rows > 0)
      return fail(MSSA_ERR_INVALID_ARG, "residual and sum come together");
    if (desc->rows == 0) return MSSA_OK;
    if (!x || !weight || !y) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    const int eb = elem_bytes(desc->dtype);
    for (const void* t : {x, residual, weight, static_cast<const void*>(sum)})
      if (!aligned_to(t, eb)) return fail(MSSA_ERR_INVALID_ARG, "a tensor is not aligned to its type");
    if (!(e4m3 ? aligned16(y) : aligned_to(y, eb)) || !aligned_to(y_scale, 4) || !aligned_to(rstd, 4))
      return fail(MSSA_ERR_INVALID_ARG, "an output is not aligned");
    if (y == x || y == residual || y == sum) return fail(MSSA_ERR_INVALID_ARG, "y must not alias x, residual or sum");
    mssa::NormArgs a{};
    a.x_stride = stride_or(desc->x_stride, desc->cols);
    a.residual_stride = stride_or(desc->residual_stride, desc->cols);
    a.sum_stride = stride_or(desc->sum_stride, desc->cols);
    if (sum && ((sum == x && a.sum_stride != a.x_stride) || (sum == residual && a.sum_stride != a.residual_stride)))
      return fail(MSSA_ERR_INVALID_ARG, "sum may be x or residual only with the same stride");
    a.weight = weight;
    a.cols = desc->cols;
    a.y_pitch = e4m3 ? static_cast<int32_t>(mssa::mx_blocks(desc->cols) * mssa::kMxBlock) : desc->cols;
    a.eps = desc->eps;
    a.inv_cols = 1.f / static_cast<float>(desc->cols);
    const int64_t step = mssa::norm_launch_rows(a.y_pitch);
    for (int64_t row = 0; row < desc->rows; row += step) {
      a.x = at_byte(x, row * a.x_stride * eb);
      a.residual = at_byte(residual, row * a.residual_stride * eb);
      a.sum = at_byte(sum, row * a.sum_stride * eb);
      a.y = at_byte(y, row * a.y_pitch * (e4m3 ? 1 : eb));
      a.y_scale = y_scale ? y_scale + row : nullptr;
      a.rstd = rstd ? rstd + row : nullptr;
      a.rows = std::min(step, desc->rows - row);
      const mssa_status launched =
          check_device(mssa::launch_norm(a, desc->dtype == MSSA_BF16, e4m3, stream_of(stream)), "norm launch");
      if (launched != MSSA_OK) return launched;
    }
    return MSSA_OK;
  });
}

mssa_status mssa_add_rms_norm_workspace_size(const mssa_norm_desc* desc, int64_t* bytes) {
  return guarded("mssa_add_rms_norm_workspace_size", [&]() -> mssa_status {
    const mssa_status s = norm_check(desc);
    if (s != MSSA_OK) return s;
    if (!bytes) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    const int64_t blocks = mssa::norm_bwd_blocks(desc->rows, desc->cols);
    *bytes = blocks > 1 ? blocks * desc->cols * 4 : 0;
    return MSSA_OK;
  });
}

mssa_status mssa_add_rms_norm_backward(const mssa_norm_desc* desc, const void* sum, const void* weight,
                                       const float* rstd, const void* dy, const void* dsum, void* workspace,
                                       int64_t workspace_bytes, void* dx, float* dweight, void* stream) {
  return guarded("mssa_add_rms_norm_backward", [&]() -> mssa_status {
    const mssa_status s = norm_check(desc);
    if (s != MSSA_OK) return s;
    if (!dweight || !aligned_to(dweight, 4)) return fail(MSSA_ERR_INVALID_ARG, "dweight must be an fp32 pointer");
    const int eb = elem_bytes(desc->dtype);
    if (desc->rows > 0) {
      if (!sum || !weight || !rstd || !dy || !dx) return fail(MSSA_ERR_INVALID_ARG, "null argument");
      for (const void* t : {sum, weight, dy, dsum, static_cast<const void*>(dx)})
        if (!aligned_to(t, eb)) return fail(MSSA_ERR_INVALID_ARG, "a tensor is not aligned to its type");
      if (!aligned_to(rstd, 4)) return fail(MSSA_ERR_INVALID_ARG, "rstd must be aligned to 4 bytes");
      if (dx == sum) return fail(MSSA_ERR_INVALID_ARG, "dx must not alias sum");
    }
    mssa::NormBwdArgs a{};
    a.blocks = mssa::norm_bwd_blocks(desc->rows, desc->cols);
    if (a.blocks > 1) {
      if (!workspace || workspace_bytes < static_cast<int64_t>(a.blocks) * desc->cols * 4)
        return fail(MSSA_ERR_WORKSPACE, "workspace smaller than mssa_add_rms_norm_workspace_size");
      if (!aligned16(workspace)) return fail(MSSA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    }
    a.sum = sum;
    a.weight = weight;
    a.dy = dy;
    a.dsum = dsum;
    a.rstd = rstd;
    a.dx = dx;
    a.dweight = dweight;
    a.partial = static_cast<float*>(workspace);
    a.rows = desc->rows;
    a.sum_stride = stride_or(desc->sum_stride, desc->cols);
    a.cols = desc->cols;
    a.inv_cols = 1.f / static_cast<float>(desc->cols);
    return check_device(mssa::launch_norm_bwd(a, desc->dtype == MSSA_BF16, stream_of(stream)), "norm backward launch");
  });
}

mssa_status mssa_mx_quantize(int64_t rows, int32_t cols, int32_t dtype, const void* x, int64_t x_stride, void* codes,
                             void* scales, void* stream) {
  return mx_convert("mssa_mx_quantize", true, rows, cols, dtype, x, x_stride, codes, scales, stream);
}

mssa_status mssa_mx_dequantize(int64_t rows, int32_t cols, int32_t dtype, const void* codes, const void* scales,
                               void* y, int64_t y_stride, void* stream) {
  return mx_convert("mssa_mx_dequantize", false, rows, cols, dtype, y, y_stride, codes, scales, stream);
}

mssa_status mssa_mx_project(const mssa_mx_project_desc* desc, const void* x, const void* x_scales, const void* w,
                            const void* w_scales, const void* bias, void* const* y, void* stream) {
  return guarded("mssa_mx_project", [&]() -> mssa_status {
    if (!desc) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    if (desc->rows < 0 || desc->rows > (1 << 30)) return fail(MSSA_ERR_INVALID_ARG, "rows must be in [0, 2^30]");
    if (desc->in_features < 1 || desc->in_features > (1 << 20) || desc->out_features < 1 || desc->out_features > (1 << 20))
      return fail(MSSA_ERR_INVALID_ARG, "feature counts must be in [1, 2^20]");
    if (desc->parts < 1 || desc->parts > mssa::kMaxParts || desc->out_features % desc->parts != 0)
      return fail(MSSA_ERR_INVALID_ARG, "parts must be 1..8 and divide out_features");
    if (desc->x_format != MSSA_E4M3 && desc->x_format != MSSA_MXFP4)
      return fail(MSSA_ERR_INVALID_ARG, "x_format must be MSSA_E4M3 or MSSA_MXFP4");
    if (desc->out_dtype != MSSA_BF16 && desc->out_dtype != MSSA_F32)
      return fail(MSSA_ERR_INVALID_ARG, "out_dtype must be bf16 or fp32");
    if (!std::isfinite(desc->part0_scale)) return fail(MSSA_ERR_INVALID_ARG, "part0_scale must be finite");
    if (desc->rows == 0) return MSSA_OK;
    if (!x || !x_scales || !w || !w_scales || !y) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    for (const void* t : {x, x_scales, w, w_scales, bias})
      if (!aligned16(t)) return fail(MSSA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
    const int64_t blocks = mssa::mx_blocks(desc->in_features);
    mssa::ProjectPlan plan;
    if (mssa::plan_mx_project(static_cast<int32_t>(desc->rows), desc->out_features, static_cast<int32_t>(blocks),
                              desc->x_format == MSSA_MXFP4, &plan) != hipSuccess)
      return fail(MSSA_ERR_UNSUPPORTED, "too many outputs for one launch");
    mssa::ProjectArgs a{};
    for (int p = 0; p < desc->parts; ++p) {
      if (!y[p]) return fail(MSSA_ERR_INVALID_ARG, "null output");
      if (!aligned16(y[p])) return fail(MSSA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
      for (const void* t : {x, x_scales, w, w_scales, bias})
        if (t == y[p]) return fail(MSSA_ERR_INVALID_ARG, "outputs must not alias the inputs");
      a.y[p] = y[p];
    }
    a.x = x;
    a.xs = x_scales;
    a.w = w;
    a.ws = w_scales;
    a.bias = bias;
    a.M = static_cast<int32_t>(desc->rows);
    a.N = desc->out_features;
    a.NB = static_cast<int32_t>(blocks);
    a.split = desc->out_features / desc->parts;
    a.part0_scale = desc->part0_scale;
    return check_device(mssa::launch_mx_project(a, desc->x_format == MSSA_MXFP4, desc->out_dtype == MSSA_BF16,
                                                stream_of(stream)),
                        "projection launch");
  });
}

mssa_status mssa_mx_attention_workspace_size(const mssa_mx_attention_desc* desc, int64_t* bytes) {
  return guarded("mssa_mx_attention_workspace_size", [&]() -> mssa_status {
    const mssa_status s = attention_check(desc);
    if (s != MSSA_OK) return s;
    if (!bytes) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    mssa::MxAttnPlan plan;
    const mssa_status planned = plan_of(desc, &plan);
    if (planned == MSSA_OK) *bytes = plan.workspace_bytes;
    return planned;
  });
}

mssa_status mssa_mx_attention(const mssa_mx_attention_desc* desc, const void* q, const void* k_codes,
                              const void* k_scales, const void* v_codes, const void* v_scales, const int32_t* kv_len,
                              const void* prior_out, const float* prior_lse, void* workspace,
                              int64_t workspace_bytes, void* out, float* lse, void* stream) {
  return guarded("mssa_mx_attention", [&]() -> mssa_status {
    const mssa_status s = attention_check(desc);
    if (s != MSSA_OK) return s;
    if (!q || !k_codes || !k_scales || !v_codes || !v_scales || !out) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    if ((prior_out != nullptr) != (prior_lse != nullptr))
      return fail(MSSA_ERR_INVALID_ARG, "prior_out and prior_lse come together");
    for (const void* t : {q, k_codes, k_scales, v_codes, v_scales, prior_out, static_cast<const void*>(out)})
      if (!aligned16(t)) return fail(MSSA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
    for (const void* t : {static_cast<const void*>(kv_len), static_cast<const void*>(prior_lse), static_cast<const void*>(lse)})
      if (!aligned_to(t, 4)) return fail(MSSA_ERR_INVALID_ARG, "kv_len and lse must be aligned to 4 bytes");
    if (out == q) return fail(MSSA_ERR_INVALID_ARG, "out must not alias q");
    mssa::MxAttnPlan plan;
    if (const mssa_status planned = plan_of(desc, &plan); planned != MSSA_OK) return planned;
    if (plan.workspace_bytes > 0) {
      if (!workspace || workspace_bytes < plan.workspace_bytes)
        return fail(MSSA_ERR_WORKSPACE, "workspace smaller than mssa_mx_attention_workspace_size");
      if (!aligned16(workspace)) return fail(MSSA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    }
    mssa::MxAttnArgs a{};
    a.q = q;
    a.kc = k_codes;
    a.ks = k_scales;
    a.vc = v_codes;
    a.vs = v_scales;
    a.kv_len = kv_len;
    a.prior_out = prior_out;
    a.prior_lse = prior_lse;
    a.out = out;
    a.lse = lse;
    a.partial = static_cast<float*>(workspace);
    a.cache_tokens = desc->cache_tokens;
    a.lse_stride = desc->lse_stride ? desc->lse_stride : desc->n_q;
    a.batch = desc->batch;
    a.n_q = desc->n_q;
    a.q_heads = desc->q_heads;
    a.kv_heads = desc->kv_heads;
    a.group = desc->q_heads / desc->kv_heads;
    a.rows = desc->n_q * a.group;
    a.items = plan.items;
    a.workers = plan.workers;
    a.slot_rows = plan.slot_rows;
    a.head_waves = plan.head_waves;
    const double scale = desc->softmax_scale > 0.f ? static_cast<double>(desc->softmax_scale)
                                                   : 1.0 / std::sqrt(static_cast<double>(desc->head_dim));
    a.scale_log2e = static_cast<float>(scale * 1.4426950408889634);
    return check_device(mssa::launch_mx_attention(a, plan, desc->head_dim, stream_of(stream)), "MXFP4 attention launch");
  });
}

}  // extern "C"
