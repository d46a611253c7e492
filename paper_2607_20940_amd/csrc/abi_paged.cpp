// C ABI of the operators for streams served together (declared in
// include/libmssa.h): every call is checked before anything is enqueued.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "abi_status.hpp"
#include "paged_args.hpp"

namespace {

using mssa::aligned16;
using mssa::check_device;
using mssa::fail;
using mssa::guarded;

bool aligned_to(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }
hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }
int64_t stride_or(int64_t stride, int64_t cols) { return stride ? stride : cols; }

constexpr int64_t kMaxRows = int64_t{1} << 30;

// rows x stride elements stay addressable in 63 bits.
bool stride_ok(int64_t stride, int64_t cols) { return stride == 0 || (stride >= cols && stride <= (int64_t{1} << 28)); }
// Rows are read in pieces of 16 bytes.
bool packed_stride_ok(int64_t stride, int64_t cols) { return stride_ok(stride, cols) && stride % 8 == 0; }

// What a packed batch over pages has in common.
template <class Desc>
mssa_status pages_check(const Desc* d) {
  if (d->tokens < 0 || d->tokens > kMaxRows) return fail(MSSA_ERR_INVALID_ARG, "tokens must be in [0, 2^30]");
  if (d->batch < 1 || d->batch > (1 << 20)) return fail(MSSA_ERR_INVALID_ARG, "batch must be in [1, 2^20]");
  if (d->kv_heads < 1 || d->kv_heads > (1 << 16) || d->q_heads < 0 || d->q_heads > (1 << 16))
    return fail(MSSA_ERR_INVALID_ARG, "head counts must be positive and at most 65536");
  if (d->page_tokens < 1 || d->page_tokens > (1 << 20)) return fail(MSSA_ERR_INVALID_ARG, "page_tokens must be in [1, 2^20]");
  if (d->table_pages < 1 || d->pages < 1) return fail(MSSA_ERR_INVALID_ARG, "table_pages and pages must be positive");
  if (static_cast<int64_t>(d->table_pages) * d->page_tokens > 0x7fffffff || d->pages > 0x7fffffff / d->page_tokens)
    return fail(MSSA_ERR_UNSUPPORTED, "2^31 tokens of pages, or more");
  return MSSA_OK;
}

// Without chunk_begin every sequence has as many rows.
mssa_status even_check(int64_t tokens, int32_t batch, const int32_t* chunk_begin) {
  if (!chunk_begin && tokens % batch != 0)
    return fail(MSSA_ERR_INVALID_ARG, "tokens must be a multiple of batch without chunk_begin");
  return MSSA_OK;
}

mssa_status project_check(const mssa_adapter_project_desc* d) {
  if (!d) return fail(MSSA_ERR_INVALID_ARG, "null argument");
  if (d->rows < 0 || d->rows > kMaxRows) return fail(MSSA_ERR_INVALID_ARG, "rows must be in [0, 2^30]");
  if (d->in_features < 1 || d->in_features > (1 << 20) || d->out_features < 1 || d->out_features > (1 << 20))
    return fail(MSSA_ERR_INVALID_ARG, "feature counts must be in [1, 2^20]");
  if (d->parts < 1 || d->parts > mssa::kMaxParts || d->out_features % d->parts != 0)
    return fail(MSSA_ERR_INVALID_ARG, "parts must be 1..8 and divide out_features");
  if (d->segments < 0 || d->segments > (1 << 20) || d->adapters < 0 || d->adapters > (1 << 20))
    return fail(MSSA_ERR_INVALID_ARG, "segments and adapters must be in [0, 2^20]");
  if (d->rank < (d->segments && d->adapters ? 1 : 0)) return fail(MSSA_ERR_INVALID_ARG, "rank must be positive");
  if (d->rank > 256) return fail(MSSA_ERR_UNSUPPORTED, "rank above 256");
  if (!std::isfinite(d->part0_scale)) return fail(MSSA_ERR_INVALID_ARG, "part0_scale must be finite");
  if (!stride_ok(d->x_stride, d->in_features)) return fail(MSSA_ERR_INVALID_ARG, "x_stride is shorter than in_features, or too long");
  return MSSA_OK;
}

mssa_status plan_of(const mssa_adapter_project_desc* d, mssa::AdapterPlan* plan) {
  if (mssa::plan_adapter_project(d->rows, d->in_features, stride_or(d->x_stride, d->in_features), d->out_features, d->parts,
                                 d->segments, d->adapters, d->rank, plan) != hipSuccess)
    return fail(MSSA_ERR_UNSUPPORTED, "too many outputs for one launch");
  return MSSA_OK;
}

mssa_status attention_check(const mssa_paged_attention_desc* d) {
  if (!d) return fail(MSSA_ERR_INVALID_ARG, "null argument");
  if (const mssa_status s = pages_check(d); s != MSSA_OK) return s;
  if (d->q_heads < 1 || d->q_heads % d->kv_heads != 0)
    return fail(MSSA_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads");
  if (d->head_dim != 64 && d->head_dim != 128) return fail(MSSA_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (d->max_chunk < 1 || d->max_chunk > kMaxRows) return fail(MSSA_ERR_INVALID_ARG, "max_chunk must be in [1, 2^30]");
  if (d->mask_block < 0) return fail(MSSA_ERR_INVALID_ARG, "mask_block must not be negative");
  if (!packed_stride_ok(d->q_stride, static_cast<int64_t>(d->q_heads) * d->head_dim))
    return fail(MSSA_ERR_INVALID_ARG, "q_stride is shorter than a row, too long or no multiple of 8");
  if (d->lse_stride != 0 && (d->lse_stride < d->tokens || d->lse_stride > (int64_t{1} << 40)))
    return fail(MSSA_ERR_INVALID_ARG, "lse_stride is shorter than tokens, or too long");
  if (!std::isfinite(d->softmax_scale)) return fail(MSSA_ERR_INVALID_ARG, "softmax_scale must be finite");
  if (std::min<int64_t>(d->max_chunk, d->tokens) * (d->q_heads / d->kv_heads) > kMaxRows)
    return fail(MSSA_ERR_UNSUPPORTED, "too many query rows");
  return MSSA_OK;
}

mssa_status plan_of(const mssa_paged_attention_desc* d, mssa::PagedAttnPlan* plan) {
  if (mssa::plan_paged_attention(d->tokens, d->batch, d->max_chunk, d->q_heads, d->kv_heads, d->head_dim,
                                 static_cast<int64_t>(d->table_pages) * d->page_tokens, plan) != hipSuccess)
    return fail(MSSA_ERR_UNSUPPORTED, "too many query rows or heads");
  return MSSA_OK;
}

}  // namespace

extern "C" {

mssa_status mssa_adapter_project_workspace_size(const mssa_adapter_project_desc* desc, int64_t* bytes) {
  return guarded("mssa_adapter_project_workspace_size", [&]() -> mssa_status {
    if (const mssa_status s = project_check(desc); s != MSSA_OK) return s;
    if (!bytes) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    mssa::AdapterPlan plan;
    const mssa_status planned = plan_of(desc, &plan);
    if (planned == MSSA_OK) *bytes = plan.workspace_bytes;
    return planned;
  });
}

mssa_status mssa_adapter_project(const mssa_adapter_project_desc* desc, const void* x, const void* w, const void* bias,
                                 const int32_t* segment_begin, const int32_t* adapter, const void* a, const void* b,
                                 const float* scale, void* workspace, int64_t workspace_bytes, void* const* y,
                                 void* stream) {
  return guarded("mssa_adapter_project", [&]() -> mssa_status {
    if (const mssa_status s = project_check(desc); s != MSSA_OK) return s;
    if (desc->rows == 0) return MSSA_OK;
    const bool low = desc->segments > 0 && desc->adapters > 0;
    if (!x || !w || !y) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    if (low && (!segment_begin || !adapter || !a || !b)) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    for (const void* t : {x, w, a})
      if (!aligned16(t)) return fail(MSSA_ERR_INVALID_ARG, "x, w and a must be 16-byte aligned");
    for (const void* t : {bias, b})
      if (!aligned_to(t, 2)) return fail(MSSA_ERR_INVALID_ARG, "a tensor is not aligned to its type");
    for (const void* t : {static_cast<const void*>(segment_begin), static_cast<const void*>(adapter), static_cast<const void*>(scale)})
      if (!aligned_to(t, 4)) return fail(MSSA_ERR_INVALID_ARG, "segments, adapters and scales must be aligned to 4 bytes");
    const int64_t x_stride = stride_or(desc->x_stride, desc->in_features);
    bool whole_y = desc->out_features / desc->parts % 8 == 0;
    for (int p = 0; p < desc->parts; ++p) whole_y = whole_y && aligned16(y[p]);
    mssa::AdapterPlan plan;
    if (const mssa_status planned = plan_of(desc, &plan); planned != MSSA_OK) return planned;
    if (plan.workspace_bytes > 0) {
      if (!workspace || workspace_bytes < plan.workspace_bytes)
        return fail(MSSA_ERR_WORKSPACE, "workspace smaller than mssa_adapter_project_workspace_size");
      if (!aligned16(workspace)) return fail(MSSA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    }
    mssa::AdapterArgs args{};
    for (int p = 0; p < desc->parts; ++p) {
      if (!y[p]) return fail(MSSA_ERR_INVALID_ARG, "null output");
      if (!aligned_to(y[p], 2)) return fail(MSSA_ERR_INVALID_ARG, "a tensor is not aligned to its type");
      for (const void* t : {x, w, bias, a, b})
        if (t == y[p]) return fail(MSSA_ERR_INVALID_ARG, "outputs must not alias the inputs");
      for (int o = 0; o < p; ++o)
        if (y[o] == y[p]) return fail(MSSA_ERR_INVALID_ARG, "outputs must not alias one another");
      args.y[p] = y[p];
    }
    args.x = x;
    args.w = w;
    args.bias = bias;
    args.a = a;
    args.b = b;
    args.segment_begin = segment_begin;
    args.adapter = adapter;
    args.scale = scale;
    args.low = workspace;
    args.x_stride = x_stride;
    args.M = static_cast<int32_t>(desc->rows);
    args.N = desc->out_features;
    args.K = desc->in_features;
    args.parts = desc->parts;
    args.split = desc->out_features / desc->parts;
    args.segments = low ? desc->segments : 0;
    args.adapters = desc->adapters;
    args.rank = desc->rank;
    args.low_rank = plan.low_rank;
    args.part0_scale = desc->part0_scale;
    args.whole = desc->in_features % 8 == 0 && x_stride % 8 == 0 && x_stride <= (1 << 21);
    args.whole_b = desc->rank % 8 == 0 && aligned16(b);
    args.whole_y = whole_y;
    return check_device(mssa::launch_adapter_project(args, plan, stream_of(stream)), "adapter projection launch");
  });
}

mssa_status mssa_paged_append(const mssa_paged_append_desc* desc, const void* q, const void* k, const void* v,
                              const int32_t* chunk_begin, const int32_t* kv_len, const int32_t* page_table,
                              const int32_t* positions, const float* freqs, void* q_out, void* k_pages, void* v_pages,
                              void* stream) {
  return guarded("mssa_paged_append", [&]() -> mssa_status {
    if (!desc) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    if (const mssa_status s = pages_check(desc); s != MSSA_OK) return s;
    const int32_t d = desc->head_dim, turned = desc->rotate_dims;
    if (d < 16 || d > 256 || d % 16 != 0) return fail(MSSA_ERR_UNSUPPORTED, "head_dim must be a multiple of 16, 16..256");
    if (turned < 0 || turned > d || turned % 2 != 0)
      return fail(MSSA_ERR_INVALID_ARG, "rotate_dims must be even, 0..head_dim");
    if (desc->halves != 0 && desc->halves != 1) return fail(MSSA_ERR_INVALID_ARG, "halves must be 0 or 1");
    if (desc->halves && turned % 16 != 0) return fail(MSSA_ERR_UNSUPPORTED, "rotate_dims of halves must be a multiple of 16");
    if (desc->axes < 1 || desc->axes > 3) return fail(MSSA_ERR_INVALID_ARG, "axes must be 1..3");
    int64_t pairs = 0;
    for (int x = 0; x < desc->axes; ++x) {
      if (desc->axis_pairs[x] < 0) return fail(MSSA_ERR_INVALID_ARG, "axis_pairs must not be negative");
      pairs += desc->axis_pairs[x];
    }
    if (pairs != turned / 2) return fail(MSSA_ERR_INVALID_ARG, "axis_pairs must be rotate_dims / 2 in all");
    const int64_t q_cols = static_cast<int64_t>(desc->q_heads) * d, kv_cols = static_cast<int64_t>(desc->kv_heads) * d;
    if (!packed_stride_ok(desc->q_stride, q_cols) || !packed_stride_ok(desc->k_stride, kv_cols) ||
        !packed_stride_ok(desc->v_stride, kv_cols))
      return fail(MSSA_ERR_INVALID_ARG, "a row stride is shorter than a row, too long or no multiple of 8");
    if (const mssa_status s = even_check(desc->tokens, desc->batch, chunk_begin); s != MSSA_OK) return s;
    if (desc->tokens == 0) return MSSA_OK;
    if (!k || !v || !kv_len || !page_table || !k_pages || !v_pages) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    if ((q != nullptr) != (desc->q_heads > 0) || (q_out != nullptr) != (desc->q_heads > 0))
      return fail(MSSA_ERR_INVALID_ARG, "q and q_out belong to q_heads > 0 and only to it");
    if (turned > 0 && !freqs) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    if (!positions && desc->axes != 1) return fail(MSSA_ERR_INVALID_ARG, "several axes need positions");
    for (const void* t : {q, k, v, static_cast<const void*>(q_out), static_cast<const void*>(k_pages), static_cast<const void*>(v_pages)})
      if (!aligned16(t)) return fail(MSSA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
    for (const void* t : {static_cast<const void*>(chunk_begin), static_cast<const void*>(kv_len), static_cast<const void*>(page_table),
                          static_cast<const void*>(positions), static_cast<const void*>(freqs)})
      if (!aligned_to(t, 4)) return fail(MSSA_ERR_INVALID_ARG, "lengths, tables, positions and freqs must be aligned to 4 bytes");
    if (q_out && (q_out == k || q_out == v || (q_out == q && stride_or(desc->q_stride, q_cols) != q_cols)))
      return fail(MSSA_ERR_INVALID_ARG, "q_out may be q only where q is contiguous, and must not be k or v");
    if (k_pages == v_pages) return fail(MSSA_ERR_INVALID_ARG, "k_pages must not be v_pages");
    for (const void* t : {q, k, v, static_cast<const void*>(q_out)})
      if (t && (t == k_pages || t == v_pages)) return fail(MSSA_ERR_INVALID_ARG, "the pages must not alias the inputs");
    mssa::AppendArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.chunk_begin = chunk_begin;
    a.kv_len = kv_len;
    a.page_table = page_table;
    a.positions = positions;
    a.freqs = freqs;
    a.q_out = q_out;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.q_stride = stride_or(desc->q_stride, q_cols);
    a.k_stride = stride_or(desc->k_stride, kv_cols);
    a.v_stride = stride_or(desc->v_stride, kv_cols);
    a.pages = desc->pages;
    a.tokens = static_cast<int32_t>(desc->tokens);
    a.batch = desc->batch;
    a.each = chunk_begin ? 0 : a.tokens / desc->batch;
    a.q_heads = desc->q_heads;
    a.kv_heads = desc->kv_heads;
    a.head_dim = d;
    a.table_pages = desc->table_pages;
    a.pairs = turned / 2;
    a.halves = desc->halves;
    a.axis_end[0] = desc->axis_pairs[0];
    a.axis_end[1] = desc->axes > 1 ? desc->axis_pairs[0] + desc->axis_pairs[1] : desc->axis_pairs[0];
    const int32_t units = (desc->q_heads + 2 * desc->kv_heads) * (d / 16);
    a.block_tokens = mssa::append_block_tokens(desc->tokens, units);
    a.page = mssa::Divisor::of(static_cast<uint32_t>(desc->page_tokens));
    a.units = mssa::Divisor::of(static_cast<uint32_t>(units));
    a.head_units = mssa::Divisor::of(static_cast<uint32_t>(d / 16));
    const int64_t step = mssa::kLaunchThreads / mssa::kAppendThreads * a.block_tokens;
    for (int64_t t = 0; t < desc->tokens; t += step) {
      a.token0 = static_cast<int32_t>(t);
      a.token1 = static_cast<int32_t>(std::min(desc->tokens, t + step));
      const mssa_status launched = check_device(mssa::launch_paged_append(a, stream_of(stream)), "paged append launch");
      if (launched != MSSA_OK) return launched;
    }
    return MSSA_OK;
  });
}

mssa_status mssa_paged_attention_workspace_size(const mssa_paged_attention_desc* desc, int64_t* bytes) {
  return guarded("mssa_paged_attention_workspace_size", [&]() -> mssa_status {
    if (const mssa_status s = attention_check(desc); s != MSSA_OK) return s;
    if (!bytes) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    mssa::PagedAttnPlan plan;
    const mssa_status planned = plan_of(desc, &plan);
    if (planned == MSSA_OK) *bytes = plan.workspace_bytes;
    return planned;
  });
}

mssa_status mssa_paged_attention(const mssa_paged_attention_desc* desc, const void* q, const void* k_pages,
                                 const void* v_pages, const int32_t* chunk_begin, const int32_t* kv_len,
                                 const int32_t* page_table, const void* prior_out, const float* prior_lse,
                                 void* workspace, int64_t workspace_bytes, void* out, float* lse, void* stream) {
  return guarded("mssa_paged_attention", [&]() -> mssa_status {
    if (const mssa_status s = attention_check(desc); s != MSSA_OK) return s;
    if (const mssa_status s = even_check(desc->tokens, desc->batch, chunk_begin); s != MSSA_OK) return s;
    if (desc->tokens == 0) return MSSA_OK;
    if (!q || !k_pages || !v_pages || !kv_len || !page_table || !out) return fail(MSSA_ERR_INVALID_ARG, "null argument");
    if ((prior_out != nullptr) != (prior_lse != nullptr))
      return fail(MSSA_ERR_INVALID_ARG, "prior_out and prior_lse come together");
    for (const void* t : {q, k_pages, v_pages, prior_out, static_cast<const void*>(out)})
      if (!aligned16(t)) return fail(MSSA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
    for (const void* t : {static_cast<const void*>(chunk_begin), static_cast<const void*>(kv_len), static_cast<const void*>(page_table),
                          static_cast<const void*>(prior_lse), static_cast<const void*>(lse)})
      if (!aligned_to(t, 4)) return fail(MSSA_ERR_INVALID_ARG, "lengths, tables and lse must be aligned to 4 bytes");
    if (out == q || out == k_pages || out == v_pages) return fail(MSSA_ERR_INVALID_ARG, "out must not alias q or the pages");
    mssa::PagedAttnPlan plan;
    if (const mssa_status planned = plan_of(desc, &plan); planned != MSSA_OK) return planned;
    if (plan.workspace_bytes > 0) {
      if (!workspace || workspace_bytes < plan.workspace_bytes)
        return fail(MSSA_ERR_WORKSPACE, "workspace smaller than mssa_paged_attention_workspace_size");
      if (!aligned16(workspace)) return fail(MSSA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    }
    mssa::PagedAttnArgs a{};
    a.q = q;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.prior_out = prior_out;
    a.chunk_begin = chunk_begin;
    a.kv_len = kv_len;
    a.page_table = page_table;
    a.prior_lse = prior_lse;
    a.out = out;
    a.lse = lse;
    a.partial = static_cast<float*>(workspace);
    a.q_stride = stride_or(desc->q_stride, static_cast<int64_t>(desc->q_heads) * desc->head_dim);
    a.lse_stride = stride_or(desc->lse_stride, desc->tokens);
    a.pages = desc->pages;
    a.capacity = static_cast<int64_t>(desc->table_pages) * desc->page_tokens;
    a.tokens = static_cast<int32_t>(desc->tokens);
    a.batch = desc->batch;
    a.each = chunk_begin ? 0 : a.tokens / desc->batch;
    a.max_chunk = desc->max_chunk;
    a.q_heads = desc->q_heads;
    a.kv_heads = desc->kv_heads;
    a.group = desc->q_heads / desc->kv_heads;
    a.table_pages = desc->table_pages;
    a.mask_block = std::min(desc->mask_block, int32_t{1} << 30);
    while (a.slot_rows() < plan.slot_rows) ++a.slot_shift;
    a.workers = plan.workers;
    a.unit_shift = plan.unit_shift;
    a.extra = plan.extra;
    a.least = plan.least;
    a.page = mssa::Divisor::of(static_cast<uint32_t>(desc->page_tokens));
    a.by_group = mssa::Divisor::of(static_cast<uint32_t>(a.group));
    a.by_mask = mssa::Divisor::of(static_cast<uint32_t>(std::max(1, a.mask_block)));
    const double scale = desc->softmax_scale > 0.f ? static_cast<double>(desc->softmax_scale)
                                                   : 1.0 / std::sqrt(static_cast<double>(desc->head_dim));
    a.scale_log2e = static_cast<float>(scale * 1.4426950408889634);
    return check_device(mssa::launch_paged_attention(a, plan, desc->head_dim, stream_of(stream)), "paged attention launch");
  });
}

}  // extern "C"
