// Host harness of the C ABI of the operators for streams served together and of
// the rules that cut their work, built without any GPU code (under
// AddressSanitizer and UndefinedBehaviorSanitizer by
// tests/test_paged_host_sanitized.py).  The kernel launchers are replaced by
// stubs that check every address range the kernel would read or write, derived
// from its argument struct, against the buffers passed; buffers that the host
// reads (lengths, chunks) are real, all others are address ranges that are never
// dereferenced.  For attention the stub walks the shares as the workers and the
// joining launch do: every tile of every item is taken once, every item is
// written, and the slots that the join reads of an item are the slots that its
// workers write.
//
// Exit status 0 iff every check passed.  With the argument "plant" every
// workspace is 256 bytes shorter than the size the harness passes, a mistake the
// range checks must report.  With the argument "odd" boundaries of chunks and
// segments are anything (negative, past the rows, decreasing) and the stubs take the
// kernels' look-ups step by step, with their 32-bit sums: whatever the values are, no
// row, table entry, tile or slot lies outside and every walk ends.
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
#include "../../paper_2607_20940_amd/csrc/paged_args.hpp"

namespace {

int g_failures = 0, g_checks = 0, g_launches = 0;
bool g_plant = false, g_walk = true, g_odd = false;
std::string g_case, g_error;

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
void* dev_alloc(int64_t bytes) {
  const uintptr_t b = g_next;
  g_next += uintptr_t{1} << 41;
  g_bufs.push_back({b, b + static_cast<uintptr_t>(std::max<int64_t>(bytes, 0))});
  return reinterpret_cast<void*>(b);
}
void dev_reset() {
  g_bufs.clear();
  g_next = uintptr_t{1} << 44;
}
void check_range(const void* p, int64_t bytes, const char* what) {
  ++g_checks;
  if (bytes <= 0) return;
  const uintptr_t b = reinterpret_cast<uintptr_t>(p);
  for (const Range& r : g_bufs)
    if (b >= r.b && b < r.e) {
      if (b + static_cast<uintptr_t>(bytes) > r.e) failure((std::string(what) + ": overrun").c_str());
      return;
    }
  failure((std::string(what) + ": address outside every buffer").c_str());
}
int64_t span(int64_t rows, int64_t cols, int64_t stride) { return rows ? ((rows - 1) * stride + cols) * 2 : 0; }

uint64_t g_seed = 88172645463325252ull;
int64_t pick(int64_t lo, int64_t hi) {
  g_seed ^= g_seed << 13;
  g_seed ^= g_seed >> 7;
  g_seed ^= g_seed << 17;
  return lo + static_cast<int64_t>(g_seed % static_cast<uint64_t>(hi - lo + 1));
}

}  // namespace

extern "C" const char* hipGetErrorString(hipError_t) { return "stub"; }

namespace mssa {
namespace {

// Every chunk's rows lie in the batch, whatever the boundaries are.
void rows_inside(const int32_t* begin, int batch, int32_t tokens) {
  for (int b = 0; b < batch; ++b) {
    const ChunkRows c = ChunkRows::of(begin, b, 0, tokens);
    check(0 <= c.first && c.first <= c.end && c.end <= tokens, "a chunk's rows");
  }
}

// The look-up of a row's sequence, 64 probes at a time (append).
void find_row(const AppendArgs& a, int32_t row) {
  int32_t lo = 0, n = a.batch;
  int rounds = 0;
  while (n > 64 && ++rounds < 8) {
    const int32_t step = (n + 63) / 64;
    int last = 0;
    for (int lane = 0; lane < 64; ++lane) {
      const int32_t at = lo + lane * step;
      if (lane * step < n && a.chunk_begin[at < a.batch ? at : a.batch] <= row) last = lane;
    }
    n = std::min(n - last * step, step);
    lo += last * step;
  }
  check(n >= 1 && n <= 64 && lo >= 0 && lo + n <= a.batch, "a row's sequence");
  for (int lane = n - 1; lane >= 0; --lane) {
    const int32_t b = lo + lane;
    if (!(a.chunk_begin[b] <= row && row < a.chunk_begin[b + 1])) continue;
    const ChunkRows c = ChunkRows::of(a.chunk_begin, b, 0, a.tokens);
    const int64_t index = int64_t{a.kv_len[b]} - (c.end - row);
    if (index >= 0 && index < int64_t{a.table_pages} * a.page.d)
      check(static_cast<int32_t>(a.page.quotient(static_cast<uint32_t>(index))) < a.table_pages, "a page table's entry");
    return;
  }
}

// Rows of the low-rank factor's tiles, and the first segment behind a row (projection).
void odd_segments(const AdapterArgs& a, const AdapterPlan& plan) {
  rows_inside(a.segment_begin, a.segments, a.M);
  for (int32_t tile = 0; tile < plan.low_tiles; ++tile) {
    int32_t left = tile;
    bool found = false;
    for (int32_t c = 0; c < a.segments && !found; c += 64) {
      int32_t pre = 0;
      for (int32_t s = c; s < std::min(a.segments, c + 64) && !found; ++s) {
        const ChunkRows g = ChunkRows::of(a.segment_begin, s, 0, a.M);
        const int32_t mine = (g.end - g.first + plan.low_rows - 1) / plan.low_rows, before = pre;
        pre += mine;
        if (pre <= left) continue;
        found = true;
        const int32_t at = left - before, first = g.first + at * plan.low_rows;
        check(at < 0 || first >= g.end || (first >= 0 && first < a.M), "a low-rank tile's rows");
      }
      left -= pre;
    }
  }
  for (int32_t row = 0; row < a.M; row += 16) {
    int32_t lo = 0, n = a.segments;
    int rounds = 0;
    while (n > 0 && ++rounds < 64) {
      const int32_t step = (n + 63) / 64;
      int last = -1;
      for (int lane = 0; lane < 64; ++lane) {
        const int32_t at = lo + lane * step;
        if (lane * step < n && a.segment_begin[(at < a.segments ? at : 0) + 1] <= row) last = lane;
      }
      if (last < 0) break;
      const int32_t skip = last * step + 1;
      n = std::min(n - skip, step - 1);
      lo += skip;
    }
    check(rounds < 64 && lo >= 0 && lo <= a.segments, "the first segment behind a row");
  }
}

// The shares of chunks that may overlap: sums are taken in 32 bits, as the workers take them.
void odd_shares(const PagedAttnArgs& a, const PagedAttnPlan& plan) {
  rows_inside(a.chunk_begin, a.batch, a.tokens);
  std::vector<PagedSeq> seqs;
  uint32_t all = 0;
  for (int b = 0; b < a.batch; ++b) {
    seqs.push_back(PagedSeq::of(a, b));
    const PagedSeq& s = seqs.back();
    check(s.n >= 0 && s.n <= a.max_chunk && s.first + s.n <= a.tokens && s.len >= 0 && s.len <= a.capacity, "a sequence's rows and length");
    all += s.head_units() * static_cast<uint32_t>(a.kv_heads);
  }
  Shares sh = Shares::of(all, all);
  if (a.workers) {
    const uint32_t most = all / static_cast<uint32_t>(a.least);
    sh = Shares::of(all, most < 1 ? 1 : std::min(most, static_cast<uint32_t>(a.workers)));
  }
  struct Spot {
    int b = -1, kvh = 0, item = 0;
    uint32_t unit = 0;
  };
  auto spot = [&](uint32_t w) {
    Spot at;
    if (w >= sh.workers) return at;
    const uint32_t x = sh.first(w);
    uint32_t base = 0;
    for (int b = 0; b < a.batch; ++b) {
      const uint32_t units = seqs[b].head_units() * static_cast<uint32_t>(a.kv_heads);
      base += units;
      if (base <= x) continue;
      const uint32_t y = x - (base - units);
      if (y >= units) return at;
      const uint32_t head = seqs[b].head_units();
      at.b = b;
      at.kvh = static_cast<int>(y / head);
      at.item = seqs[b].item_of(y - at.kvh * head);
      at.unit = y - at.kvh * head - seqs[b].before(at.item);
      return at;
    }
    return at;
  };
  for (uint32_t w = 0; w < plan.blocks; ++w) {
    Spot at = spot(w);
    if (at.b < 0) continue;
    uint32_t todo = sh.first(w + 1) - sh.first(w);
    int64_t pieces = 0;
    for (int seg = 0;; ++seg) {
      const PagedSeq& s = seqs[at.b];
      check(at.kvh >= 0 && at.kvh < a.kv_heads && at.item >= 0 && at.item < s.items, "a worker's item");
      const int tiles = s.tiles(at.item, a);
      const uint32_t cost = s.cost(at.item), take = std::min(todo, cost - at.unit);
      check(at.unit < cost && take > 0, "a worker goes on");
      if (at.unit >= cost || !take || ++pieces > 1 << 20) break;
      const int t0 = PagedSeq::tile_at(at.unit, tiles, cost), t1 = PagedSeq::tile_at(at.unit + take, tiles, cost);
      check(0 <= t0 && t0 <= t1 && t1 <= (s.len + kPagedTile - 1) / kPagedTile, "a piece's tiles");
      check(take == cost || (a.workers && 2 * w + (seg > 0) < 2 * static_cast<uint32_t>(a.workers)), "a piece's slot");
      todo -= take;
      at.unit = 0;
      if (!todo) break;
      if (++at.item < s.items) continue;
      at.item = 0;
      if (++at.kvh < a.kv_heads) continue;
      at.kvh = 0;
      do ++at.b;
      while (at.b < a.batch && seqs[at.b].items == 0);
      if (at.b >= a.batch) break;
    }
  }
  for (uint32_t j = 0; a.workers && j + 1 < static_cast<uint32_t>(a.workers); ++j) {
    const Spot at = spot(j + 1);
    const uint32_t start = sh.first(j + 1) - at.unit;
    if (at.b < 0 || at.unit == 0 || sh.first(j) > start) continue;
    const uint32_t w1 = std::min(sh.worker_of(start + seqs[at.b].cost(at.item) - 1), sh.workers - 1);
    check(w1 < static_cast<uint32_t>(a.workers) && at.item < seqs[at.b].items, "slots that are joined");
  }
}

}  // namespace

mssa_status fail(mssa_status s, const char* msg) noexcept {
  g_error = msg;
  return s;
}
mssa_status fail(mssa_status s, const char* what, const char* detail) noexcept {
  g_error = std::string(what) + ": " + detail;
  return s;
}

hipError_t launch_paged_append(const AppendArgs& a, hipStream_t) {
  ++g_launches;
  const int64_t d = a.head_dim;
  check(a.token0 >= 0 && a.token0 < a.token1 && a.token1 <= a.tokens, "rows of the launch");
  check(a.block_tokens >= 1 && a.block_tokens <= kAppendMaxTokens && a.pairs <= kAppendMaxPairs, "the block's LDS");
  check((int64_t{a.token1} - a.token0 + a.block_tokens - 1) / a.block_tokens * kAppendThreads < int64_t{1} << 32, "threads of a launch");
  if (a.q_heads) {
    check_range(a.q, span(a.tokens, a.q_heads * d, a.q_stride), "q");
    check_range(a.q_out, span(a.tokens, a.q_heads * d, a.q_heads * d), "q_out");
  }
  check_range(a.k, span(a.tokens, a.kv_heads * d, a.k_stride), "k");
  check_range(a.v, span(a.tokens, a.kv_heads * d, a.v_stride), "v");
  const int64_t pool = a.pages * a.page.d * a.kv_heads * d * 2;
  check(a.pages * a.page.d <= 0x7fffffff, "slots have 31 bits");
  check_range(a.k_pages, pool, "k_pages");
  check_range(a.v_pages, pool, "v_pages");
  check_range(a.page_table, int64_t{a.batch} * a.table_pages * 4, "page_table");
  check(a.axis_end[0] <= a.axis_end[1] && a.axis_end[1] <= a.pairs, "axes");
  if (a.positions) check_range(a.positions, int64_t{a.tokens} * (a.axis_end[0] == a.pairs ? 1 : a.axis_end[1] == a.pairs ? 2 : 3) * 4, "positions");
  if (a.pairs) check_range(a.freqs, a.pairs * 4, "freqs");
  // the pieces of a token's heads, as the threads take them
  const uint32_t units = a.units.d, hu = a.head_units.d;
  check(units == (a.q_heads + 2 * a.kv_heads) * hu && hu * 16 == static_cast<uint32_t>(d), "pieces of a token");
  const uint32_t half = a.pairs / 8;
  std::vector<int> chunks(2 * hu, 0);
  for (uint32_t p = 0; p < hu; ++p) {
    uint32_t c0 = p, c1 = p + hu;
    if (a.halves && p < half) c1 = p + half;
    if (a.halves && p >= half) c0 = p + half;
    if (c0 < 2 * hu && c1 < 2 * hu) ++chunks[c0], ++chunks[c1];
  }
  check(std::all_of(chunks.begin(), chunks.end(), [](int n) { return n == 1; }), "every chunk of a head once");
  if (g_odd) {
    rows_inside(a.chunk_begin, a.batch, a.tokens);
    for (int32_t row = a.token0; row < a.token1; ++row) find_row(a, row);
  }
  return hipSuccess;
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, const PagedAttnPlan& plan, int d, hipStream_t) {
  ++g_launches;
  check_range(a.q, span(a.tokens, int64_t{a.q_heads} * d, a.q_stride), "q");
  check_range(a.out, span(a.tokens, int64_t{a.q_heads} * d, int64_t{a.q_heads} * d), "out");
  if (a.lse) check_range(a.lse, (int64_t{a.q_heads - 1} * a.lse_stride + a.tokens) * 4, "lse");
  if (a.prior_out) check_range(a.prior_out, span(a.tokens, int64_t{a.q_heads} * d, int64_t{a.q_heads} * d), "prior_out");
  if (a.prior_lse) check_range(a.prior_lse, (int64_t{a.q_heads - 1} * a.lse_stride + a.tokens) * 4, "prior_lse");
  const int64_t pool = a.pages * a.page.d * a.kv_heads * d * 2;
  check_range(a.k_pages, pool, "k_pages");
  check_range(a.v_pages, pool, "v_pages");
  check_range(a.page_table, int64_t{a.batch} * a.table_pages * 4, "page_table");
  check(a.slot_rows() == plan.slot_rows && plan.slot_rows % plan.join_rows == 0, "rows of an item");
  check(plan.slot_rows == (plan.waves ? plan.waves * 32 : plan.slot_rows), "rows of a block");
  check(a.workers <= kPagedMaxWorkers && plan.blocks * plan.threads() < int64_t{1} << 32, "blocks");
  if (a.workers) {
    const int64_t slots = 2 * int64_t{a.workers} * a.slot_rows();
    check_range(a.partial, slots * (d + 2) * 4, "workspace");
  }
  if (!g_walk) return hipSuccess;
  if (g_odd) {
    odd_shares(a, plan);
    return hipSuccess;
  }

  // The shares, as find_share and next_item see them.
  std::vector<PagedSeq> seqs;
  uint64_t all = 0;
  std::vector<uint32_t> begin;
  for (int b = 0; b < a.batch; ++b) {
    seqs.push_back(PagedSeq::of(a, b));
    const PagedSeq& s = seqs.back();
    check(s.first >= 0 && s.n >= 0 && s.first + s.n <= a.tokens && s.len >= 0 && s.len <= a.capacity, "a sequence's rows and length");
    check(plan.waves || s.items <= 1, "few rows are one item");
    begin.push_back(static_cast<uint32_t>(all));
    all += uint64_t{s.head_units()} * a.kv_heads;
    for (int i = 0; i < s.items; ++i) {
      check(s.item_of(s.before(i)) == i && s.item_of(s.before(i + 1) - 1) == i, "the item of a unit");
      check(s.cost(i) == s.before(i + 1) - s.before(i) && s.cost(i) > 0, "an item's units");
      check(s.tiles(i, a) <= (s.len + kPagedTile - 1) / kPagedTile, "an item's tiles");
    }
  }
  check(all <= 0x7fffffff, "units have 31 bits");
  Shares sh = Shares::of(static_cast<uint32_t>(all), static_cast<uint32_t>(all));
  if (a.workers) {
    const uint32_t most = static_cast<uint32_t>(all) / static_cast<uint32_t>(a.least), workers = static_cast<uint32_t>(a.workers);
    sh = Shares::of(static_cast<uint32_t>(all), most < 1 ? 1 : std::min(most, workers));
  }
  check(sh.workers <= plan.blocks, "a block a worker");
  struct Key {
    int b, kvh, item;
    bool operator<(const Key& o) const { return std::tie(b, kvh, item) < std::tie(o.b, o.kvh, o.item); }
  };
  std::map<Key, std::vector<int>> taken;       // tiles
  std::map<Key, std::vector<uint32_t>> slots;  // written, in the workers' order
  std::map<Key, int> direct;
  auto spot = [&](uint32_t x, uint32_t* unit) {
    int b = 0;
    while (b + 1 < a.batch && begin[b + 1] <= x) ++b;
    const uint32_t y = x - begin[b], head = seqs[b].head_units();
    const int kvh = static_cast<int>(y / head), item = seqs[b].item_of(y - kvh * head);
    *unit = y - kvh * head - seqs[b].before(item);
    return Key{b, kvh, item};
  };
  for (uint32_t w = 0; w < sh.workers; ++w) {
    uint32_t unit, todo = sh.first(w + 1) - sh.first(w);
    Key at = spot(sh.first(w), &unit);
    check(todo > 0, "a worker's share");
    for (int seg = 0; todo; ++seg) {
      const PagedSeq& s = seqs[at.b];
      const int tiles = s.tiles(at.item, a);
      const uint32_t cost = s.cost(at.item), take = std::min(todo, cost - unit);
      const int t0 = PagedSeq::tile_at(unit, tiles, cost), t1 = PagedSeq::tile_at(unit + take, tiles, cost);
      check(0 <= t0 && t0 <= t1 && t1 <= tiles, "a piece's tiles");
      auto& n = taken[at];
      n.resize(tiles);
      for (int t = t0; t < t1; ++t) ++n[t];
      if (take == cost)
        ++direct[at];
      else
        slots[at].push_back(2 * w + (seg > 0));
      check(take == cost || seg == 0 || take == todo, "a shared item is a worker's first or last");
      todo -= take;
      unit = 0;
      if (!todo) break;
      if (++at.item == s.items) {
        at.item = 0;
        if (++at.kvh == a.kv_heads) {
          at.kvh = 0;
          do ++at.b;
          while (at.b < a.batch && seqs[at.b].items == 0);
        }
      }
    }
  }
  std::map<Key, int> joined;
  for (uint32_t j = 0; j + 1 < sh.workers; ++j) {  // as the joining launch's blocks
    uint32_t unit;
    const Key at = spot(sh.first(j + 1), &unit);
    const uint32_t start = sh.first(j + 1) - unit;
    if (unit == 0 || sh.first(j) > start) continue;
    const uint32_t w1 = sh.worker_of(start + seqs[at.b].cost(at.item) - 1);
    std::vector<uint32_t> read{sh.first(j) != start ? 2 * j + 1 : 2 * j};
    for (uint32_t w = j + 1; w <= w1; ++w) read.push_back(2 * w);
    check(read == slots[at], "the join reads an item's slots");
    check(read.size() <= static_cast<size_t>(kPagedMaxWorkers), "slots of an item");
    ++joined[at];
  }
  for (int b = 0; b < a.batch; ++b)
    for (int k = 0; k < a.kv_heads; ++k)
      for (int i = 0; i < seqs[b].items; ++i) {
        const Key at{b, k, i};
        check(direct[at] + joined[at] == 1, "every item is written once");
        auto& n = taken[at];
        n.resize(seqs[b].tiles(i, a));
        check(std::all_of(n.begin(), n.end(), [](int c) { return c == 1; }), "every tile is taken once");
      }
  return hipSuccess;
}

hipError_t launch_adapter_project(const AdapterArgs& a, const AdapterPlan& plan, hipStream_t) {
  ++g_launches;
  check_range(a.x, span(a.M, a.K, a.x_stride), "x");
  check_range(a.w, span(a.N, a.K, a.K), "w");
  if (a.bias) check_range(a.bias, int64_t{a.N} * 2, "bias");
  check(a.N == a.parts * a.split, "parts");
  for (int p = 0; p < a.parts; ++p) check_range(a.y[p], span(a.M, a.split, a.split), "y");
  static const int side[][2] = {{kAdapterFewTokens, kAdapterFewFeatures}, {64, 64}, {128, 128}, {256, 256}};
  const int* t = side[static_cast<int>(plan.kernel)];
  check(plan.blocks == (a.M + t[0] - 1) / t[0] * ((int64_t{a.N} + t[1] - 1) / t[1]), "a block a tile");
  check(plan.kernel != AdapterKernel::kFew || a.M <= kAdapterFewTokens, "few tokens");
  const bool few = plan.kernel == AdapterKernel::kFew;
  if (few)
    check(a.M > kAdapterFewOdd ? a.whole || plan.pack_x : plan.pack_x == (a.K < 8) && plan.pack_w == plan.pack_x, "odd rows of few are copied");
  else
    check(a.whole || plan.pack_x, "odd rows of many are copied");
  check(a.whole || a.M <= kAdapterFewOdd || plan.pack_w || a.K % 8 == 0, "odd weights are copied");
  const int64_t k8 = (a.K + 7) / 8 * 8, stride = plan.pack_x ? k8 : a.x_stride;
  if (a.M > kAdapterFewOdd || a.whole) {
    check(256 * stride * 2 + 128 < 0x7ffffff0 && 256 * k8 * 2 + 128 < 0x7ffffff0, "offsets inside a tile");
    check(stride % 8 == 0 && (reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) % 16 == 0, "whole chunks");
  }
  // the copies behind the low-rank factors
  int64_t copies = plan.pack_x ? a.M * k8 : 0;
  if (plan.pack_w) copies += (a.N + (a.segments ? int64_t{a.adapters} * a.parts * a.rank : 0)) * k8;
  check(copies / 8 <= kLaunchThreads, "threads of the copies");
  if (copies) check_range(static_cast<char*>(a.low) + plan.low_bytes, copies * 2, "workspace");
  check(plan.low_bytes % 256 == 0, "the copies' alignment");
  if (a.segments) {
    check_range(a.segment_begin, (int64_t{a.segments} + 1) * 4, "segment_begin");
    check_range(a.adapter, int64_t{a.segments} * 4, "adapter");
    check_range(a.a, int64_t{a.adapters} * a.parts * a.rank * a.K * 2, "a");
    check_range(a.b, int64_t{a.adapters} * a.N * a.rank * 2, "b");
    check_range(a.low, int64_t{a.M} * a.parts * a.low_rank * 2, "workspace");
    check(a.low_rank % 16 == 0 && a.low_rank >= a.rank && a.low_rank < a.rank + 16, "ranks rounded up");
    check(int64_t{256} * a.parts * a.low_rank * 2 < 0x7ffffff0, "offsets inside a tile");
    // the most tiles that segments of these rows can have
    check(plan.low_tiles >= std::min<int64_t>(a.M, a.segments + (a.M - 1) / plan.low_rows), "a block a tile of the low-rank factor");
    const int64_t cols = int64_t{a.parts} * a.low_rank;
    check(plan.low_columns % 16 == 0 && (plan.low_rows == kLowRows ? plan.low_columns == 16 : plan.low_columns <= 96) &&
              plan.low_across == (cols + plan.low_columns - 1) / plan.low_columns, "the low-rank factor's columns");
    check(plan.low_rows == kLowRows ? plan.low_tiles * 1024 < int64_t{1} << 32 : plan.low_tiles * plan.low_across * 256 < int64_t{1} << 32,
          "threads of the low-rank factor's launch");
    if (g_odd) odd_segments(a, plan);
  }
  return hipSuccess;
}

}  // namespace mssa

namespace {

std::vector<int32_t> g_begin, g_len;

void lengths(int batch, int64_t tokens, bool odd) {
  g_begin.assign(batch + 1, 0);
  for (int b = 1; b < batch; ++b) g_begin[b] = static_cast<int32_t>(pick(0, tokens));
  g_begin[batch] = static_cast<int32_t>(tokens);
  std::sort(g_begin.begin(), g_begin.end());
  if (odd && batch > 1) g_begin[pick(0, batch)] = static_cast<int32_t>(pick(-5, tokens + 5));  // may decrease: clamped
  g_len.assign(batch, 0);
  if (g_odd)
    for (int32_t& r : g_begin)
      if (!pick(0, 3)) r = static_cast<int32_t>(pick(0, 3) ? pick(-5, tokens + 5) : pick(0, 1) ? 0x7fffffff : -0x7fffffff - 1);
}

void attend(int64_t tokens, int batch, int max_chunk, int q_heads, int kv_heads, int d, int page, int table, int mask, int most) {
  dev_reset();
  mssa_paged_attention_desc desc{};
  desc.tokens = tokens;
  desc.batch = batch;
  desc.max_chunk = max_chunk;
  desc.q_heads = q_heads;
  desc.kv_heads = kv_heads;
  desc.head_dim = d;
  desc.page_tokens = page;
  desc.table_pages = table;
  desc.pages = pick(1, 50);
  desc.mask_block = mask;
  desc.q_stride = pick(0, 1) ? 0 : int64_t{q_heads} * d + 8 * pick(0, 3);
  desc.lse_stride = pick(0, 1) ? 0 : tokens + pick(0, 5);
  char name[200];
  std::snprintf(name, sizeof name, "attend tokens %" PRId64 " batch %d chunk %d heads %d/%d d %d page %d x %d mask %d", tokens, batch,
                max_chunk, q_heads, kv_heads, d, page, table, mask);
  g_case = name;
  lengths(batch, tokens, false);
  for (int b = 0; b < batch; ++b) g_len[b] = static_cast<int32_t>(pick(0, 9) ? pick(-3, most) : pick(0, 1) ? 0 : 0x7fffffff);
  int64_t bytes = 0;
  const mssa_status s = mssa_paged_attention_workspace_size(&desc, &bytes);
  check(s == MSSA_OK, g_error.c_str());
  if (s != MSSA_OK) return;
  const int64_t qs = desc.q_stride ? desc.q_stride : int64_t{q_heads} * d, ls = desc.lse_stride ? desc.lse_stride : tokens;
  void* q = dev_alloc(span(tokens, int64_t{q_heads} * d, qs));
  void* k = dev_alloc(desc.pages * page * kv_heads * d * 2);
  void* v = dev_alloc(desc.pages * page * kv_heads * d * 2);
  void* t = dev_alloc(int64_t{batch} * table * 4);
  void* ws = dev_alloc(bytes - (g_plant ? 256 : 0));
  void* out = dev_alloc(tokens * q_heads * d * 2);
  void* lse = dev_alloc((int64_t{q_heads - 1} * ls + tokens) * 4);
  const int before = g_launches;
  check(mssa_paged_attention(&desc, q, k, v, g_begin.data(), g_len.data(), static_cast<int32_t*>(t), out, static_cast<float*>(lse), ws,
                             bytes, out, static_cast<float*>(lse), nullptr) == MSSA_OK, g_error.c_str());
  check(g_launches == before + (tokens > 0), "launches");
}

void append(int64_t tokens, int batch, int q_heads, int kv_heads, int d, int page, int turned, int halves) {
  dev_reset();
  mssa_paged_append_desc desc{};
  desc.tokens = tokens;
  desc.batch = batch;
  desc.q_heads = q_heads;
  desc.kv_heads = kv_heads;
  desc.head_dim = d;
  desc.page_tokens = page;
  desc.table_pages = static_cast<int32_t>(pick(1, 20));
  desc.pages = pick(1, 50);
  desc.rotate_dims = turned;
  desc.halves = halves;
  desc.axes = static_cast<int32_t>(pick(1, 3));
  int left = turned / 2;
  for (int x = 0; x < desc.axes; ++x) {
    desc.axis_pairs[x] = x + 1 == desc.axes ? left : static_cast<int32_t>(pick(0, left));
    left -= desc.axis_pairs[x];
  }
  desc.q_stride = pick(0, 1) ? 0 : int64_t{q_heads} * d + 8 * pick(0, 3);
  desc.v_stride = pick(0, 1) ? 0 : int64_t{kv_heads} * d + 8 * pick(0, 3);
  char name[200];
  std::snprintf(name, sizeof name, "append tokens %" PRId64 " batch %d heads %d/%d d %d page %d turned %d halves %d", tokens, batch,
                q_heads, kv_heads, d, page, turned, halves);
  g_case = name;
  lengths(batch, tokens, true);
  const int64_t qs = desc.q_stride ? desc.q_stride : int64_t{q_heads} * d, vs = desc.v_stride ? desc.v_stride : int64_t{kv_heads} * d;
  void* q = q_heads ? dev_alloc(span(tokens, int64_t{q_heads} * d, qs)) : nullptr;
  void* k = dev_alloc(tokens * kv_heads * d * 2);
  void* v = dev_alloc(span(tokens, int64_t{kv_heads} * d, vs));
  void* t = dev_alloc(int64_t{batch} * desc.table_pages * 4);
  void* pos = dev_alloc(tokens * desc.axes * 4);
  void* freqs = dev_alloc(turned / 2 * 4);
  void* q_out = q_heads ? dev_alloc(tokens * q_heads * d * 2) : nullptr;
  void* kp = dev_alloc(desc.pages * page * kv_heads * d * 2);
  void* vp = dev_alloc(desc.pages * page * kv_heads * d * 2);
  check(mssa_paged_append(&desc, q, k, v, g_begin.data(), g_len.data(), static_cast<int32_t*>(t), static_cast<int32_t*>(pos),
                          static_cast<float*>(freqs), q_out, kp, vp, nullptr) == MSSA_OK, g_error.c_str());
}

void project(int64_t rows, int k, int n, int parts, int segments, int adapters, int rank, int pad) {
  dev_reset();
  mssa_adapter_project_desc desc{rows, k, n, parts, segments, adapters, rank, 1.f, pad ? k + pad : 0};
  char name[200];
  std::snprintf(name, sizeof name, "project %" PRId64 " x %d -> %d, parts %d, segments %d, adapters %d, rank %d, pad %d", rows, k, n,
                parts, segments, adapters, rank, pad);
  g_case = name;
  int64_t bytes = 0;
  check(mssa_adapter_project_workspace_size(&desc, &bytes) == MSSA_OK, g_error.c_str());
  void* x = dev_alloc(span(rows, k, k + pad));
  void* w = dev_alloc(int64_t{n} * k * 2);
  void* bias = dev_alloc(int64_t{n} * 2);
  void* seg = dev_alloc((int64_t{segments} + 1) * 4);
  void* which = dev_alloc(int64_t{segments} * 4);
  void* a = dev_alloc(int64_t{adapters} * parts * rank * k * 2);
  void* b = dev_alloc(int64_t{adapters} * n * rank * 2);
  void* ws = dev_alloc(bytes - (g_plant ? 256 : 0));
  void* y[8];
  for (int p = 0; p < parts; ++p) y[p] = dev_alloc(rows * (n / parts) * 2);
  if (g_odd) {
    lengths(segments, rows, true);
    seg = g_begin.data();
    g_bufs.push_back({reinterpret_cast<uintptr_t>(seg), reinterpret_cast<uintptr_t>(seg) + g_begin.size() * 4});
  }
  check(mssa_adapter_project(&desc, x, w, bias, static_cast<int32_t*>(seg), static_cast<int32_t*>(which), a, b, nullptr, ws, bytes, y,
                             nullptr) == MSSA_OK, g_error.c_str());
}

}  // namespace

int main(int argc, char** argv) {
  g_plant = argc > 1 && !std::strcmp(argv[1], "plant");
  g_odd = argc > 1 && !std::strcmp(argv[1], "odd");
  // quotients, at the numbers where they change and at the ends
  for (int i = 0; i < 4000; ++i) {
    const uint32_t d = static_cast<uint32_t>(i < 200 ? i + 1 : pick(1, i < 2000 ? 1 << 20 : 0x7fffffff));
    const mssa::Divisor div = mssa::Divisor::of(d);
    g_case = "divisor " + std::to_string(d);
    for (int64_t q : {int64_t{0}, int64_t{1}, pick(0, 0x7fffffff / d), int64_t{0x7fffffff / d}})
      for (int64_t n : {q * d - 1, q * d, q * d + 1, q * d + d - 1, int64_t{0x7fffffff}})
        if (n >= 0 && n <= 0x7fffffff) check(div.quotient(static_cast<uint32_t>(n)) == static_cast<uint32_t>(n) / d, "quotient");
  }
  for (int i = 0; i < 500; ++i) {
    const int batch = static_cast<int>(pick(0, 3) ? pick(1, 6) : pick(1, 90)), kv = static_cast<int>(pick(1, 4));
    const int64_t tokens = pick(0, 2) ? pick(0, 40) : pick(0, 3000);
    const int page = static_cast<int>(pick(1, 100)), table = static_cast<int>(pick(1, 60));
    const int mask = pick(0, 1) ? 0 : pick(0, 1) ? 1 : static_cast<int>(pick(1, pick(0, 1) ? 700 : 0x7fffffff));
    attend(tokens, batch, static_cast<int>(pick(0, 1) ? std::max<int64_t>(1, tokens) : pick(1, 3000)), kv * static_cast<int>(pick(1, 5)), kv,
           pick(0, 1) ? 64 : 128, page, table, mask, page * table + 5);
  }
  attend(9360, 1, 9360, 12, 12, 128, 1560, 24, 1560, 37440);
  attend(23400, 3, 9360, 12, 12, 128, 256, 128, 1560, 32760);
  attend(2048, 2048, 1, 8, 8, 128, 16, 60, 1, 900);
  for (int i = 0; i < 300; ++i) {
    const int d = 16 * static_cast<int>(pick(1, 16)), halves = static_cast<int>(pick(0, 1));
    append(pick(1, 3000), static_cast<int>(pick(1, 100)), static_cast<int>(pick(0, 12)), static_cast<int>(pick(1, 12)), d,
           static_cast<int>(pick(1, 300)), halves ? 16 * static_cast<int>(pick(0, d / 16)) : 2 * static_cast<int>(pick(0, d / 2)), halves);
  }
  if (!g_odd) append((int64_t{1} << 30), 3, 1, 1, 16, 16, 16, 0);  // made in slices
  for (int i = 0; i < 400; ++i) {
    const int parts = static_cast<int>(pick(1, 4)), k = static_cast<int>(pick(0, 1) ? 8 * pick(1, 700) : pick(1, 3000));
    project(pick(0, 2) ? pick(1, 200) : pick(1, 30000), k, parts * static_cast<int>(pick(1, 3000)), parts, static_cast<int>(pick(0, 50)),
            static_cast<int>(pick(0, 9)), static_cast<int>(pick(1, 256)), static_cast<int>(pick(0, 1) ? 0 : pick(1, 20)));
  }
  project(64, 1 << 20, 64, 1, 1, 1, 8, 0);
  for (int k = 1; k < 10; ++k)
    for (int rows : {1, 17, 64, 65}) project(rows, k, 100, 2, 3, 2, 12, k % 3);
  project(300, 64, 512, 1, 2, 1, 8, (1 << 21) - 64);
  project(300, 64, 512, 1, 2, 1, 8, 1 << 25);
  // no launch of 2^32 threads
  g_walk = false;
  mssa_paged_attention_desc big{int64_t{1} << 30, 1 << 20, 1 << 20, 64, 64, 128, 1 << 10, 1 << 20, 1, 0, 0, 0, 0.f};
  int64_t bytes = 0;
  check(mssa_paged_attention_workspace_size(&big, &bytes) == MSSA_ERR_UNSUPPORTED, "too many items are refused");
  std::printf("%d checks, %d launches, %d failures\n", g_checks, g_launches, g_failures);
  return g_failures ? 1 : 0;
}
