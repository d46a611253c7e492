// Rotation of a packed batch's queries and keys, and storing of its keys and
// values in the pages of their sequences (mssa_paged_append).
//
// A block takes one token, or a few of narrow ones: its waves look up the
// tokens' places, its threads turn positions into cosines and sines (once for
// all heads, in LDS), then take pieces of 16 values of a head: two 16-byte
// chunks, those whose values are pairs where halves are paired.  The angle is
// taken in turns, position * freq / 2 pi in 64 bits, and its fraction alone
// goes to 32 bits: a position of 2^31 leaves an angle as exact as one of 1.
//
// Bound by HBM: every value is read once and written once.  A thread takes
// four pieces at most, so a block has all its loads on their way at once;
// narrow tokens share a block so that its look-ups and sines, which no load of a
// value waits for but every store does, are not its whole time.  35100 tokens of
// 40 + 2 x 40 heads, 2.2 GB: 400 us, 5.4 TB/s (a large copy reaches 5.2); 4680 tokens of
// 12 + 2 x 12 heads: 19 us, 4.5 TB/s; one token: 4.4 us on the device, a launch and
// three dependent loads.
#include <hip/hip_runtime.h>

#include "paged_args.hpp"

namespace mssa {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr double kTurn = 0.15915494309189533577;  // 1 / 2 pi

// What of a token a block's threads share.  slot: its token in the pool, or -1
// (stored nowhere); index: its cache index; there: it belongs to a sequence.
struct Token {
  int32_t slot, index;
  bool there;
};

// The token's sequence is the last b with begin[b] <= row < begin[b + 1]: the
// wave probes 64 places at a time.
__device__ inline Token find(const AppendArgs& a, int32_t row) {
  const int lane = threadIdx.x & 63;
  int32_t b;
  ChunkRows c;
  if (!a.chunk_begin) {
    b = row / a.each;
    c = ChunkRows::of(nullptr, b, a.each, a.tokens);
  } else {
    int32_t lo = 0, n = a.batch;  // the sequence is one of lo .. lo + n - 1, if there is one
    while (n > 64) {
      const int32_t step = (n + 63) / 64, at = lo + lane * step;
      // sequences that begin behind the row cannot hold it: what is kept starts at the last probe that does not
      const uint64_t ahead = __ballot(lane * step < n && a.chunk_begin[at < a.batch ? at : a.batch] <= row);
      const int last = ahead ? 63 - __builtin_clzll(ahead) : 0;
      n = n - last * step < step ? n - last * step : step;
      lo += last * step;
    }
    const bool mine = lane < n && a.chunk_begin[lo + lane] <= row && row < a.chunk_begin[lo + lane + 1];
    const uint64_t hit = __ballot(mine);
    if (!hit) return {-1, 0, false};
    b = lo + 63 - __builtin_clzll(hit);
    c = ChunkRows::of(a.chunk_begin, b, a.each, a.tokens);
  }
  const int64_t index = static_cast<int64_t>(a.kv_len[b]) - (c.end - row);
  int32_t slot = -1;
  if (index >= 0 && index < static_cast<int64_t>(a.table_pages) * a.page.d) {
    const uint32_t entry = a.page.quotient(static_cast<uint32_t>(index));
    const int32_t page = a.page_table[static_cast<int64_t>(b) * a.table_pages + entry];
    if (page >= 0 && page < a.pages) slot = page * static_cast<int32_t>(a.page.d) + static_cast<int32_t>(index - entry * a.page.d);
  }
  return {slot, static_cast<int32_t>(index), true};
}

__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a) {
  __shared__ float2 turn[kAppendMaxTokens * kAppendMaxPairs];  // cos, sin of a token's pairs
  __shared__ int32_t slots[kAppendMaxTokens], indices[kAppendMaxTokens];
  const int tid = threadIdx.x, wave = tid >> 6;
  const int32_t first = a.token0 + static_cast<int32_t>(blockIdx.x) * a.block_tokens;
  const int32_t n = min(a.block_tokens, a.token1 - first);
  for (int t = wave; t < n; t += kAppendThreads / 64) {
    const Token at = find(a, first + t);
    if ((tid & 63) == 0) {
      slots[t] = at.there ? at.slot : -2;
      indices[t] = at.index;
    }
  }
  __syncthreads();
  for (int i = tid; i < n * a.pairs; i += kAppendThreads) {
    const int t = i / a.pairs, p = i - t * a.pairs;
    const int axis = p < a.axis_end[0] ? 0 : p < a.axis_end[1] ? 1 : 2;
    const int32_t at = a.positions ? a.positions[static_cast<int64_t>(axis) * a.tokens + first + t] : indices[t];
    const double turns = static_cast<double>(at) * static_cast<double>(a.freqs[p]) * kTurn;
    float s, c;
    sincospif(2.f * static_cast<float>(turns - rint(turns)), &s, &c);
    turn[t * a.pairs + p] = make_float2(c, s);
  }
  __syncthreads();
  const int hu = a.head_dim / 16, half = a.pairs / 8;  // pieces of a head; chunks of a half
  const int total = n * static_cast<int>(a.units.d);
  for (int i = tid; i < total; i += kAppendThreads) {
    const int t = static_cast<int>(a.units.quotient(i)), u = i - t * static_cast<int>(a.units.d);
    if (slots[t] == -2) continue;
    const int h = static_cast<int>(a.head_units.quotient(u)), piece = u - h * hu;
    const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.kv_heads;
    const int kh = is_q ? h : is_v ? h - a.q_heads - a.kv_heads : h - a.q_heads;
    if (!is_q && slots[t] < 0) continue;
    // chunks of 8 values: c0 and c1 hold pairs of each other where halves are paired
    int c0 = piece, c1 = piece + hu;
    if (a.halves) {
      if (piece < half) {
        c1 = piece + half;
      } else {
        c0 = piece + half;
        c1 = piece + hu;
      }
    }
    const int64_t row = first + t;
    const __bf16* src = (is_q ? static_cast<const __bf16*>(a.q) + row * a.q_stride
                              : is_v ? static_cast<const __bf16*>(a.v) + row * a.v_stride
                                     : static_cast<const __bf16*>(a.k) + row * a.k_stride) +
                        static_cast<int64_t>(kh) * a.head_dim;
    __bf16* dst = is_q ? static_cast<__bf16*>(a.q_out) + (row * a.q_heads + kh) * a.head_dim
                       : static_cast<__bf16*>(is_v ? a.v_pages : a.k_pages) +
                             (static_cast<int64_t>(slots[t]) * a.kv_heads + kh) * a.head_dim;
    bf16x8 x = *reinterpret_cast<const bf16x8*>(src + c0 * 8), y = *reinterpret_cast<const bf16x8*>(src + c1 * 8);
    if (!is_v) {
      const float2* w = turn + t * a.pairs;
      if (a.halves) {
        if (piece < half) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 cs = w[piece * 8 + e];
            const float p = static_cast<float>(x[e]), q = static_cast<float>(y[e]);
            x[e] = static_cast<__bf16>(p * cs.x - q * cs.y);
            y[e] = static_cast<__bf16>(p * cs.y + q * cs.x);
          }
        }
      } else {
        auto pairs_of = [&](bf16x8& z, int c) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (c * 4 + e >= a.pairs) break;
            const float2 cs = w[c * 4 + e];
            const float p = static_cast<float>(z[2 * e]), q = static_cast<float>(z[2 * e + 1]);
            z[2 * e] = static_cast<__bf16>(p * cs.x - q * cs.y);
            z[2 * e + 1] = static_cast<__bf16>(p * cs.y + q * cs.x);
          }
        };
        pairs_of(x, c0);
        pairs_of(y, c1);
      }
    }
    *reinterpret_cast<bf16x8*>(dst + c0 * 8) = x;
    *reinterpret_cast<bf16x8*>(dst + c1 * 8) = y;
  }
}

}  // namespace

hipError_t launch_paged_append(const AppendArgs& a, hipStream_t stream) {
  const int32_t n = a.token1 - a.token0;
  hipLaunchKernelGGL(append_kernel, dim3(static_cast<uint32_t>((n + a.block_tokens - 1) / a.block_tokens)),
                     dim3(kAppendThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace mssa
