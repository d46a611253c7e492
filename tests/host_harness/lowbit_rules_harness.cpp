// Host harness of the low-bit kernels' rules on sizes, built without any GPU
// code (under AddressSanitizer and UndefinedBehaviorSanitizer by
// tests/test_lowbit_rules.py).  The harness walks each rule the way its kernel
// does and checks what the kernel relies on.  Exit status 0 iff every check
// passed.
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstring>
#include <string>
#include <vector>

#include "../../paper_2607_20940_amd/csrc/lowbit_args.hpp"

namespace {

int g_failures = 0, g_checks = 0;

void check(bool ok, const std::string& what) {
  ++g_checks;
  if (!ok && ++g_failures <= 40) std::fprintf(stderr, "FAIL %s\n", what.c_str());
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

int main() {
  scale_groups<8, 2>();  // MXFP4 tokens
  scale_groups<4, 1>();  // 8-bit tokens
  std::printf("%d checks, %d failures\n", g_checks, g_failures);
  return g_failures ? 1 : 0;
}
