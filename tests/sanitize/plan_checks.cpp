// How the log probabilities of a linear layer are cut: which kernels the tests' sizes take, and the limits that launches and offsets have, over the documented
// sizes.  Built and run by tests/test_token_ends_plans.py.
#include <cstdio>

#include "zeno_linear_plan.h"

#define CHECK(cond)                                                                                                     \
  do {                                                                                                                  \
    if (!(cond)) {                                                                                                      \
      std::fprintf(stderr, "check failed at line %d: %s (%d x %d x %d, type %d, m %d)\n", __LINE__, #cond, rows, vocab, width, dtype, m); \
      return 1;                                                                                                         \
    }                                                                                                                   \
  } while (0)

using namespace zeno;

constexpr long long kMostBlocks = (1LL << 24) - 1;   // of 256 threads, in a dimension

int main() {
  int rows = 0, vocab = 0, width = 0, dtype = 0, m = 1;
  for (dtype = 0; dtype < 3; ++dtype) {
    // the sizes of tests/test_gpu_linear_logprobs_wide.py
    rows = 2100, vocab = 12600, width = 1000, m = 2;
    CHECK(backward_plan(rows, vocab, width, dtype, m).wide_weight && backward_plan(rows, vocab, width, dtype, m).wide_logits);
    rows = 2101, vocab = 25090, width = 1024, m = 1;
    CHECK(backward_plan(rows, vocab, width, dtype, m).wide_weight);
    rows = 8200, vocab = 8500, width = 1544, m = 2;
    const BackwardPlan two = backward_plan(rows, vocab, width, dtype, m);
    CHECK(two.wide_weight && two.wide_hidden && two.wide_logits && two.piece < vocab);
    // tests/test_gpu_linear_logprobs_corners.py
    rows = 70, vocab = 10000, width = 8191, m = 1;
    CHECK(backward_plan(rows, vocab, width, dtype, m).pack < backward_plan(rows, vocab, width, dtype, m).piece);
    rows = 2000, vocab = 6400, width = 512, m = 4;
    CHECK(!backward_plan(rows, vocab, width, dtype, m).wide_weight);
  }
  const int many[] = {1, 64, 65, 256, 257, 1000, 40000, 65281, 65536, 300000, ZENO_MAX_TOKENS};
  const int values[] = {1, 31, 257, 50257, 1 << 18, (1 << 18) + 1, 1 << 21, ZENO_MAX_OUTPUTS - 255, ZENO_MAX_OUTPUTS};
  const int widths[] = {1, 8, 1001, 4096, ZENO_MAX_HIDDEN};
  for (int r : many)
    for (int v : values)
      for (int w : widths)
        for (dtype = 0; dtype < 3; ++dtype)
          for (m = 1; m <= ZENO_MAX_CANDIDATES; m *= 32) {
            rows = r, vocab = v, width = w;
            if ((long long)vocab * width > 1LL << 36) continue;
            const ForwardPlan f = forward_plan(rows, vocab, width, dtype);
            CHECK(f.block >= 1 && f.block <= rows && f.piece % 256 == 0);
            if (f.few) {
              CHECK(f.block == rows);
            } else {
              // weights that are read as they stand are one launch
              const int side = f.wide ? kWideSide : kTileSide;
              CHECK(tiles_along(vocab, side) * tiles_along(f.block, side) <= kMostBlocks);
              CHECK(tiles_along(vocab, f.slice) * f.block <= kSliceSums);
            }
            const BackwardPlan b = backward_plan(rows, vocab, width, dtype, m);
            CHECK(b.piece % 256 == 0 && b.splits >= 1 && b.parts >= 1);
            CHECK(b.pack % 256 == 0 && b.pack <= b.piece && (b.pack == 256 || (long long)b.pack * padded_width(width) <= kPackElements));
            const int s = b.wide_logits ? kWideSide : kTileSide, t = b.wide_weight ? kWideSide : kTileSide;
            CHECK(tiles_along(b.piece, s) * tiles_along(rows, s) <= kMostBlocks);
            CHECK(tiles_along(b.piece, t) * tiles_along(width, t) <= kMostBlocks);
            // a tile's offsets in dz are counted in 32 bits: its rows, or a stage of 32 of the contraction
            const long long high = rows < kWideSide ? rows : kWideSide;
            CHECK(2 * ((high - 1) * b.piece + 32) < 1LL << 32 && 2 * (32LL * b.piece + b.piece) < 1LL << 32);
          }
  std::puts("plan checks passed");
  return 0;
}
