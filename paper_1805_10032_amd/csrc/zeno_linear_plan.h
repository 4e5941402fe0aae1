// How the log probabilities of a linear layer and their gradients are cut: pieces of the vocabulary, blocks and parts of the tokens, tiles, and what stands where
// in the workspace.  Plain host code, which can be checked without a GPU.
#ifndef ZENO_LINEAR_PLAN_H_
#define ZENO_LINEAR_PLAN_H_

#include <algorithm>
#include <cstddef>
#include "zeno.h"

namespace zeno {

constexpr int kWideSide = 256, kTileSide = 128;   // of the tiles; a tile of logits is two slices of the vocabulary
constexpr int kFewSlice = 32;

inline long long tiles_along(long long n, long long side) { return (n + side - 1) / side; }
inline int padded_width(int width) { return (width + 7) / 8 * 8; }
inline int planes_of(int dtype) { return dtype == ZENO_F32 ? 3 : 1; }                             // of an operand
inline int dz_planes_of(int dtype) { return dtype == ZENO_F32 ? 3 : (dtype == ZENO_F16 ? 2 : 4); }

constexpr long long kPackElements = 64LL << 20;    // of W that are packed at a time, a plane
// Tokens whose slices are kept at a time, and how many sums that may be (twelve bytes each): vocabularies beyond 2^18 values take fewer tokens, so that their sums stay
// below 1.7 GB (2^24 values of 65536 tokens would be 103) and their tiles, 2^18 of them, in a dimension of a launch, which ends at 2^32 threads.
constexpr int kRowBlock = 1 << 16;
constexpr long long kSliceSums = 1LL << 27;

// Wide tiles of weight gradients: from so many tokens a worker on.  Shorter sums leave the tile's first loads and its 256 KB of stores, which only
// another workgroup of the compute unit can run beside (20 x 100 tokens, 32000 x 1024: 646 us in 128 x 128 tiles, 794 in wide ones; logits and weight gradients
// of 600 tokens, 50257 x 1600: 457 and 491, 4 x 600, 32000 x 1024: 732 and 768, 4 x 1000: 1086 and 1068, 4 x 2048, 8192 x 4096: 1623 and 1606).
constexpr int kLongGroup = 1024;
// Wide tiles where they give most compute units one (250 tokens, 50257 x 1600, 197 tiles: 63 us, 128 x 128 tiles 75; 2000 tokens, 32000 x 1024: 186 and 211).
inline bool enough_wide_tiles(long long m, long long n) { return tiles_along(m, kWideSide) * tiles_along(n, kWideSide) >= 192; }

struct PlanLayout {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  }
};

// Few tokens: 16-bit operands are as fast in tiles of 128 tokens from 65 on (32000 x 4096: 64 tokens 74 us, 65 in tiles 69); float32,
// which tiles take in six products, from 257 on (1024 columns: 256 tokens 209 us, 250 in tiles 211; 4096 columns 832 and 939).
constexpr int kFewRows = 64, kFewRowsF32 = 256;
inline bool few_tokens(int rows, int dtype) { return rows <= (dtype == ZENO_F32 ? kFewRowsF32 : kFewRows); }

// Of so many rows of W, multiples of 256.
inline int packed_at_a_time(long long values, long long padded) {
  return (int)std::min<long long>(tiles_along(values, 256) * 256, std::max<long long>(256, kPackElements / padded / 256 * 256));
}

struct ForwardPlan {
  bool few, wide;
  int slice;          // values of the vocabulary in a slice
  int piece;          // values that are packed at a time
  int block;          // tokens at a time
  size_t hidden, weight, part, part_u, label, bytes;
};
inline ForwardPlan forward_plan(int rows, int vocab, int width, int dtype) {
  ForwardPlan p;
  p.few = few_tokens(rows, dtype);
  p.block = std::min(rows, kRowBlock);
  if (!p.few) p.block = (int)std::min<long long>(p.block, kSliceSums / (tiles_along(vocab, kWideSide / 2) + 4) / 256 * 256);   // (tiles are wide where this is less)
  p.wide = enough_wide_tiles(vocab, p.block);
  p.slice = p.few ? kFewSlice : (p.wide ? kWideSide : kTileSide) / 2;
  const long long padded = padded_width(width);
  p.piece = packed_at_a_time(vocab, padded);
  PlanLayout l;
  p.hidden = l.take(p.few ? 0 : (size_t)planes_of(dtype) * p.block * padded * 2);
  p.weight = l.take(p.few ? 0 : (size_t)planes_of(dtype) * std::min(p.piece, vocab) * padded * 2);
  const size_t slices = (size_t)tiles_along(vocab, p.slice) + 4;
  p.part = l.take(slices * p.block * 8);
  p.part_u = l.take(slices * p.block * 4);
  p.label = l.take((size_t)p.block * 4);
  p.bytes = l.at + 256;
  return p;
}

struct BackwardPlan {
  bool few, wide_logits, wide_hidden, wide_weight;
  int piece;          // values of the vocabulary at a time
  int pack;           // values that are packed at a time
  int planes;         // of dz
  int splits, parts;
  size_t hidden, weight, dz, slots, sums, power, up, half, columns, bytes;
};
inline BackwardPlan backward_plan(int rows, int vocab, int width, int dtype, int m) {
  BackwardPlan p;
  const long long padded = padded_width(width), n = std::max(rows, 1);
  p.planes = dz_planes_of(dtype);
  // 64 M values of dz at a time: its planes stay near the caches, and a piece still has a thousand tiles.  Of more than 32768 tokens 2048 values each, or every piece's
  // sums for the hidden states would cost more than its products: dz grows with the tokens then (2^20 tokens in bf16: 17 GB).
  const long long most = std::max<long long>(2048, ((64LL << 20) / n) / 256 * 256);
  const long long pieces = (vocab + most - 1) / most;
  p.piece = (int)(((vocab + pieces - 1) / pieces + 255) / 256 * 256);
  p.pack = packed_at_a_time(p.piece, padded);
  p.few = few_tokens(rows, dtype);
  p.wide_logits = enough_wide_tiles(p.piece, n);
  p.wide_hidden = enough_wide_tiles(n, width);
  p.wide_weight = enough_wide_tiles((long long)p.piece * m, width) && n / m >= kLongGroup;
  const int side = p.wide_hidden ? kWideSide : kTileSide;
  const long long tiles = tiles_along(n, side) * tiles_along(width, side);
  p.splits = (int)std::max<long long>(1, std::min<long long>(p.piece / 512, (p.wide_hidden ? 256 : 512) / tiles));
  // Weight gradients of few tiles: a group's tokens in parts, from twice 512 on (logits and weight gradients of 14141 tokens, 11 x 19 bf16: 64 us, in one part
  // 290; 16384, 1000 x 512 bf16 146 and 363, float32 308 and 1655; 1024, 11 x 19 54 and 60).
  const long long weights = tiles_along(p.piece, kTileSide) * tiles_along(width, kTileSide) * m;
  p.parts = (int)std::max<long long>(1, std::min<long long>(n / m / 512, 512 / weights));
  PlanLayout l;
  p.hidden = l.take((size_t)planes_of(dtype) * n * padded * 2);
  p.weight = l.take((size_t)planes_of(dtype) * p.pack * padded * 2);
  p.dz = l.take((size_t)p.planes * n * p.piece * 2);
  p.slots = l.take((size_t)p.splits * n * width * 4);
  p.sums = l.take(p.parts > 1 ? (size_t)p.parts * m * std::min(p.piece, vocab) * (width + 1LL) * 4 : 0);
  p.power = l.take((size_t)m * 4);
  p.up = l.take((size_t)n * 4);
  p.half = l.take(dtype == ZENO_BF16 ? (size_t)n * padded * 2 : 0);
  p.columns = l.take(dtype == ZENO_BF16 ? (size_t)m * width * 4 : 0);
  p.bytes = l.at + 256;
  return p;
}

}  // namespace zeno
#endif
