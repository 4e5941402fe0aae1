// Weight gradients of a linear layer from 8-bit activations, per group of rows (a worker's tokens):
//   dW_g[o][k] = sum_{t in g} dy[t][o] a[t][k],   db_g[o] = sum_{t in g} dy[t][o].
//
// A matrix product over tokens on the bf16 matrix cores.  An e4m3 value times its power-of-two scale has four significant bits: it is
// exact in bf16.  dy goes in as bf16 pieces: one for bf16, two for fp16 (11 bits), three for float32 (24 bits), so every product is
// exact and the only rounding is that of the float32 sums.
// Both operands have the tokens as their slow axis, and a lane of the matrix instruction wants eight tokens of one column: tiles
// stay as they are in LDS and the transposing LDS read turns four tokens x sixteen columns at a time.
#include "zeno_tokens.h"
#include <algorithm>
#include <type_traits>

namespace zeno {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 32;   // pieces of a group's tokens are multiples of it

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A workgroup of four waves: WO of them along the outputs, 4 / WO along the inputs; a wave takes 32 FO x 32 FI of the product.
// dy goes in as P pieces; a stage is KT tokens.
// ODD: the outputs are not a multiple of eight.
template <int WO_, int FO_, int FI_, int P_, bool ODD_>
struct Tile {
  static constexpr bool ODD = ODD_;
  static constexpr int WO = WO_, FO = FO_, FI = FI_, P = P_, KT = P == 1 ? 32 : 16;
  static constexpr int OUT = 32 * FO * WO, IN = 32 * FI * (4 / WO);
  // bf16 of an LDS row, 64 bytes behind a multiple of 256: the four rows of a transposing read lie on different banks (writes are not free of conflicts)
  static constexpr int PITCH_O = OUT + 32, PITCH_I = IN + 32;
  // what a thread fetches of a stage: 8 outputs of CO tokens, 16 inputs of CI
  static constexpr int CHUNKS_O = OUT / 8 * KT, CHUNKS_I = IN / 16 * KT;
  static constexpr int CO = (CHUNKS_O + kThreads - 1) / kThreads, CI = (CHUNKS_I + kThreads - 1) / kThreads;
};
// 256 x 256, or 128 x 256 with several pieces of dy: half the sums, so that two workgroups share a compute unit and one's first loads and
// stores run beside the other's products (20 x 100 tokens, 2048 x 2048: float32 129 -> 113 us, fp16 107 -> 98, with events around each
// launch; 4 x 4096 tokens 377 -> 360 and 254 -> 247).  In bf16 the narrower tile spills and is slower (8 x 2048 tokens, 4096 x 4096: 660 -> 705 us).
template <int P, bool ODD = false> using WideTile = Tile<2, (P > 1 ? 2 : 4), 4, P, ODD>;
template <int P, bool ODD = false> using MidTile = Tile<2, 2, 2, P, ODD>;    // 128 x 128

struct Span {
  int begin, end;
};
__device__ inline Span piece_of(const WeightGradArgs& a, int g, int piece, int pieces) {
  const int b = group_offset(a.offsets, g, a.rows), e = group_offset(a.offsets, g + 1, a.rows);
  const int n = e > b ? e - b : 0;
  const int len = (int)(((n + pieces - 1LL) / pieces + kTokens - 1) / kTokens * kTokens);
  const long long lo = b + (long long)len * piece, hi = lo + len;
  Span s;
  s.begin = (int)(lo < b + n ? lo : b + n);
  s.end = (int)(hi < b + n ? hi : b + n);
  return s;
}

// Eight values as sums of P bf16 pieces, each the leading eight bits of what the pieces before it leave: two take fp16's 11 bits and three
// float32's 24, nothing is rounded, and no finite value becomes infinite.
template <int P>
__device__ inline void split(const float (&v)[8], uint4 (&piece)[P]) {
  float rest[8], largest = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    rest[j] = v[j];
    largest = fmaxf(largest, fabsf(v[j]));
  }
  const bool finite = largest < __builtin_inff();   // (a NaN hides from it and stays one: what it leaves is NaN)
#pragma unroll
  for (int p = 0; p < P; ++p) {
    unsigned bits[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) bits[j] = __float_as_uint(rest[j]);
    // the upper halves of two words
    piece[p] = make_uint4(__builtin_amdgcn_perm(bits[1], bits[0], 0x07060302), __builtin_amdgcn_perm(bits[3], bits[2], 0x07060302),
                          __builtin_amdgcn_perm(bits[5], bits[4], 0x07060302), __builtin_amdgcn_perm(bits[7], bits[6], 0x07060302));
    if (p + 1 < P) {
#pragma unroll
      for (int j = 0; j < 8; ++j) rest[j] -= __uint_as_float(bits[j] & 0xffff0000u);
      if (!finite) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (fabsf(v[j]) == __builtin_inff()) rest[j] = 0.f;   // (infinity less itself is NaN)
      }
    }
  }
}

// One operand of a matrix instruction: 32 columns from `col` on of 16 tokens, lane l column l % 32, tokens 8 (l / 32) + 0..7.
template <int PITCH>
__device__ inline bf16x8 read_columns(const __bf16* tile, int col, int token, int lane) {
  const int at = (token + 8 * (lane / 32) + (lane % 16) / 4) * PITCH + col + 16 * ((lane / 16) % 2) + 4 * (lane % 4);
  typedef __attribute__((address_space(3))) s16x4* lds;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(tile + at));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(tile + at + 4 * PITCH));
  const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, both);
}

template <typename T, typename S>
struct Fetched {
  typename Wide<T>::type dy[S::CO][8 / Wide<T>::N];
  uint4 a[S::CI];
  uint8_t scale[S::CI];
};

// Where a thread's part of a stage lies: its first token's, a stage further with every fetch.  Columns behind a matrix's last one are
// those before it once more: no load is behind a branch, and no output takes them.  Eight outputs of which only some are left are
// fetched as the row's last eight, and moved down by `shift` on their way to LDS.
template <typename T, typename S>
struct Source {
  const T* dy;
  const uint8_t *values, *scales;
  int shift;
};
template <typename T, typename S>
__device__ inline Source<T, S> source_of(const WeightGradArgs& a, int first, int o0, int k0, int blocks, int tid) {
  constexpr int PO = S::OUT / 8, PI = S::IN / 16;
  Source<T, S> s;
  const int o = o0 + 8 * (tid % PO), k = k0 + 16 * (tid % PI);
  const int from = o + 8 <= a.out ? o : a.out - 8;
  s.shift = o < a.out ? o - from : 0;
  s.dy = reinterpret_cast<const T*>(a.dy) + (long long)(first + tid / PO) * a.lddy + from;
  const int at = k < blocks * kCkptBlock ? k : 0;
  s.values = a.values + (long long)(first + tid / PI) * (blocks * kCkptBlock) + at;
  s.scales = a.scales + (long long)(first + tid / PI) * blocks + at / kCkptBlock;
  return s;
}

// One stage in CO + CI pieces, the last of which moves on by `advance` tokens.  The last stage of a span ends where the span ends and
// begins among tokens that the stage before has had already: deposit_piece() puts zeros in the place of their dy (their activations are
// finite or have made the sums NaN already), and no load needs a test.  WHOLE: the span holds a stage; otherwise the stage begins at
// token `base` < 0, and what lies before the span's first token comes as copies of it.
template <typename T, typename S, bool WHOLE>
__device__ inline void fetch_piece(int piece, const WeightGradArgs& a, Source<T, S>& s, int base, int advance, int blocks, int tid,
                                   Fetched<T, S>& f) {
  constexpr int N = Wide<T>::N, PO = S::OUT / 8, PI = S::IN / 16, RO = kThreads / PO, RI = kThreads / PI;
  if (piece < S::CO) {
    const int h = piece, token = tid / PO + RO * h;
    if (S::CHUNKS_O >= kThreads || tid < S::CHUNKS_O) {
      const T* p = s.dy + (long long)(WHOLE ? RO * h : (base + token > 0 ? base + token : 0) - tid / PO) * a.lddy;
#pragma unroll
      for (int i = 0; i < 8 / N; ++i) f.dy[h][i] = *reinterpret_cast<const typename Wide<T>::unaligned*>(p + i * N);
    }
  } else if (piece < S::CO + S::CI) {
    const int h = piece - S::CO, token = tid / PI + RI * h;
    if (S::CHUNKS_I >= kThreads || tid < S::CHUNKS_I) {
      const long long row = WHOLE ? RI * h : (base + token > 0 ? base + token : 0) - tid / PI;
      f.a[h] = *reinterpret_cast<const uint4*>(s.values + row * (blocks * kCkptBlock));
      f.scale[h] = s.scales[row * blocks];
    }
  }
  if (WHOLE && piece == S::CO + S::CI - 1) {
    s.dy += (long long)advance * a.lddy;
    s.values += (long long)advance * (blocks * kCkptBlock);
    s.scales += (long long)advance * blocks;
  }
}
template <typename T, typename S, bool WHOLE>
__device__ inline void fetch(const WeightGradArgs& a, Source<T, S>& s, int base, int advance, int blocks, int tid, Fetched<T, S>& f) {
#pragma unroll
  for (int piece = 0; piece < S::CO + S::CI; ++piece) fetch_piece<T, S, WHOLE>(piece, a, s, base, advance, blocks, tid, f);
}

__device__ inline bf16x8 widen8(unsigned x, unsigned y, float s) {
  const bf16x2 q0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, false), q1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, true);
  const bf16x2 q2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, s, false), q3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, s, true);
  return bf16x8{q0.x, q0.y, q1.x, q1.y, q2.x, q2.y, q3.x, q3.y};
}

template <typename S>
struct Stage {
  __bf16 y[S::P][S::KT * S::PITCH_O];
  __bf16 a[S::KT * S::PITCH_I];
};

// Piece h < CO: eight outputs' dy of one token into LDS as bf16, and into the sums of the bias where the workgroup has these to take;
// piece CO + h: sixteen activations.  The stage's first `skip` tokens do not count.
template <typename T, typename S, bool WHOLE>
__device__ inline void deposit_piece(int piece, const Fetched<T, S>& f, Stage<S>& st, int skip, int shift, int tid, bool sums,
                                     float (&bias)[8]) {
  constexpr int N = Wide<T>::N, P = S::P;
  if (piece < S::CO) {
    if (S::CHUNKS_O < kThreads && tid >= S::CHUNKS_O) return;
    constexpr int PER = S::OUT / 8;
    const int h = piece, token = tid / PER + kThreads / PER * h;
    const bool live = WHOLE || token >= skip;
    uint4 plane[P];
    if constexpr (P == 1) {
      static_assert(P > 1 || sizeof(T) == 2, "one piece is dy itself");
      uint4 raw = __builtin_bit_cast(uint4, f.dy[h][0]);
      if (S::ODD && shift != 0) {
        if (shift & 4) raw = make_uint4(raw.z, raw.w, raw.w, raw.w);
        if (shift & 2) raw = make_uint4(raw.y, raw.z, raw.w, raw.w);
        if (shift & 1)
          raw = make_uint4(__builtin_amdgcn_alignbit(raw.y, raw.x, 16), __builtin_amdgcn_alignbit(raw.z, raw.y, 16),
                           __builtin_amdgcn_alignbit(raw.w, raw.z, 16), raw.w >> 16);
      }
      plane[0] = make_uint4(live ? raw.x : 0, live ? raw.y : 0, live ? raw.z : 0, live ? raw.w : 0);
      if (sums) {
        const bf16x8 v = __builtin_bit_cast(bf16x8, plane[0]);
#pragma unroll
        for (int j = 0; j < 8; ++j) bias[j] += (float)v[j];
      }
    } else {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = (float)f.dy[h][j / N][j % N];
      if (S::ODD && shift != 0) {
#pragma unroll
        for (int by = 4; by > 0; by /= 2)
          if (shift & by) {
#pragma unroll
            for (int j = 0; j + by < 8; ++j) v[j] = v[j + by];
          }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!live) v[j] = 0.f;
        if (sums) bias[j] += v[j];
      }
      split<P>(v, plane);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) *reinterpret_cast<uint4*>(&st.y[i][token * S::PITCH_O + 8 * (tid % PER)]) = plane[i];
  } else if (piece < S::CO + S::CI) {
    if (S::CHUNKS_I < kThreads && tid >= S::CHUNKS_I) return;
    constexpr int PER = S::IN / 16;
    const int h = piece - S::CO;
    const float s = ckpt_scale((int)f.scale[h] - 127);
    __bf16* to = &st.a[(tid / PER + kThreads / PER * h) * S::PITCH_I + 16 * (tid % PER)];
    *reinterpret_cast<bf16x8*>(to) = widen8(f.a[h].x, f.a[h].y, s);
    *reinterpret_cast<bf16x8*>(to + 8) = widen8(f.a[h].z, f.a[h].w, s);
  }
}
template <typename T, typename S>
__device__ inline void deposit(const Fetched<T, S>& f, Stage<S>& st, int skip, int shift, int tid, bool sums, float (&bias)[8]) {
#pragma unroll
  for (int piece = 0; piece < S::CO + S::CI; ++piece) deposit_piece<T, S, false>(piece, f, st, skip, shift, tid, sums, bias);
}

// The operands of 16 tokens.
template <typename S>
struct Operands {
  bf16x8 x[S::FI], y[S::P][S::FO];
};
template <typename S>
__device__ inline void read_operand(int which, const Stage<S>& st, int t, int wo, int wk, int lane, Operands<S>& f) {
  if (which < S::FI) {
    f.x[which] = read_columns<S::PITCH_I>(st.a, wk + 32 * which, t, lane);
  } else {
    const int r = (which - S::FI) / S::P, p = (which - S::FI) % S::P;
    f.y[p][r] = read_columns<S::PITCH_O>(st.y[p], wo + 32 * r, t, lane);
  }
}
template <typename S>
__device__ inline void read_operands(const Stage<S>& st, int t, int wo, int wk, int lane, Operands<S>& f) {
#pragma unroll
  for (int i = 0; i < S::FI + S::FO * S::P; ++i) read_operand<S>(i, st, t, wo, wk, lane, f);
}
// between(i) stands behind the i-th matrix instruction and stays there
template <typename S, typename F>
__device__ inline void multiply(const Operands<S>& f, f32x16 (&acc)[S::FO][S::FI], F between) {
  int i = 0;
#pragma unroll
  for (int r = 0; r < S::FO; ++r)
#pragma unroll
    for (int p = S::P - 1; p >= 0; --p)   // the smallest piece first
#pragma unroll
      for (int j = 0; j < S::FI; ++j) {
        acc[r][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.y[p][r], f.x[j], acc[r][j], 0, 0, 0);
        between(i++);
      }
}
template <typename S>
__device__ inline void multiply(const Operands<S>& f, f32x16 (&acc)[S::FO][S::FI]) {
  multiply<S>(f, acc, [](int) {});
}

// Several pieces: a stage has P times the matrix instructions, and holding all its operands twice would take more registers than there
// are.  The inputs' operands are held for this stage and the next, the outputs' RN - 1 ahead in a ring of RN.
template <typename S, int RN>
__device__ inline void read_ring(int q, const Stage<S>& st, int wo, int lane, bf16x8 (&y)[RN], int slot) {
  y[slot] = read_columns<S::PITCH_O>(st.y[S::P - 1 - q % S::P], wo + 32 * (q / S::P), 0, lane);   // the smallest piece first
}

// Three stages in LDS: one that is multiplied, one that is whole, from which the first operands behind the barrier have been read
// before it, and one that is being written; two more are on their way from memory.
// Tiles: a wave's 128 x 128 of the product reads the fewest operands from LDS that the registers allow, at one wave a SIMD, which issues in
// order: what runs beside the matrix instructions stands between them.
// 8 x 2048 tokens, 4096 x 4096, bf16: 550-605 us (910-1000 TFLOP/s; a large bf16 product of the library with its operands stored this way
// 1187, stored the other way 1369).  The matrix pipes are busy for 52 % of the time and the clock gives way under them; waves stand ready but
// unissued for 40 %.  LDS is active for 29 % of the cycles, a fifth of that conflicts.
// 20 x 100 tokens, 2048 x 2048, float32: 86-92 us, 3.9 TB/s of gradients written; a tile has seven stages, and what is left is its first loads and its
// 128 KB of stores where both workgroups of a compute unit are in them.  128 x 128 tiles: 134 us (102 with these before the stores went past
// the caches).
template <typename T, typename S>
__global__ __launch_bounds__(kThreads, S::FO == 4 ? 1 : 2) void weight_grad_kernel(WeightGradArgs a, int tiles_in, int pieces,
                                                                                  float* partial) {
  extern __shared__ __align__(16) unsigned char memory[];
  Stage<S>* stage = reinterpret_cast<Stage<S>*>(memory);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
  const int o0 = (int)(blockIdx.x / tiles_in) * S::OUT, k0 = (int)(blockIdx.x % tiles_in) * S::IN;
  const int g = blockIdx.y / pieces, piece = blockIdx.y % pieces;
  const Span span = piece_of(a, g, piece, pieces);
  const int blocks = ckpt_blocks(a.width);
  const int wo = 32 * S::FO * (wave % S::WO), wk = 32 * S::FI * (wave / S::WO);
  f32x16 acc[S::FO][S::FI] = {};
  float bias[8] = {};
  const int n = span.end - span.begin, stages = (n + S::KT - 1) / S::KT;
  const bool sums = k0 == 0 && a.dbias != nullptr;
  Source<T, S> from = source_of<T, S>(a, span.begin, o0, k0, blocks, tid);
  // where stage s begins, and how many of its tokens the stages before have had (all of them behind the last stage)
  auto base = [&](int s) { return s * S::KT < n - S::KT ? s * S::KT : n - S::KT; };
  auto skip = [&](int s) { return s < stages ? s * S::KT - base(s) : S::KT; };
  if (stages > 0) {
    Fetched<T, S> even = {}, odd = {};
    {
      Fetched<T, S> first = {}, second = {};   // (all four on their way at once)
      if (n >= S::KT) {
        fetch<T, S, true>(a, from, 0, base(1), blocks, tid, first);
        fetch<T, S, true>(a, from, 0, base(2) - base(1), blocks, tid, second);
        fetch<T, S, true>(a, from, 0, base(3) - base(2), blocks, tid, even);
        fetch<T, S, true>(a, from, 0, base(4) - base(3), blocks, tid, odd);
      } else {
        fetch<T, S, false>(a, from, n - S::KT, 0, blocks, tid, first);
      }
      deposit<T, S>(first, stage[0], skip(0), from.shift, tid, sums, bias);
      deposit<T, S>(second, stage[1], skip(1), from.shift, tid, sums, bias);
    }
    __syncthreads();
    constexpr bool RING = S::FI == 4 && S::P > 1;
    constexpr int RN = S::FO * S::P % 4 == 0 ? 4 : 3;
    Operands<S> now, next;
    bf16x8 xa[S::FI], xb[S::FI], ring[RN];
    if constexpr (RING) {
#pragma unroll
      for (int j = 0; j < S::FI; ++j) xa[j] = read_columns<S::PITCH_I>(stage[0].a, wk + 32 * j, 0, lane);
#pragma unroll
      for (int q = 0; q < RN - 1; ++q) read_ring<S, RN>(q, stage[0], wo, lane, ring, q);
    } else {
      read_operands<S>(stage[0], 0, wo, wk, lane, now);
    }
    int at = 0, i = 0;   // at = i % 3
    // One stage; `f` holds the one after next, and takes the second after that.
    auto step = [&](Fetched<T, S>& f, int i, auto with_sums, auto whole) __attribute__((always_inline)) {
      constexpr bool SUMS = decltype(with_sums)::value, WHOLE = decltype(whole)::value;
      const int after = at == 2 ? 0 : at + 1, last = after == 2 ? 0 : after + 1;
      // Reads first, one a step; the conversions and LDS writes spread over the steps behind them; loads last.
      constexpr int STEPS = S::FO * S::FI * S::P, READS = S::FI + S::FO * S::P, PIECES = S::CO + S::CI;
      constexpr bool TWO = S::KT == 32;
      constexpr int FROM = READS < STEPS ? READS : STEPS, ROOM = TWO ? STEPS - FROM : (STEPS - FROM) / 2;
      constexpr int EVERY = ROOM / PIECES > 0 ? ROOM / PIECES : 1, LOADS_FROM = TWO ? (STEPS > PIECES ? STEPS - PIECES : 0) : FROM + EVERY * PIECES;
      const int skipped = skip(i + 2), advance = base(i + 5) - base(i + 4);
      auto pin = [] { __builtin_amdgcn_sched_barrier(0); };
      auto read_next = [&](int i) { read_operand<S>(i, TWO ? stage[at] : stage[after], TWO ? 16 : 0, wo, wk, lane, next); };
      auto read_now = [&](int i) { read_operand<S>(i, stage[after], 0, wo, wk, lane, now); };
      auto write = [&](int piece) { deposit_piece<T, S, WHOLE>(piece, f, stage[last], skipped, from.shift, tid, SUMS, bias); };
      auto load = [&](int piece) { fetch_piece<T, S, true>(piece, a, from, 0, advance, blocks, tid, f); };
      int reads = 0, writes = 0, loads = 0;   // (constants once the steps are unrolled)
      pin();
      multiply<S>(now, acc, [&](int m) {
        if (reads < READS) read_next(reads++);
        if (m >= FROM && (m - FROM) % EVERY == 0 && writes < PIECES) write(writes++);
        if (!TWO && m >= LOADS_FROM && loads < PIECES) load(loads++);
        pin();
      });
#pragma unroll
      for (int i = FROM < READS ? FROM : READS; i < READS; ++i) read_next(i);
#pragma unroll
      for (int i = STEPS > FROM ? (STEPS - FROM + EVERY - 1) / EVERY : 0; i < PIECES; ++i) write(i);
      if (TWO) {
        int again = 0;
        multiply<S>(next, acc, [&](int m) {
          if (again < READS) read_now(again++);
          if (m >= LOADS_FROM && loads < PIECES) load(loads++);
          pin();
        });
#pragma unroll
        for (int i = FROM < READS ? FROM : READS; i < READS; ++i) read_now(i);
      } else {
        now = next;
      }
#pragma unroll
      for (int i = STEPS > LOADS_FROM ? STEPS - LOADS_FROM : 0; i < PIECES; ++i) load(i);
      __syncthreads();
      at = after;
    };
    auto ring_step = [&](Fetched<T, S>& f, int i, bf16x8 (&x)[S::FI], bf16x8 (&x_next)[S::FI], auto whole) __attribute__((always_inline)) {
      constexpr bool WHOLE = decltype(whole)::value;
      constexpr int GROUPS = S::FO * S::P;
      static_assert(!RING || GROUPS % RN == 0, "the ring is where it was at the end of a stage");
      const int after = at == 2 ? 0 : at + 1, last = after == 2 ? 0 : after + 1;
      const int skipped = skip(i + 2), advance = base(i + 5) - base(i + 4);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) {
        const int r = q / S::P;
#pragma unroll
        for (int j = 0; j < S::FI; ++j) acc[r][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[q % RN], x[j], acc[r][j], 0, 0, 0);
        if (q + RN - 1 < GROUPS) read_ring<S, RN>(q + RN - 1, stage[at], wo, lane, ring, (q + RN - 1) % RN);
        else read_ring<S, RN>(q + RN - 1 - GROUPS, stage[after], wo, lane, ring, (q + RN - 1) % RN);
        if (q < S::FI) x_next[q] = read_columns<S::PITCH_I>(stage[after].a, wk + 32 * q, 0, lane);
        constexpr int PIECES = S::CO + S::CI, FIRST = GROUPS > 2 * PIECES ? 1 : 0;
        static_assert(!RING || GROUPS >= FIRST + 2 * PIECES, "every piece has its place");
        if (q >= FIRST && q - FIRST < PIECES) deposit_piece<T, S, WHOLE>(q - FIRST, f, stage[last], skipped, from.shift, tid, true, bias);
        if (q >= FIRST + PIECES && q - FIRST - PIECES < PIECES) fetch_piece<T, S, true>(q - FIRST - PIECES, a, from, 0, advance, blocks, tid, f);
      }
#pragma unroll
      for (int m = 0; m < GROUPS * S::FI; ++m) {
        constexpr int kValu = 0x2, kMfma = 0x8, kRead = 0x100;
        __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kValu, 5, 0);
        if (m % 2 == 0) __builtin_amdgcn_sched_group_barrier(kRead, 2, 0);
      }
      __syncthreads();
      at = after;
    };
    // One wave a SIMD issues in order: what is to run beside the matrix instructions has to stand between them.
    auto run = [&](auto with_sums) __attribute__((always_inline)) {
      for (; (i + 4) * S::KT <= n; i += 2) {   // (the stages that are written, the one after next and the one behind it, are whole)
        step(even, i, with_sums, std::true_type());
        step(odd, i + 1, with_sums, std::true_type());
      }
      for (; i < stages; i += 2) {
        step(even, i, with_sums, std::false_type());
        if (i + 1 < stages) step(odd, i + 1, with_sums, std::false_type());
      }
    };
    if constexpr (RING) {
      if (n < S::KT) {
        read_operands<S>(stage[0], 0, wo, wk, lane, now);
        multiply<S>(now, acc);
      } else {
        for (; (i + 4) * S::KT <= n; i += 2) {
          ring_step(even, i, xa, xb, std::true_type());
          ring_step(odd, i + 1, xb, xa, std::true_type());
        }
        for (; i < stages; i += 2) {
          ring_step(even, i, xa, xb, std::false_type());
          if (i + 1 < stages) ring_step(odd, i + 1, xb, xa, std::false_type());
        }
      }
    } else if (n < S::KT) {
      multiply<S>(now, acc);
      if (S::KT == 32) {
        read_operands<S>(stage[0], 16, wo, wk, lane, next);
        multiply<S>(next, acc);
      }
    } else if (S::P > 1 || sums) {   // (beside the splitting the additions do not matter)
      run(std::true_type());
    } else {
      run(std::integral_constant<bool, (S::P > 1)>());
    }
  }
  __syncthreads();
  const long long size = (long long)a.out * a.width;
  float* dw = pieces == 1 ? a.dweight + g * a.ldw : partial + (long long)blockIdx.y * (size + a.out);
  const bool inside = o0 + S::OUT <= a.out && k0 + S::IN <= a.width;
  // Gradients are read when all layers have theirs, so they go past the caches, whatever their size: G as a whole is what the caches would have to
  // hold.  Ordinary / past, us: 20 x 100 tokens, 2048 x 2048 float32 alone 108 / 92, with the scores and the update behind it 211 / 205 (bf16 204 /
  // 206; 84 MB of G 71 / 73; 8 x 400 tokens, 4096 x 4096 424 / 381); whole iterations with 20 workers, three layers: 2048 wide and 8192 outputs
  // float32 2935 / 2730, bf16 1757 / 1575, 1024 wide and 4096 outputs float32 924 / 876.  Pieces are joined at once.
  const bool past = inside && pieces == 1 && a.width % 32 == 0 && on_line(dw);
  if (past) {
#pragma unroll
    for (int r = 0; r < S::FO; ++r)
#pragma unroll
      for (int j = 0; j < S::FI; ++j) {
        float* to = dw + (long long)(o0 + wo + 32 * r + 4 * (lane / 32)) * a.width + k0 + wk + 32 * j + lane % 32;
#pragma unroll
        for (int e = 0; e < 16; ++e) __builtin_nontemporal_store(acc[r][j][e], &to[(long long)(8 * (e / 4) + e % 4) * a.width]);
      }
    keep_apart();
  } else {
#pragma unroll
    for (int r = 0; r < S::FO; ++r)
#pragma unroll
      for (int j = 0; j < S::FI; ++j) {
        const int k = k0 + wk + 32 * j + lane % 32, o = o0 + wo + 32 * r + 4 * (lane / 32);
        float* to = dw + (long long)o * a.width + k;
        if (inside) {
#pragma unroll
          for (int e = 0; e < 16; ++e) to[(long long)(8 * (e / 4) + e % 4) * a.width] = acc[r][j][e];
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (o + 8 * (e / 4) + e % 4 < a.out && k < a.width) to[(long long)(8 * (e / 4) + e % 4) * a.width] = acc[r][j][e];
        }
      }
  }
  if (sums) {
    constexpr int PER = S::OUT / 8, PARTS = (S::CHUNKS_O < kThreads ? S::CHUNKS_O : kThreads) / PER;
    float (*part)[S::OUT] = reinterpret_cast<float (*)[S::OUT]>(memory);
    if (tid < S::CHUNKS_O) {
#pragma unroll
      for (int j = 0; j < 8; ++j) part[tid / PER][8 * (tid % PER) + j] = bias[j];
    }
    __syncthreads();
    if (tid < S::OUT && o0 + tid < a.out) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < PARTS; ++i) sum += part[i][tid];
      float* db = pieces == 1 ? a.dbias + g * a.ldb : dw + size;
      db[o0 + tid] = sum;
    }
  }
}

// At most 32 outputs: reading the activations is what counts.  Each of a workgroup's four waves goes down its own tokens, 32 at a time, with
// LDS of its own and no barrier; the waves share 128 inputs and add up at the end.  The bias is the product with a column of ones.
// Ten outputs, 65536 tokens of 1000 inputs, fp16: 26 us (2.7 TB/s) and 4 us for the join of 64 pieces.  A SIMD issues vector instructions for 15
// thousand cycles of some 50 (widening the activations, splitting dy) and matrix instructions for 8; its two waves wait for half of their time,
// each at its own LDS writes and reads.  A second batch on its way: 29.9 instead of 28.5 us for both launches; twice the pieces: 37.5.
constexpr int kFewOutputs = 32, kFewInputs = 128, kFewTokens = 32;
constexpr int kFewPitchI = kFewInputs + 32, kFewPitchO = kFewOutputs;   // rows of 320 and 64 bytes: four lie on different banks when read

// (16-bit values in words of their own: packing them in pairs would wait for the loads)
template <typename T>
__device__ inline unsigned raw_bits(const T* p) {
  if constexpr (sizeof(T) == 2) return *reinterpret_cast<const uint16_t*>(p);
  else return *reinterpret_cast<const unsigned*>(p);
}
template <typename T>
__device__ inline float from_bits(unsigned bits) {
  if constexpr (sizeof(T) == 2) return (float)__builtin_bit_cast(T, (uint16_t)bits);
  else return __uint_as_float(bits);
}

template <int P>
struct FewStage {
  __bf16 a[16 * kFewPitchI];             // half a batch
  __bf16 y[P][kFewTokens * kFewPitchO];
};

// EACH: dy of a batch for a lane, at least kFewTokens * a.out / 64.
template <typename T, int P, int EACH>
__global__ __launch_bounds__(kThreads, EACH > 8 ? 1 : 2) void weight_grad_few_kernel(WeightGradArgs a, int pieces, float* partial) {
  constexpr int kWaves = kThreads / 64, FI = kFewInputs / 32;
  __shared__ union {
    FewStage<P> stage[kWaves];
    float joined[kFewOutputs][kFewInputs + 1];   // (the last column: the bias)
  } memory;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
  const int g = blockIdx.y / pieces, piece = blockIdx.y % pieces;
  const Span span = piece_of(a, g, piece, pieces);
  const int blocks = ckpt_blocks(a.width);
  const int k0 = (int)blockIdx.x * kFewInputs;
  const bool sums = blockIdx.x == 0 && a.dbias != nullptr;
  FewStage<P>& st = memory.stage[wave];
  // outputs behind the last are zeros for good
  for (int i = lane; i < P * kFewTokens * kFewPitchO; i += 64) (&st.y[0][0])[i] = (__bf16)0.f;
  f32x16 acc[FI] = {}, acc_bias = {};
  bf16x8 ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.f;
  // a lane's part of a batch: sixteen activations of four tokens, and every 64th of the batch's dy
  const int col = k0 + 16 * (lane % 8), at = col < blocks * kCkptBlock ? col : 0;   // (columns behind the last: the first ones)
  const unsigned pitch = (unsigned)blocks * kCkptBlock;
  const int elements = kFewTokens * a.out, magic = (65536 + a.out - 1) / a.out;
  auto token_of = [&](int i) { return (64 * i + lane) * magic >> 16; };   // (of 64 i + lane < 1024, a.out <= 32: the quotient is exact)
  // from the batch's first token on; beyond 32 bits only if lddy is, which the slow way below takes
  unsigned dy_at[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int e = 64 * i + lane < elements ? 64 * i + lane : 0, t = e * magic >> 16;
    dy_at[i] = (unsigned)t * (unsigned)a.lddy + (unsigned)(e - t * a.out);
  }
  const bool near = a.lddy < (1 << 24);
  struct Batch {
    uint4 words[4];
    uint8_t scale[4];
    unsigned dy[EACH];
  };
  auto load = [&](int t0, Batch& b) __attribute__((always_inline)) {
    if (t0 + kFewTokens <= span.end && near) {
      const uint8_t* values = a.values + (long long)t0 * pitch;
      const uint8_t* scales = a.scales + (long long)t0 * blocks;
      const T* dy = reinterpret_cast<const T*>(a.dy) + (long long)t0 * a.lddy;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        b.words[q] = *reinterpret_cast<const uint4*>(values + ((unsigned)(8 * q + lane / 8) * pitch + (unsigned)at));
        b.scale[q] = scales[(unsigned)(8 * q + lane / 8) * (unsigned)blocks + (unsigned)(at / kCkptBlock)];
      }
#pragma unroll
      for (int i = 0; i < EACH; ++i) b.dy[i] = raw_bits(dy + dy_at[i]);
    } else {
      const int last = span.end - 1;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const long long row = t0 + 8 * q + lane / 8 < last ? t0 + 8 * q + lane / 8 : last;   // (a copy of the last token has no dy)
        b.words[q] = *reinterpret_cast<const uint4*>(a.values + row * pitch + at);
        b.scale[q] = a.scales[row * blocks + at / kCkptBlock];
      }
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const int e = 64 * i + lane < elements ? 64 * i + lane : 0, t = e * magic >> 16;
        const long long row = t0 + t < last ? t0 + t : last;
        b.dy[i] = raw_bits(reinterpret_cast<const T*>(a.dy) + row * a.lddy + (e - t * a.out));
      }
    }
  };
  Batch now, next;
  const int step = kFewTokens * kWaves;
  int t0 = span.begin + kFewTokens * wave;
  if (t0 < span.end) load(t0, now);
  for (; t0 < span.end; t0 += step) {
    const int n = span.end - t0;
    load(t0 + step < span.end ? t0 + step : t0, next);   // (always: loads that may not have been sent are waited for as if they were the last)
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int e = 64 * i + lane, t = token_of(i), o = e - t * a.out;
      float rest = t < n ? from_bits<T>(now.dy[i]) : 0.f;
      const bool infinite = fabsf(rest) == __builtin_inff();
      if (e < elements) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const unsigned bits = __float_as_uint(rest);
          *reinterpret_cast<uint16_t*>(&st.y[p][t * kFewPitchO + o]) = (uint16_t)(bits >> 16);
          // (infinity less itself would be NaN; a NaN whose bits the first piece loses is one in the next)
          rest = infinite ? 0.f : rest - __uint_as_float(bits & 0xffff0000u);
        }
      }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      row_sync<1>();
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const float s = ckpt_scale((int)now.scale[2 * half + q] - 127);
        const uint4 w = now.words[2 * half + q];
        __bf16* to = &st.a[(8 * q + lane / 8) * kFewPitchI + 16 * (lane % 8)];
        *reinterpret_cast<bf16x8*>(to) = widen8(w.x, w.y, s);
        *reinterpret_cast<bf16x8*>(to + 8) = widen8(w.z, w.w, s);
      }
      row_sync<1>();
      bf16x8 x[FI];
#pragma unroll
      for (int j = 0; j < FI; ++j) x[j] = read_columns<kFewPitchI>(st.a, 32 * j, 0, lane);
#pragma unroll
      for (int p = P - 1; p >= 0; --p) {
        const bf16x8 y = read_columns<kFewPitchO>(st.y[p], 0, 16 * half, lane);
#pragma unroll
        for (int j = 0; j < FI; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, x[j], acc[j], 0, 0, 0);
        if (sums) acc_bias = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, ones, acc_bias, 0, 0, 0);
      }
    }
    row_sync<1>();
    now = next;
  }
  for (int w = 0; w < kWaves; ++w) {
    __syncthreads();
    if (wave == w) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int o = 8 * (e / 4) + 4 * (lane / 32) + e % 4;
#pragma unroll
        for (int j = 0; j < FI; ++j) {
          float& sum = memory.joined[o][32 * j + lane % 32];
          sum = w == 0 ? acc[j][e] : sum + acc[j][e];
        }
        if (lane % 32 == 0) {
          float& sum = memory.joined[o][kFewInputs];
          sum = w == 0 ? acc_bias[e] : sum + acc_bias[e];
        }
      }
    }
  }
  __syncthreads();
  const long long size = (long long)a.out * a.width;
  float* dw = pieces == 1 ? a.dweight + g * a.ldw : partial + (long long)blockIdx.y * (size + a.out);
  for (int i = tid; i < a.out * kFewInputs; i += kThreads) {
    const int o = i / kFewInputs, k = k0 + i % kFewInputs;
    if (k < a.width) dw[(long long)o * a.width + k] = memory.joined[o][i % kFewInputs];
  }
  if (sums && tid < a.out) (pieces == 1 ? a.dbias + g * a.ldb : dw + size)[tid] = memory.joined[tid][kFewInputs];
}

// The pieces of a group's tokens.  A wave takes 64 gradients and every so-manieth piece; the waves' sums are added in their order.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(64 * kJoinWaves) void weight_grad_join_kernel(WeightGradArgs a, int pieces, const float* __restrict__ partial) {
  __shared__ float shared[kJoinWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, waves = blockDim.x / 64, g = blockIdx.y;
  const long long n = (long long)a.out * a.width, all = n + (a.dbias != nullptr ? a.out : 0), stride = n + a.out;
  const float* p = partial + (long long)g * pieces * stride;
  for (long long base = 64LL * blockIdx.x; base < all; base += 64LL * gridDim.x) {
    const long long i = base + lane;
    float sum = 0.f;
    if (i < all) {
#pragma unroll 4
      for (int s = wave; s < pieces; s += waves) sum += p[s * stride + i];
    }
    shared[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && i < all) {
      for (int w = 1; w < waves; ++w) sum += shared[w][lane];
      if (i < n)
        a.dweight[g * a.ldw + i] = sum;
      else
        a.dbias[g * a.ldb + i - n] = sum;
    }
    __syncthreads();
  }
}

template <typename S>
long long tiles_of(int out, int width) { return (long long)ceil_div(out, S::OUT) * ceil_div(width, S::IN); }

enum Shape { kFew, kMid, kWide };
struct Plan {
  Shape shape;
  int pieces;   // that a group's tokens are cut into: where the output alone leaves most of the chip idle
};
Plan plan_for(int rows, int out, int width, int m) {
  Plan p;
  if (out <= kFewOutputs) {
    p.shape = kFew;
    const long long strips = (long long)ceil_div(width, kFewInputs) * m;
    const long long pieces = 512 / strips, most = rows / m / (kFewTokens * 4);
    p.pieces = (int)std::max(1LL, std::min(pieces, most));
    return p;
  }
  p.shape = kMid;
  if (out > MidTile<1>::OUT && width > MidTile<1>::IN) {
    // wide tiles, one for every compute unit at least: as they are, or the tokens cut where they are many (bf16, 16384 tokens,
    // 4096 x 1024: 154 us with four pieces of wide tiles, 197 with two of 128 x 128)
    const long long wide = tiles_of<WideTile<1>>(out, width) * m, pieces = (255 + wide) / wide;
    if (rows / m >= (wide >= 256 ? 64 : 1024 * pieces)) {
      p.shape = kWide;
      p.pieces = (int)pieces;
      return p;
    }
  }
  // two workgroups a compute unit, or one where the output is so small that joining the pieces counts (bf16, 6292 tokens, 64 x 2112: 20.5 us
  // with 256 workgroups, 24.4 with 512; 8192 tokens, 1000 x 1024: 44.0 and 42.5)
  const long long tiles = tiles_of<MidTile<1>>(out, width) * m, pieces = (tiles < 64 ? 256 : 512) / tiles, most = rows / m / 128;
  p.pieces = (int)std::max(1LL, std::min(pieces, most));
  return p;
}

template <typename T, int P, int EACH>
hipError_t start_few(const WeightGradArgs& a, int pieces, float* partial, hipStream_t stream) {
  hipLaunchKernelGGL((weight_grad_few_kernel<T, P, EACH>), dim3(ceil_div(a.width, kFewInputs), a.m * pieces), dim3(kThreads), 0, stream, a,
                     pieces, partial);
  return hipGetLastError();
}
template <typename T, int P>
hipError_t start_few(const WeightGradArgs& a, int pieces, float* partial, hipStream_t stream) {
  if (a.out <= 4) return start_few<T, P, 2>(a, pieces, partial, stream);
  if (a.out <= 12) return start_few<T, P, 6>(a, pieces, partial, stream);
  if (a.out <= 16) return start_few<T, P, 8>(a, pieces, partial, stream);
  return start_few<T, P, 16>(a, pieces, partial, stream);
}

template <typename T, typename S>
hipError_t start(const WeightGradArgs& a, int pieces, float* partial, hipStream_t stream) {
  constexpr size_t lds = 3 * sizeof(Stage<S>);
  static_assert(lds <= 160 * 1024 && sizeof(float) * 8 * (S::CHUNKS_O < kThreads ? S::CHUNKS_O : kThreads) <= lds, "LDS");
  const auto kernel = weight_grad_kernel<T, S>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)tiles_of<S>(a.out, a.width), a.m * pieces), dim3(kThreads), lds, stream, a,
                     ceil_div(a.width, S::IN), pieces, partial);
  return hipGetLastError();
}

template <typename T, int P, bool ODD>
hipError_t start_shape(const WeightGradArgs& a, const Plan& p, float* partial, hipStream_t stream) {
  switch (p.shape) {
    case kFew: return start_few<T, P>(a, p.pieces, partial, stream);
    case kMid: return start<T, MidTile<P, ODD>>(a, p.pieces, partial, stream);
    default: return start<T, WideTile<P, ODD>>(a, p.pieces, partial, stream);
  }
}
template <typename T, int P>
hipError_t start_type(const WeightGradArgs& a, const Plan& p, float* partial, hipStream_t stream) {
  return a.out % 8 != 0 ? start_shape<T, P, true>(a, p, partial, stream) : start_shape<T, P, false>(a, p, partial, stream);
}

}  // namespace

bool weight_gradient_fits(int out, int width) { return tiles_of<MidTile<1>>(out, width) * kThreads < (1LL << 31); }

size_t weight_gradient_workspace_bytes(int rows, int out, int width, int m) {
  const Plan p = plan_for(rows, out, width, m);
  if (p.pieces == 1) return 256;
  return align_up((size_t)m * p.pieces * ((size_t)out * width + out) * sizeof(float), 256);
}

hipError_t launch_weight_gradient(const WeightGradArgs& a, void* workspace, hipStream_t stream) {
  const Plan p = plan_for(a.rows, a.out, a.width, a.m);
  float* partial = reinterpret_cast<float*>(workspace);
  hipError_t e;
  switch (a.dtype) {
    case ZENO_F32: e = start_type<float, 3>(a, p, partial, stream); break;
    case ZENO_BF16: e = start_type<__bf16, 1>(a, p, partial, stream); break;
    default: e = start_type<_Float16, 2>(a, p, partial, stream); break;
  }
  if (e != hipSuccess || p.pieces == 1) return e;
  const long long n = (long long)a.out * a.width + a.out, blocks = (n + 63) / 64;
  int waves = 1;
  while (waves < kJoinWaves && 4 * waves < p.pieces) waves *= 2;   // four pieces a wave
  hipLaunchKernelGGL(weight_grad_join_kernel, dim3((unsigned)(blocks < 8192 ? blocks : 8192), a.m), dim3(64 * waves), 0, stream, a, p.pieces,
                     partial);
  return hipGetLastError();
}

}  // namespace zeno
