// Log probabilities of a linear layer's outputs, z = h W^T + bias, without keeping the logits, and their gradients:
//   log p_y = z_y - M - log s,  M = max z,  s = sum exp(z - M),  H = log s - (sum exp(z - M) (z - M)) / s,
//   dz_j = g [j = y] - p_j (g + q (log p_j + H)),  dh = dz W,  dW_g = dz_g^T h_g,  db_g = sum dz.
//
// Forward: tiles of h W^T on the matrix cores; a tile leaves (max, sum of exponentials) for each of its tokens, which are joined behind.  The
// logits stay float32 and never leave the registers.
// Backward: the vocabulary in pieces.  A piece's logits are formed again, their dz goes to the workspace as 16-bit planes, and two products read
// it: with W for dh, with h for dW.
// Operands are planes of 16 bits: bf16 and fp16 as they are; float32 is a sum of three bf16 pieces, of whose nine products six are taken, those
// that are left out lie below 2^-24 of the product.
// dz in 16-bit types.  dh is rounded to the type itself, and takes dz as two planes of it, 16 or 22 bits: dz sums to nothing over the vocabulary, so what the
// rows of W share cancels, and one plane's roundings, which do not cancel, would stand out by as much (rows that share ten times their spread, peaked tokens:
// dh five times as far from 64 bits as its own rounding, ten times for the entropy's gradient alone).  dW and db are float32 and take dz as two fp16 planes, 22 bits, scaled
// so that the largest gradient comes near fp16's largest: the sum of two bf16 planes has 16 bits, and its error (4e-6 of dW) would be several times that of the float32 sums.
// fp16 planes need h in fp16 too: bf16's eight bits fit, once a power of two for each column has brought its range there.
#include "zeno_linear_plan.h"
#include "zeno_tokens.h"
#include <algorithm>
#include <type_traits>

namespace zeno {
namespace {

typedef unsigned short u16;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) unsigned char* lds_ptr;

constexpr int kStep = 32;      // of the contraction in a stage

// BM x BN of the product for a workgroup of WM x WN waves.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_ = 4>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int FM = BM / WM / 32, FN = BN / WN / 32;   // 32 x 32 blocks of a wave
  static constexpr int A_BYTES = BM * kStep * 2, STAGE = (BM + BN) * kStep * 2;
  static constexpr int LOADS_A = A_BYTES / 1024 / WAVES, LOADS_B = BN * kStep * 2 / 1024 / WAVES, LOADS = LOADS_A + LOADS_B;
  // stages in LDS: one that is multiplied, one that is whole, and what is on its way (of two: what is on its way); with two planes of A in a stage they
  // are longer and fewer
  template <int PLANES> static constexpr int STAGE_OF = STAGE + (PLANES - 1) * A_BYTES;
  template <int PLANES> static constexpr int STAGES_OF = PLANES == 1 ? STAGES_ : STAGES_ - 1;
  static constexpr int GROUPS = BM == 256 ? 1 : (STAGES_ == 4 ? 2 : 3);   // workgroups of a compute unit
  static constexpr int PITCH = BM + 8;                         // of planes of dz on their way out, [32 WN tokens][vocabulary]
  static constexpr int DZ_PLANES = 3;                          // at a time
  static constexpr int DZ = DZ_PLANES * 32 * WN * PITCH * 2;
  template <int PLANES> static constexpr int LDS = STAGES_OF<PLANES> * STAGE_OF<PLANES>;
  static_assert(GROUPS * DZ <= 160 * 1024 && GROUPS * LDS<2> <= 160 * 1024 && GROUPS * LDS<1> <= 160 * 1024, "what there is");
};
using WideTile = Tile<256, 256, 2, 2>;
using MidTile = Tile<128, 128, 2, 2>;
// Three workgroups a compute unit, a stage less: logits and weight gradients, whose stores and exponentials another workgroup runs beside (20 x 100 tokens'
// weight gradients, 32000 x 1024: 646 us, with two workgroups 700; 777 x 10007 x 513 float32: logits 108 and 111, weight gradients 83 and 85).  Sums over
// the vocabulary keep two: with one plane of dz they were faster so (20 x 100 tokens' dz W 171 us, with three 190); with two planes there is little between them (294 and 286,
// 250 tokens 103 and 100; float32 120 and 110).
using ThirdTile = Tile<128, 128, 2, 2, 3>;

// An operand: planes of 16-bit values, `plane` elements apart, rows ld apart and on 16 bytes.
struct Side {
  const u16* p;
  long long ld, plane;
  int extent;   // rows along the contraction: how many there are; across it: columns, a multiple of eight
};
// Which planes are multiplied, the smallest products first.
struct Pairs {
  int count;
  unsigned a, b;   // four bits a plane, the first pair's lowest
};
__device__ inline int plane_of(unsigned planes, int i) { return (int)(planes >> (4 * i) & 15); }

__device__ __attribute__((aligned(16))) unsigned zero_chunk[4];

// N times 64 lanes x 16 bytes, from `base` + off[n] + 1024 n to consecutive bytes of LDS from `to` on (the instruction's offset counts on both sides), in
// no register and unseen by the compiler's wait counts (which would drain all loads before every read of LDS); begin_stage() waits for
// them.  m0 is saved because it cannot be declared as written.
template <int N>
__device__ inline void copy_to_lds(const unsigned char* base, const unsigned (&off)[N], unsigned to) {
  static_assert(N == 2 || N == 4, "copies of a wave");
  unsigned saved;
  if constexpr (N == 4)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %6\n\t"
                 "global_load_lds_dwordx4 %2, %6 offset:1024\n\tglobal_load_lds_dwordx4 %3, %6 offset:2048\n\t"
                 "global_load_lds_dwordx4 %4, %6 offset:3072\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(to), "s"(base)
                 : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %4\n\t"
                 "global_load_lds_dwordx4 %2, %4 offset:1024\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "v"(off[0]), "v"(off[1]), "s"(to), "s"(base)
                 : "memory");
}
__device__ inline void copy_to_lds(const unsigned char* from, unsigned to) {   // each lane from its own address
  unsigned saved;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
               : "=&s"(saved)
               : "v"(from), "s"(to)
               : "memory");
}
// All but the `pending` copies issued last have arrived, for every wave, and every wave has read what the stage before held.
template <int PENDING>
__device__ inline void begin_stage() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PENDING) : "memory");
}

// A side's part of a stage.  ACROSS false: rows of the side along the contraction, 64 bytes a row; chunk c of row r stands at c ^ (r / 4 % 4),
// so that sixteen rows' chunks lie on all banks.  ACROSS true: the contraction's rows, B columns each; blocks of 32 columns are
// exchanged by a row's number for the same reason.
template <int B>
__device__ inline int block_of(int k) { return B >= 256 ? (k & 3) | ((k >> 1) & 4) : (k & 3); }

// What a wave copies: N times 1 KB of the part, one behind the other.
template <bool ACROSS, int B, int WAVES>
struct Loader {
  static constexpr int N = B * kStep * 2 / 1024 / WAVES, PER = 512 / B;   // PER: rows of a copy, if ACROSS
  const unsigned char* base;   // of this stage, less 1024 (N - 1)
  unsigned off[N];             // the lane's; offsets are below 2^32 because pitches are below kMostPitch
  unsigned to;                 // in LDS
  int k;                       // of the lane's first value in its first copy
  __device__ inline void start(const Side& s, int plane, long long first, long long x0, int wave, int lane, unsigned lds) {
    to = lds + 1024 * N * wave;
    const u16* p = s.p + plane * s.plane + (ACROSS ? first * s.ld + x0 : x0 * s.ld + first);
    base = reinterpret_cast<const unsigned char*>(p) - 1024 * (N - 1);
    k = ACROSS ? PER * N * wave + lane / (64 / PER) : 8 * ((lane % 4) ^ (lane / 16));
#pragma unroll
    for (int n = 0; n < N; ++n) {
      unsigned at;
      if (!ACROSS) {
        const long long row = x0 + 16 * (N * wave + n) + lane / 4;   // a row behind the last is the last once more
        at = (unsigned)(((row < s.extent ? row : s.extent - 1) - x0) * s.ld) + k;
      } else {
        const int slot = lane % (64 / PER), col = 32 * ((slot / 4) ^ block_of<B>(k + PER * n)) + 8 * (slot % 4);
        at = (unsigned)((k + PER * n) * s.ld) + (x0 + col < s.extent ? col : 0);   // (columns behind the last: any, their products are dropped)
      }
      off[n] = 2 * at + 1024 * (N - 1 - n);
    }
  }
  // A stage whose contraction is there as a whole, or of which `left` is, and zeros behind.
  // `further`: bytes to another plane.
  __device__ inline void issue(long long further, unsigned stage_offset) { copy_to_lds<N>(base + further, off, to + stage_offset); }
  __device__ inline void issue_end(long long further, unsigned stage_offset, int left) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const bool live = k + (ACROSS ? PER * n : 0) < left;
      copy_to_lds(live ? base + further + off[n] + 1024 * n : reinterpret_cast<const unsigned char*>(zero_chunk), to + stage_offset + 1024 * n);
    }
  }
};
constexpr long long kMostPitch = 1LL << 22;

// Operands of 32 rows (columns) and sixteen of the contraction: lane l has row l % 32, values 8 (l / 32) + 0..7.  F of them are a wave's, from
// row w on.
template <bool ACROSS, int B, int F>
struct Reader {
  unsigned base[ACROSS ? F : 2];
  __device__ inline void start(unsigned part, int w, int lane) {
    if (!ACROSS) {
      base[0] = part + (w + lane % 32) * (2 * kStep) + 16 * ((lane / 32) ^ (lane % 32 / 4 % 4));
      base[1] = base[0] ^ 32;   // the chunks of the second sixteen (parts begin on 64 bytes)
    } else {
      const int row = 8 * (lane / 32) + lane % 16 / 4;
#pragma unroll
      for (int r = 0; r < F; ++r)
        base[r] = part + row * (2 * B) + 64 * ((w / 32 + r) ^ block_of<B>(row)) + 32 * (lane / 16 % 2) + 8 * (lane % 4);
    }
  }
  __device__ inline s16x8 read(int r, int k, unsigned stage_offset) const {
    if constexpr (!ACROSS) {
      typedef const __attribute__((address_space(3))) s16x8* p;
      return *(p)(base[k / 16] + stage_offset + r * 32 * (2 * kStep));
    } else {
      typedef __attribute__((address_space(3))) s16x4* p;
      const unsigned at = base[r] + stage_offset;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p)(at + k * (2 * B)));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p)(at + (k + 4) * (2 * B)));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};
template <bool HALF>
__device__ inline f32x16 multiply(s16x8 a, s16x8 b, f32x16 c) {
  if constexpr (HALF)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The operands of sixteen of the contraction.
template <typename S, int PLANES>
struct Operands {
  s16x8 x[PLANES][S::FM], y[S::FN];
};

// acc += the product of BM rows (columns) of A from m0 on and BN of B from n0 on over `length` of the contraction, which begins at `first`.
// While a stage is multiplied the next is whole, so that its first operands are read before the barrier; those behind it are on their way.
// A wave of a wide tile has its SIMD to itself and issues in order: what runs beside the matrix instructions stands between them.
// PLANES: 1, pairs of planes one after the other; 2, the first two planes of A in one stage, the second, smaller one first, each times B's first.
// SUMS: also the sums of A's rows over the contraction, as products with ones; the WN waves that have the same rows take FM / WN blocks of them each.
template <typename S, bool HALF, bool A_ACROSS, bool B_ACROSS, int PLANES, bool SUMS>
__device__ inline void product(const Side& a, const Side& b, const Pairs& pairs, long long m0, long long n0, long long first, int length,
                               unsigned char* memory, f32x16 (&acc)[S::FM][S::FN], f32x16 (&sums)[S::FM / S::WN]) {
  constexpr int STAGE = S::template STAGE_OF<PLANES>, STAGES = S::template STAGES_OF<PLANES>, LOADS = S::LOADS + (PLANES - 1) * S::LOADS_A;
  constexpr int OPERANDS = PLANES * S::FM + S::FN, PRODUCTS = PLANES * S::FM * S::FN, READ_UNTIL = PRODUCTS > 8 ? PRODUCTS / 2 : PRODUCTS;
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wm = (wave % S::WM) * (32 * S::FM), wn = (wave / S::WM) * (32 * S::FN);
  const unsigned lds = (unsigned)(uintptr_t)(lds_ptr)memory, lds_b = lds + PLANES * S::A_BYTES;
  const int steps = (length + kStep - 1) / kStep, total = PLANES == 1 ? steps * pairs.count : steps;
  if (total == 0) return;
  Loader<A_ACROSS, S::BM, S::WAVES> la;
  Loader<B_ACROSS, S::BN, S::WAVES> lb;
  la.start(a, PLANES == 1 ? plane_of(pairs.a, 0) : 0, first, m0, wave, lane, lds);
  lb.start(b, PLANES == 1 ? plane_of(pairs.b, 0) : 0, first, n0, wave, lane, lds_b);
  Reader<A_ACROSS, S::BM, S::FM> ra;
  Reader<B_ACROSS, S::BN, S::FN> rb;
  ra.start(lds, wm, lane);
  rb.start(lds_b, wn, lane);
  const long long step_a = 2 * kStep * (A_ACROSS ? a.ld : 1), step_b = 2 * kStep * (B_ACROSS ? b.ld : 1);
  int pair = 0, left = length;   // of the next stage to fetch
  auto fetched = [&]() __attribute__((always_inline)) {
    la.base += step_a;
    lb.base += step_b;
    left -= kStep;
    if (PLANES == 1 && left <= 0 && pair + 1 < pairs.count) {
      la.base += 2 * (plane_of(pairs.a, pair + 1) - plane_of(pairs.a, pair)) * a.plane - steps * step_a;
      lb.base += 2 * (plane_of(pairs.b, pair + 1) - plane_of(pairs.b, pair)) * b.plane - steps * step_b;
      left = length;
      ++pair;
    }
  };
  // part 0 .. PLANES - 1: a plane of A, PLANES: B
  auto send = [&](int part, unsigned at, bool whole) __attribute__((always_inline)) {
    if (part < PLANES) {
      if (whole) la.issue(2 * part * a.plane, at + part * S::A_BYTES);
      else la.issue_end(2 * part * a.plane, at + part * S::A_BYTES, left);
    } else {
      if (whole) lb.issue(0, at);
      else lb.issue_end(0, at, left);
    }
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i)
    if (i < total) {
#pragma unroll
      for (int part = 0; part <= PLANES; ++part) send(part, i * STAGE, false);
      fetched();
    }
  if (STAGES == 4 && total > 2) begin_stage<LOADS>();   // the first two are whole
  else if (STAGES > 2) begin_stage<0>();
  Operands<S, PLANES> now, next;
  auto read_one = [&](int n, int k, unsigned at, Operands<S, PLANES>& o) __attribute__((always_inline)) {   // in the order in which they are needed
    if (n >= 1 && n <= S::FN) {
      o.y[n - 1] = rb.read(n - 1, k, at);
    } else {
      const int i = n == 0 ? 0 : n - S::FN, plane = PLANES - 1 - i / S::FM;
      o.x[plane][i % S::FM] = ra.read(i % S::FM, k, at + plane * S::A_BYTES);
    }
  };
  s16x8 ones;                    // of B's first plane: each plane of A counts once
  int its = 0, until = 0;        // pair that is multiplied, and the step where the next begins
  auto set_ones = [&](int i) __attribute__((always_inline)) {
    if (!SUMS || i < until) return;
    its = i == 0 ? 0 : its + 1;
    until += steps;
    const short one = PLANES == 1 && plane_of(pairs.b, its) != 0 ? 0 : (HALF ? 0x3c00 : 0x3f80);
    ones = s16x8{one, one, one, one, one, one, one, one};
  };
  // Sixteen of the contraction; the next sixteen's operands are read behind the first products.
  auto half = [&](const Operands<S, PLANES>& use, Operands<S, PLANES>& fill, int k, unsigned at, auto beside) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < PRODUCTS; ++q) {
      const int plane = PLANES - 1 - q / (S::FM * S::FN), r = q / S::FN % S::FM, j = q % S::FN;
      acc[r][j] = multiply<HALF>(use.x[plane][r], use.y[j], acc[r][j]);
      if (SUMS && j == S::FN - 1 && r % S::WN == S::WN - 1) {
        static_assert(S::WN == 2, "two waves have the same rows");
        sums[r / 2] = multiply<HALF>(wave / S::WM == 0 ? use.x[plane][r - 1] : use.x[plane][r], ones, sums[r / 2]);
      }
#pragma unroll
      for (int n = 0; n < OPERANDS; ++n)
        if (k >= 0 && n * READ_UNTIL / OPERANDS == q) read_one(n, k, at, fill);
      beside(q);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  unsigned at = 0;               // the stage that is multiplied
  if constexpr (STAGES == 2) {   // the other workgroups of the compute unit run beside what this one waits for
    for (int i = 0; i < total; ++i) {
      begin_stage<0>();
      if (i + 1 < total) {
        const bool whole = left >= kStep;
#pragma unroll
        for (int part = 0; part <= PLANES; ++part) send(part, STAGE - at, whole);
        fetched();
      }
      set_ones(i);
#pragma unroll
      for (int n = 0; n < OPERANDS; ++n) read_one(n, 0, at, now);
      half(now, next, 16, at, [](int) __attribute__((always_inline)) {});
      half(next, now, -1, at, [](int) __attribute__((always_inline)) {});
      at = STAGE - at;
    }
    return;
  }
#pragma unroll
  for (int n = 0; n < OPERANDS; ++n) read_one(n, 0, 0, now);
  for (int i = 0; i < total; ++i) {
    const unsigned after = at + STAGE == STAGES * STAGE ? 0 : at + STAGE, to = at == 0 ? (STAGES - 1) * STAGE : at - STAGE;
    const bool more = i + STAGES - 1 < total, whole = left >= kStep;   // a stage is fetched; it is whole
    set_ones(i);
    half(now, next, 16, at, [&](int q) __attribute__((always_inline)) {
#pragma unroll
      for (int part = 0; part <= PLANES; ++part)
        if (q == part * PRODUCTS / (PLANES + 1) && more) {
          send(part, to, whole);
          if (part == PLANES) fetched();
        }
    });
    // (behind the last stage: what stands in LDS, for no one)
    half(next, now, 0, after, [](int) __attribute__((always_inline)) {});
    if (STAGES == 4 && more) begin_stage<LOADS>();   // the stage after next is whole
    else begin_stage<0>();
    at = after;
  }
}
template <typename S, bool HALF, bool A_ACROSS, bool B_ACROSS>
__device__ inline void product(const Side& a, const Side& b, const Pairs& pairs, long long m0, long long n0, long long first, int length,
                               unsigned char* memory, f32x16 (&acc)[S::FM][S::FN]) {
  f32x16 none[S::FM / S::WN];
  product<S, HALF, A_ACROSS, B_ACROSS, 1, false>(a, b, pairs, m0, n0, first, length, memory, acc, none);
}

// Where a workgroup's tile lies: each of the eight dies, to which workgroups go in turn, takes a run of tiles, in patches of eight rows of tiles.
struct Place {
  int m, n;
};
__device__ inline Place place_of(unsigned id, unsigned tiles_m, unsigned tiles_n) {
  const unsigned total = tiles_m * tiles_n, die = id % 8, q = total / 8, r = total % 8;
  const unsigned at = die * q + (die < r ? die : r) + id / 8;
  constexpr unsigned ROWS = 8;
  const unsigned patch = ROWS * tiles_n, first = at / patch * ROWS, rows = tiles_m - first < ROWS ? tiles_m - first : ROWS;
  Place p;
  p.m = (int)(first + at % patch % rows);
  p.n = (int)(at % patch / rows);
  return p;
}

constexpr float kLog2e = 1.4426950408889634f;
__device__ inline float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// What the logits' kernels share: A = rows of W from the vocabulary's `v0` on, B = h.
struct LogitArgs {
  Side w, h;
  Pairs pairs;
  int tiles_m, tiles_n, width;
  int v0, vocab, rows;     // first value of this launch's vocabulary; the whole one; tokens
  const float* bias;
  const int32_t* labels;
};
// Row of a wave's 32 x 32 block that element e of a lane holds.
__device__ inline int row_of(int e, int lane) { return 8 * (e / 4) + 4 * (lane / 32) + e % 4; }
// The place 16 r + e of a row among FM blocks, if the lane holds it; -1 if it does not.
template <int FM>
__device__ inline int place_in(int row, int lane) {
  const bool mine = row >= 0 && row < 32 * FM && (row / 4 & 1) == lane / 32;
  return mine ? row / 32 * 16 + row % 32 / 8 * 4 + row % 4 : -1;
}
// The value at a place, and another one in it; a place of -1 is none.
template <int FM>
__device__ inline float value_at(const float (&z)[FM][16], int place) {
  float v = 0.f;
#pragma unroll
  for (int r = 0; r < FM; ++r)
#pragma unroll
    for (int e = 0; e < 16; ++e) v = place == 16 * r + e ? z[r][e] : v;
  return v;
}
template <int FM>
__device__ inline void put_at(float (&z)[FM][16], int place, float v) {
  asm volatile("" : "+v"(place));   // (or the comparisons of value_at() are kept for here, in registers that there are too few of)
#pragma unroll
  for (int r = 0; r < FM; ++r)
#pragma unroll
    for (int e = 0; e < 16; ++e) z[r][e] = place == 16 * r + e ? v : z[r][e];
}

// The bias of a wave's rows from v on.  What lies behind the vocabulary gets -inf: its products are copies of the last row's, so this makes a NaN of
// none that is not there.
template <typename S>
struct Bias {
  float b[S::FM][16];
};
template <typename S>
__device__ inline void load_bias(const LogitArgs& a, int v, int lane, Bias<S>& o) {
  const bool whole = v + 32 * S::FM <= a.vocab;
#pragma unroll
  for (int r = 0; r < S::FM; ++r)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int at = v + 32 * r + row_of(4 * q, lane);
      f32x4 raw = {0.f, 0.f, 0.f, 0.f};
      if (whole) {
        if (a.bias != nullptr) raw = *reinterpret_cast<const f32x4_a4*>(a.bias + at);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (at + i >= a.vocab) raw[i] = -__builtin_inff();
          else if (a.bias != nullptr) raw[i] = a.bias[at + i];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) o.b[r][4 * q + i] = raw[i];
    }
}
// A block of 32 tokens' logits.
template <typename S>
__device__ inline void logits_of(const Bias<S>& bias, const f32x16 (&acc)[S::FM][S::FN], int j, float (&z)[S::FM][16]) {
#pragma unroll
  for (int r = 0; r < S::FM; ++r)
#pragma unroll
    for (int e = 0; e < 16; ++e) z[r][e] = acc[r][j][e] + bias.b[r][e];
}
// ---- forward: for each token and each slice of 32 FM values (max, sum of exp(z - max)) and, for the entropy, the sum of exp(z - max) (z - max)
// A lane's share of FM blocks of logits of one token, which lane ^ 32 has the other share of, as a slice's sums at `at`; `hit`: the label's place in the
// slice, of which `inside` values exist.
template <int FM>
__device__ inline void leave_stats(const float (&z)[FM][16], int lane, int token, bool live, int hit, int inside, long long at, float2* part_s,
                                   float* part_u, float* label_logit) {
  float top = -__builtin_inff();
#pragma unroll
  for (int r = 0; r < FM; ++r)
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, z[r][e]);
  top = fmaxf(top, __shfl_xor(top, 32));
  const float from = top == -__builtin_inff() ? 0.f : top;
  // (the largest value's exponential is 1, to the bit: of a token that is nearly certain, what is left counts)
  float part[2] = {}, u = 0.f;
  if (part_u == nullptr) {
#pragma unroll
    for (int r = 0; r < FM; ++r)
#pragma unroll
      for (int e = 0; e < 16; ++e) part[e % 2] += exp_fast(z[r][e] - from);
  } else {
#pragma unroll
    for (int r = 0; r < FM; ++r)
#pragma unroll
      for (int e = 0; e < 16; ++e) {   // (where the exponential is 0, its argument is cut off: 0 * -inf would be NaN)
        const float d = z[r][e] - from, x = exp_fast(d);
        part[e % 2] += x;
        u = fmaf(x, fmaxf(d, -256.f), u);
      }
  }
  float s = part[0] + part[1];
  s += __shfl_xor(s, 32);
  if (part_u != nullptr) u += __shfl_xor(u, 32);
  if (live && lane < 32) {
    part_s[at] = make_float2(top, s);
    if (part_u != nullptr) part_u[at] = u;
  }
  const int place = live && hit < inside ? place_in<FM>(hit, lane) : -1;
  if (__any(place >= 0)) {
    const float own = value_at<FM>(z, place);
    if (place >= 0) label_logit[token] = own;
  }
}

struct StatArgs {
  LogitArgs l;
  int slice0;            // of this launch's vocabulary
  float2* part;          // [slices][rows]
  float* part_u;         // [slices][rows] or nullptr
  float* label_logit;    // [rows]
};
template <typename S, bool HALF>
__global__ __launch_bounds__(S::THREADS, S::GROUPS) void logit_stats_kernel(StatArgs a) {
  extern __shared__ __align__(1024) unsigned char memory[];
  const Place t = place_of(blockIdx.x, a.l.tiles_m, a.l.tiles_n);
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int v = a.l.v0 + t.m * S::BM + (wave % S::WM) * (32 * S::FM), token0 = t.n * S::BN + (wave / S::WM) * (32 * S::FN) + lane % 32;
  Bias<S> bias;   // (these arrive beside the operands)
  load_bias<S>(a.l, v, lane, bias);
  int label[S::FN];
#pragma unroll
  for (int j = 0; j < S::FN; ++j) label[j] = a.l.labels != nullptr && token0 + 32 * j < a.l.rows ? a.l.labels[token0 + 32 * j] : -1;
  f32x16 acc[S::FM][S::FN] = {};
  product<S, HALF, false, false>(a.l.w, a.l.h, a.l.pairs, (long long)t.m * S::BM, (long long)t.n * S::BN, 0, a.l.width, memory, acc);
  const int slice = a.slice0 + t.m * S::WM + wave % S::WM;
#pragma unroll
  for (int j = 0; j < S::FN; ++j) {
    __builtin_amdgcn_sched_barrier(0);   // (one block of tokens after the other, or all their values want registers at once)
    const int token = token0 + 32 * j;
    const bool live = token < a.l.rows;
    const int hit = label[j] - v;
    float z[S::FM][16];
    logits_of<S>(bias, acc, j, z);
    leave_stats<S::FM>(z, lane, token, live, hit, a.l.vocab - v, (long long)slice * a.l.rows + token, a.part, a.part_u, a.label_logit);
  }
}

// Few tokens: the weights are what has to be read.  A workgroup takes 32 rows of them, its four waves a share of the contraction each; operands go
// from memory to the matrix instructions' registers, as they stand: any type, pitch and alignment.  16 x 16 instructions: four lanes have 64
// bytes of a row in a run, so a load has sixteen pieces to fetch (32 x 32: 64 pieces of 16 bytes, and 1 x 32000 x 4096 bf16 took 56 us).  Which values of the
// contraction an instruction multiplies does not matter as long as both operands agree.
struct FewArgs {
  const void *hidden, *weight;   // weight: from the vocabulary's v0 on
  long long ldh, ldw;
  int rows, values, width;       // values: of the vocabulary in this launch
};
// 32 rows a workgroup for one block of tokens (1 token, 32000 x 4096 bf16: 56 us with the join and the host, 64 rows 63), 64 for more (32 tokens: 82 and 65; 64: 106 and 74).
// (Rows of 16-bit values between two words, shifted together from whole words: 24 tokens, 50257 x 1001 fp16 69 -> 83 us where the weights come from
// memory, 56 -> 50 where they stand in the caches.)
constexpr int kFewWaves = 4;
template <typename T>
using Piece = typename Wide<T>::type;   // 16 bytes of a row
template <typename T>
__device__ inline Piece<T> load_piece(const T* p) { return *reinterpret_cast<const typename Wide<T>::unaligned*>(p); }
template <typename T>
__device__ inline Piece<T> load_piece_end(const T* p, int n) {   // the first n, zeros behind
  Piece<T> v;
#pragma unroll
  for (int j = 0; j < Wide<T>::N; ++j) v[j] = j < n ? p[j] : (T)0.f;
  return v;
}
template <typename T>
__device__ inline f32x4 multiply_piece(Piece<T> a, Piece<T> b, f32x4 c) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  } else if constexpr (std::is_same<T, _Float16>::value) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  } else {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  return c;
}
// 16 R rows of W, a multiple of 32, from v on times 16 FN tokens from token0 on: sums[wave][row][token] of the waves' shares.
template <int R, int FN>
using FewSums = float[kFewWaves][16 * R][16 * FN + 1];
template <typename T, int R, int FN>
__device__ inline void few_products(const FewArgs& a, FewSums<R, FN>& shared, int v, int token0) {
  constexpr int N = Wide<T>::N, STEP = 8 * N;   // of the contraction: 128 bytes of a row, two pieces a lane
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int steps = (a.width + STEP - 1) / STEP, begin = steps * wave / kFewWaves, end = steps * (wave + 1) / kFewWaves;
  const int from = lane / 16 * N;
  const T *w[R], *h[FN];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = v + 16 * r + lane % 16;   // (behind the last: the last once more)
    w[r] = reinterpret_cast<const T*>(a.weight) + (row < a.values ? row : a.values - 1) * a.ldw + from;
  }
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int token = token0 + 16 * j + lane % 16;
    h[j] = reinterpret_cast<const T*>(a.hidden) + (token < a.rows ? token : a.rows - 1) * a.ldh + from;
  }
  f32x4 acc[R][FN] = {};
  const int whole = a.width / STEP < end ? a.width / STEP : end;
  int i = begin;
  constexpr int AHEAD = R * FN < 8 ? 2 : 1;   // steps whose loads are sent for at once
  for (; i + AHEAD <= whole; i += AHEAD) {
    Piece<T> x[2 * AHEAD][R], y[2 * AHEAD][FN];
#pragma unroll
    for (int u = 0; u < 2 * AHEAD; ++u) {
#pragma unroll
      for (int r = 0; r < R; ++r) x[u][r] = load_piece<T>(w[r] + i * STEP + u * 4 * N);
#pragma unroll
      for (int j = 0; j < FN; ++j) y[u][j] = load_piece<T>(h[j] + i * STEP + u * 4 * N);
    }
#pragma unroll
    for (int u = 0; u < 2 * AHEAD; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[r][j] = multiply_piece<T>(x[u][r], y[u][j], acc[r][j]);
  }
  for (; i < end; ++i) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int at = i * STEP + u * 4 * N, n = a.width - at - from;
      Piece<T> x[R], y[FN];
#pragma unroll
      for (int r = 0; r < R; ++r) x[r] = n >= N ? load_piece<T>(w[r] + at) : load_piece_end<T>(w[r] + at, n);
#pragma unroll
      for (int j = 0; j < FN; ++j) y[j] = n >= N ? load_piece<T>(h[j] + at) : load_piece_end<T>(h[j] + at, n);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[r][j] = multiply_piece<T>(x[r], y[j], acc[r][j]);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) shared[wave][16 * r + 4 * (lane / 16) + e][16 * j + lane % 16] = acc[r][j][e];
  __syncthreads();
}
// A wave's 32 rows and 32 tokens: logits as a 32 x 32 block holds them, the vocabulary's from v on.
template <int R, int FN>
__device__ inline void few_logits(const FewSums<R, FN>& shared, int row0, int here, int lane, int v, int vocab, const float* bias, float (&z)[1][16]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int row = row0 + row_of(e, lane), at = v + row_of(e, lane);
    float sum = shared[0][row][here];
#pragma unroll
    for (int p = 1; p < kFewWaves; ++p) sum += shared[p][row][here];
    z[0][e] = at < vocab ? sum + (bias != nullptr ? bias[at] : 0.f) : -__builtin_inff();
  }
}
template <typename T, int R, int FN>
__global__ __launch_bounds__(64 * kFewWaves) void few_stats_kernel(FewArgs a, StatArgs s) {
  __shared__ FewSums<R, FN> shared;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, v = blockIdx.x * (16 * R), token0 = blockIdx.y * (16 * FN);
  few_products<T, R, FN>(a, shared, v, token0);
  constexpr int TOKENS = (16 * FN + 31) / 32;
  for (int block = wave; block < R / 2 * TOKENS; block += kFewWaves) {
    const int row0 = 32 * (block / TOKENS), v32 = v + row0, t32 = 32 * (block % TOKENS) + lane % 32, token = token0 + t32;
    float z[1][16];
    few_logits<R, FN>(shared, row0, t32 < 16 * FN ? t32 : 16 * FN - 1, lane, v32, s.l.vocab, s.l.bias, z);
    const bool live = t32 < 16 * FN && token < a.rows;
    const int hit = live && s.l.labels != nullptr ? s.l.labels[token] - v32 : -1;
    leave_stats<1>(z, lane, token, live, hit, s.l.vocab - v32, (long long)(v32 / 32) * a.rows + token, s.part, s.part_u, s.label_logit);
  }
}
template <typename T>
hipError_t start_few(const FewArgs& a, const StatArgs& s, hipStream_t stream) {
  if (a.rows <= 16) few_stats_kernel<T, 2, 1><<<(unsigned)ceil_div(a.values, 32), 64 * kFewWaves, 0, stream>>>(a, s);
  else if (a.rows <= 32) few_stats_kernel<T, 4, 2><<<(unsigned)ceil_div(a.values, 64), 64 * kFewWaves, 0, stream>>>(a, s);
  else few_stats_kernel<T, 4, 4><<<dim3((unsigned)ceil_div(a.values, 64), (unsigned)ceil_div(a.rows, 64)), 64 * kFewWaves, 0, stream>>>(a, s);
  return hipGetLastError();
}

// Slices joined: `tokens` of them a workgroup, the other threads along the slices.
constexpr int kJoinThreads = 1024;
struct JoinArgs {
  const float2* part;
  const float* part_u;
  const float* label_logit;
  const int32_t* labels;
  int slices, rows, vocab;
  float *logp, *entropy, *stats;
};
struct Sums {
  float top, s, u;
  __device__ inline void add(float t, float x, float y) {   // (exp(-inf) of nothing yet: a top of -inf adds nothing)
    if (t == -__builtin_inff()) {
      s += x;                                               // (0, or a NaN that has no place else)
      return;
    }
    if (t > top) {
      const float d = top - t, f = top == -__builtin_inff() ? 0.f : exp_fast(d);
      u = f > 0.f ? f * (u + s * d) : 0.f;
      s = s * f;                                            // (a NaN stays one)
      top = t;
      s += x;
      u += y;
    } else {
      const float d = t - top, f = exp_fast(d);
      s += f * x;
      u += f > 0.f ? f * (y + x * d) : 0.f;
    }
  }
};
__global__ __launch_bounds__(kJoinThreads) void logit_join_kernel(JoinArgs a, int tokens) {
  __shared__ float shared[3][kJoinThreads];
  const int tid = threadIdx.x, lines = kJoinThreads / tokens, line = tid / tokens;
  const long long token = (long long)blockIdx.x * tokens + tid % tokens;
  const bool live = token < a.rows;
  Sums m = {-__builtin_inff(), 0.f, 0.f};
  if (live) {
#pragma unroll 4
    for (int i = line; i < a.slices; i += lines) {
      const float2 p = a.part[(long long)i * a.rows + token];
      m.add(p.x, p.y, a.part_u != nullptr ? a.part_u[(long long)i * a.rows + token] : 0.f);
    }
  }
  for (int half = lines / 2; half > 0; half /= 2) {
    shared[0][tid] = m.top;
    shared[1][tid] = m.s;
    shared[2][tid] = m.u;
    __syncthreads();
    if (line < half) m.add(shared[0][tid + half * tokens], shared[1][tid + half * tokens], shared[2][tid + half * tokens]);
    __syncthreads();
  }
  if (line != 0 || !live) return;
  const bool empty = m.top == -__builtin_inff() && m.s == 0.f;
  const float log_s = empty ? 0.f : logf(m.s);
  if (a.stats != nullptr) {
    a.stats[2 * token] = m.top;
    a.stats[2 * token + 1] = log_s;
  }
  if (a.entropy != nullptr) a.entropy[token] = empty ? 0.f : log_s - m.u / m.s;
  if (a.logp != nullptr) {
    const int y = a.labels[token];
    float lp = 0.f;
    if (y != -1) {
      if (y < 0 || y >= a.vocab) lp = __builtin_nanf("");
      else if (empty) lp = -__builtin_inff();
      else lp = (a.label_logit[token] - m.top) - log_s;
    }
    a.logp[token] = lp;
  }
}

// ---- operands

// bf16 pieces of a float32, x = h + m + l up to 2^-25 of it.  No finite value becomes infinite; what is not finite has no remainder.
__device__ inline void pieces_of(float x, u16 (&p)[3]) {
  const bool finite = fabsf(x) < __builtin_inff();
  float h = (float)(__bf16)x;
  if (finite && !(fabsf(h) < __builtin_inff())) h = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  const float r = finite ? x - h : 0.f, m = (float)(__bf16)r;
  p[0] = (u16)(__float_as_uint(h) >> 16);
  p[1] = (u16)(__float_as_uint(m) >> 16);
  p[2] = __builtin_bit_cast(u16, (__bf16)(r - m));
}
// Rows on 16 bytes, a multiple of eight columns, zeros behind the last: a copy of 16-bit values or a float32's pieces, eight a thread.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T* x, long long ldx, int rows, int width, int padded, u16* out, long long plane) {
  const long long chunks = padded / 8, all = chunks * rows;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
    const long long row = i / chunks;
    const int col = (int)(i % chunks) * 8;
    const T* from = x + row * ldx + col;
    u16* to = out + row * padded + col;
    if constexpr (sizeof(T) == 2) {
      u16 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = col + j < width ? from[j] : (u16)0;
      s16x8 raw;
#pragma unroll
      for (int j = 0; j < 8; ++j) raw[j] = (short)v[j];
      *reinterpret_cast<s16x8*>(to) = raw;
    } else {
      s16x8 raw[3];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        u16 p[3];
        pieces_of(col + j < width ? (float)from[j] : 0.f, p);
#pragma unroll
        for (int q = 0; q < 3; ++q) raw[q][j] = (short)p[q];
      }
#pragma unroll
      for (int q = 0; q < 3; ++q) *reinterpret_cast<s16x8*>(to + q * plane) = raw[q];
    }
  }
}

// Whether a matrix can be read as it stands: 16-byte pieces of 16-bit values.
bool as_it_is(const void* p, long long ld, int dtype, int width) {
  return dtype != ZENO_F32 && width % 8 == 0 && ld % 8 == 0 && ld < kMostPitch && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}
hipError_t pack(const void* x, long long ldx, int dtype, int rows, int width, u16* out, hipStream_t stream) {
  const int padded = padded_width(width);
  const long long plane = (long long)rows * padded, threads = plane / 8;
  const unsigned blocks = (unsigned)std::min<long long>((threads + 255) / 256, 16384);
  if (dtype == ZENO_F32)
    pack_kernel<float><<<blocks, 256, 0, stream>>>(reinterpret_cast<const float*>(x), ldx, rows, width, padded, out, plane);
  else
    pack_kernel<u16><<<blocks, 256, 0, stream>>>(reinterpret_cast<const u16*>(x), ldx, rows, width, padded, out, plane);
  return hipGetLastError();
}
Pairs pairs_of(int a, int b) {   // planes of the two sides: three and three, two and one, one and one
  if (a == 3 && b == 3) return {6, 0x001102, 0x010120};
  if (a == 2) return {2, 0x01, 0x00};
  return {1, 0, 0};
}

// ---- backward

static_assert(WideTile::BM == kWideSide && WideTile::WM == 2 && MidTile::BM == kTileSide && ThirdTile::BM == kTileSide &&
                  ThirdTile::WM == 2,
              "as the plans have it");
__device__ inline float power_of_two(int k) { return __uint_as_float((unsigned)(127 + k) << 23); }   // k from -126 to 127
// dz is formed within 2^14, from gradients times a power of two: that of the largest, |dz| <= |g| + 22 |q| (p |log p| <= 1/e, p H <= ln V < 21).  In 16 bits, which
// hold dz as it is formed, the largest of a worker; one workgroup a worker: another's gradients, or those of nobody, do not show.  float32's pieces have its range and hold dz
// itself: a token's own.  Powers from -119 (the largest finite g and q) to 126 are float32's own, and so are their inverses.  `clear`: a worker's n words to set to zero on
// the way.
struct ScaleArgs {
  const float *g, *q;
  const int32_t *labels, *offsets;
  int rows;
  bool own;              // each token its own
  int* power;            // [m]
  float* up;             // [rows] 2^power
  unsigned* clear;
  int n;
};
// Of a 32nd of the largest, which no finite gradients take beyond float32.
__device__ inline int grad_power(float largest) {
  const int e = (int)((__float_as_uint(largest) >> 23) & 255) - 126 + 5;   // 32 largest < 2^e
  return 14 - e < 126 ? 14 - e : 126;
}
__global__ __launch_bounds__(1024) void grad_scale_kernel(ScaleArgs a) {
  __shared__ float shared[16];
  __shared__ int all;
  const int worker = blockIdx.x, begin = group_offset(a.offsets, worker, a.rows), end = group_offset(a.offsets, worker + 1, a.rows);
  auto size_of = [&](int t) {
    float b = a.g != nullptr && a.labels[t] != -1 ? fabsf(a.g[t]) * 0.03125f : 0.f;
    if (a.q != nullptr) b += 0.6875f * fabsf(a.q[t]);
    return b;
  };
  float largest = 0.f;
  for (int i = threadIdx.x; i < a.n; i += 1024) a.clear[(long long)worker * a.n + i] = 0;
  for (int t = begin + threadIdx.x; t < end; t += 1024) {
    const float b = size_of(t);
    if (a.own) a.up[t] = power_of_two(grad_power(b));
    else if (b < __builtin_inff()) largest = fmaxf(largest, b);
  }
  if (a.own) return;
  largest = wave_max_f(largest);
  if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = largest;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) largest = fmaxf(largest, shared[w]);
    all = grad_power(largest);
    a.power[worker] = all;
  }
  __syncthreads();
  const float up = power_of_two(all);
  for (int t = begin + threadIdx.x; t < end; t += 1024) a.up[t] = up;
}

// bf16 hidden states as fp16, each column of a worker times the power of two that brings its largest finite value to 2^14 .. 2^15: exact down to 2^-32
// of that value.
__device__ inline int column_power(unsigned largest) {   // largest magnitude, as float32 bits
  if (largest == 0) return 0;
  const int up = 14 + 127 - (int)(largest >> 23);
  return up > 126 ? 126 : up;                            // (not below 14 + 127 - 254)
}
__host__ __device__ inline int padded_stride(int width) { return (width + 7) / 8 * 8; }
constexpr int kColumnRows = 256;   // of a workgroup
struct ColumnArgs {
  Side h;
  int width, m, rows;
  const int32_t* offsets;
  unsigned* largest;     // [m][width]
  u16* out;
};
// The worker of a row (of one that belongs to somebody): the last that begins there or before.
__device__ inline int worker_of(const int32_t* offsets, int m, int row) {
  if (offsets == nullptr) return 0;
  int lo = 0, hi = m;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (offsets[mid] <= row) lo = mid;
    else hi = mid;
  }
  return lo;
}
__global__ __launch_bounds__(1024) void column_max_kernel(ColumnArgs a) {
  __shared__ unsigned shared[16][512];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = blockIdx.x * 512 + lane * 8;
  const int from = group_offset(a.offsets, 0, a.rows), until = group_offset(a.offsets, a.offsets == nullptr ? 1 : a.m, a.rows);
  const int begin = max((int)blockIdx.y * kColumnRows, from), end = min((int)(blockIdx.y + 1) * kColumnRows, until);
  if (begin >= end) return;
  const int first = worker_of(a.offsets, a.m, begin), last = worker_of(a.offsets, a.m, end - 1);
  for (int g = first; g <= last; ++g) {   // (most often one)
    const int lo = max(begin, group_offset(a.offsets, g, a.rows)), hi = min(end, group_offset(a.offsets, g + 1, a.rows));
    unsigned m[8] = {};
    if (col < a.width) {
#pragma unroll 4
      for (int row = lo + wave; row < hi; row += 16) {
        const s16x8 raw = *reinterpret_cast<const s16x8*>(a.h.p + row * a.h.ld + col);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const unsigned v = (unsigned)raw[j] & 0x7fff;
          m[j] = v < 0x7f80 && v > m[j] ? v : m[j];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) shared[wave][8 * lane + j] = m[j];
    __syncthreads();
    if (threadIdx.x < 512) {
      unsigned most = 0;
      for (int w = 0; w < 16; ++w) most = shared[w][threadIdx.x] > most ? shared[w][threadIdx.x] : most;
      const int c = blockIdx.x * 512 + threadIdx.x;
      if (most != 0 && c < a.width) atomicMax(&a.largest[(long long)g * a.width + c], most << 16);
    }
    __syncthreads();
  }
}
__global__ __launch_bounds__(1024) void column_half_kernel(ColumnArgs a) {
  const int col = (blockIdx.x * 64 + threadIdx.x % 64) * 8;
  const int from = group_offset(a.offsets, 0, a.rows), until = group_offset(a.offsets, a.offsets == nullptr ? 1 : a.m, a.rows);
  const int begin = max((int)blockIdx.y * kColumnRows, from), end = min((int)(blockIdx.y + 1) * kColumnRows, until);
  if (col >= a.width || begin >= end) return;
  const int first = worker_of(a.offsets, a.m, begin), last = worker_of(a.offsets, a.m, end - 1);
  for (int g = first; g <= last; ++g) {
    const int lo = max(begin, group_offset(a.offsets, g, a.rows)), hi = min(end, group_offset(a.offsets, g + 1, a.rows));
    float up[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) up[j] = power_of_two(column_power(col + j < a.width ? a.largest[(long long)g * a.width + col + j] : 0));
#pragma unroll 4
    for (int row = lo + threadIdx.x / 64; row < hi; row += 16) {
      const s16x8 raw = *reinterpret_cast<const s16x8*>(a.h.p + row * a.h.ld + col);
      s16x8 half;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const short bits = raw[j];
        half[j] = __builtin_bit_cast(short, (_Float16)(__uint_as_float((unsigned)(u16)bits << 16) * up[j]));
      }
      *reinterpret_cast<s16x8*>(a.out + (long long)row * padded_stride(a.width) + col) = half;
    }
  }
}

struct DzArgs {
  LogitArgs l;
  const float *stats, *grad_logp, *entropy, *grad_entropy;
  const float* up;       // [rows]
  u16* dz;               // [planes][rows][ldz]
  long long ldz, plane;
};
// Planes of dz.
enum Planes { kBf16Three, kBf16TwoHalfTwo, kHalfTwo };   // three bf16 pieces; two bf16 pieces, and two fp16 pieces; two fp16 pieces
__host__ __device__ constexpr int count_of(Planes p) { return p == kHalfTwo ? 2 : (p == kBf16Three ? 3 : 4); }
__host__ __device__ constexpr int sums_of(Planes p) { return p == kBf16TwoHalfTwo ? 2 : 1; }   // each is dz
// A token, as far as its gradients need it.
struct TokenGrad {
  float M, log_s;        // of its logits
  float g, q, H;         // gradients of its log probability and of its entropy, both times `up`; its entropy
  int y;                 // its label, -1: none
  float up;              // what its gradients are multiplied by
};
__device__ inline TokenGrad token_grad(const DzArgs& a, int token) {
  TokenGrad t = {-__builtin_inff(), 0.f, 0.f, 0.f, 0.f, -1, 1.f};   // behind the last: no distribution
  if (token < a.l.rows) {
    t.M = a.stats[2 * token];
    t.log_s = a.stats[2 * token + 1];
    t.up = a.up[token];
    if (a.grad_logp != nullptr) {
      t.y = a.l.labels[token];
      t.g = a.grad_logp[token] * t.up;
    }
    if (a.grad_entropy != nullptr) {
      t.q = a.grad_entropy[token] * t.up;
      t.H = a.entropy[token];
    }
  }
  return t;
}
// dz, scaled in 16-bit types, in the place of a lane's share of FM blocks of logits from v on.  The label's is -g expm1(log p), which keeps what is left of a
// token that is nearly certain.
template <int FM, Planes P>
__device__ inline void logit_grads(float (&z)[FM][16], int lane, TokenGrad t, bool with_entropy, int v, int vocab) {
  const float back = P == kBf16Three ? 1.f / t.up : 1.f;   // (a power of two)
  const bool empty = t.M == -__builtin_inff() && t.log_s == 0.f;
  const float g = t.y == -1 ? 0.f : (t.y >= 0 && t.y < vocab ? t.g : __builtin_nanf(""));
  const float M = empty ? 0.f : t.M, log_s = empty ? __builtin_inff() : t.log_s;   // (empty: every probability is 0)
  const int place = t.y < vocab ? place_in<FM>(t.y - v, lane) : -1;
  const bool any = __any(place >= 0);
  const float own = any ? value_at<FM>(z, place) : 0.f;
  if (with_entropy) {
    const float base = fmaf(t.q, t.H, g);
#pragma unroll
    for (int r = 0; r < FM; ++r)
#pragma unroll
      for (int e = 0; e < 16; ++e) {   // (where p is 0, its logarithm is cut off: 0 * -inf would be NaN)
        const float lp = (z[r][e] - M) - log_s;
        z[r][e] = -exp_fast(lp) * fmaf(t.q, fmaxf(lp, -256.f), base) * back;
      }
  } else {
    const float base = -g * back;
#pragma unroll
    for (int r = 0; r < FM; ++r)
#pragma unroll
      for (int e = 0; e < 16; ++e) z[r][e] = exp_fast((z[r][e] - M) - log_s) * base;
  }
  if (any) {
    const float lp = (own - M) - log_s;
    float d = -g * expm1f(lp);
    if (with_entropy) d -= exp_fast(lp) * (t.q * (fmaxf(lp, -256.f) + t.H));
    d = empty ? 0.f : d * back;
    put_at<FM>(z, place, d);
  }
}
// Four values as the planes of sum `sum`.
template <Planes P>
constexpr int kPlanesOfSum = count_of(P) / sums_of(P);
template <Planes P>
__device__ inline void planes_of_dz(const float* from, int sum, s16x4 (&out)[kPlanesOfSum<P>]) {
  const bool half = P == kHalfTwo || sum == 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float d = from[i];
#pragma unroll
    for (int plane = 0; plane < kPlanesOfSum<P>; ++plane) {
      if (half) {
        const _Float16 x = (_Float16)d;
        out[plane][i] = __builtin_bit_cast(short, x);
        d -= (float)x;
      } else {
        const __bf16 x = (__bf16)d;
        out[plane][i] = __builtin_bit_cast(short, x);
        d -= (float)x;
      }
    }
  }
}
template <typename S, bool HALF, Planes P>
__global__ __launch_bounds__(S::THREADS, S::GROUPS) void logit_grad_kernel(DzArgs a) {
  extern __shared__ __align__(1024) unsigned char memory[];
  const Place t = place_of(blockIdx.x, a.l.tiles_m, a.l.tiles_n);
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int wm = (wave % S::WM) * (32 * S::FM), wn = (wave / S::WM) * (32 * S::FN), v = a.l.v0 + t.m * S::BM + wm;
  Bias<S> bias;   // (these arrive beside the operands)
  load_bias<S>(a.l, v, lane, bias);
  TokenGrad token[S::FN];
#pragma unroll
  for (int j = 0; j < S::FN; ++j)
    token[j] = token_grad(a, t.n * S::BN + wn + 32 * j + lane % 32);
  f32x16 acc[S::FM][S::FN] = {};
  product<S, HALF, false, false>(a.l.w, a.l.h, a.l.pairs, (long long)t.m * S::BM, (long long)t.n * S::BN, 0, a.l.width, memory, acc);
#pragma unroll
  for (int j = 0; j < S::FN; ++j) {
    __builtin_amdgcn_sched_barrier(0);   // (one block of tokens after the other, or all their values want registers at once)
    float z[S::FM][16];
    logits_of<S>(bias, acc, j, z);
    logit_grads<S::FM, P>(z, lane, token[j], a.grad_entropy != nullptr, v, a.l.vocab);
    // this block of every wave's tokens through LDS, so that rows leave in whole lines; one sum's planes after the other's
    u16* tile = reinterpret_cast<u16*>(memory);
    constexpr int TOKENS = 32 * S::WN, PLANE = TOKENS * S::PITCH, COUNT = kPlanesOfSum<P>;
    static_assert(COUNT <= S::DZ_PLANES, "what there is");
#pragma unroll
    for (int sum = 0; sum < sums_of(P); ++sum) {
      if (j > 0 || sum > 0) __syncthreads();
#pragma unroll
      for (int r = 0; r < S::FM; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s16x4 out[COUNT];
          planes_of_dz<P>(z[r] + 4 * c, sum, out);
          u16* to = tile + (32 * (wave / S::WM) + lane % 32) * S::PITCH + wm + 32 * r + row_of(4 * c, lane);
#pragma unroll
          for (int plane = 0; plane < COUNT; ++plane) *reinterpret_cast<s16x4*>(to + plane * PLANE) = out[plane];
        }
      __syncthreads();
      constexpr int CHUNKS = S::BM / 8;
#pragma unroll 4
      for (int i = threadIdx.x; i < COUNT * TOKENS * CHUNKS; i += S::THREADS) {
        const int plane = i / (TOKENS * CHUNKS), row = i / CHUNKS % TOKENS, col = i % CHUNKS * 8;
        const long long to = (long long)t.n * S::BN + row / 32 * (32 * S::FN) + 32 * j + row % 32;
        if (to < a.l.rows)
          *reinterpret_cast<s16x8*>(a.dz + (sum * COUNT + plane) * a.plane + to * a.ldz + t.m * S::BM + col) =
              *reinterpret_cast<const s16x8*>(tile + plane * PLANE + row * S::PITCH + col);
      }
    }
  }
}

// The same of few tokens: the logits have to be the forward pass's to the bit, or a nearly certain token's gradient is the difference of two roundings.
template <typename T, int R, int FN, Planes P>
__global__ __launch_bounds__(64 * kFewWaves) void few_grad_kernel(FewArgs a, DzArgs d) {
  __shared__ FewSums<R, FN> shared;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, v = blockIdx.x * (16 * R), token0 = blockIdx.y * (16 * FN);
  few_products<T, R, FN>(a, shared, v, token0);
  constexpr int TOKENS = (16 * FN + 31) / 32;
  for (int block = wave; block < R / 2 * TOKENS; block += kFewWaves) {
    const int row0 = 32 * (block / TOKENS), t32 = 32 * (block % TOKENS) + lane % 32, token = t32 < 16 * FN ? token0 + t32 : a.rows;
    float z[1][16];
    few_logits<R, FN>(shared, row0, t32 < 16 * FN ? t32 : 16 * FN - 1, lane, d.l.v0 + v + row0, d.l.vocab, d.l.bias, z);
    logit_grads<1, P>(z, lane, token_grad(d, token), d.grad_entropy != nullptr, d.l.v0 + v + row0, d.l.vocab);
    if (token >= a.rows) continue;
    constexpr int COUNT = kPlanesOfSum<P>;
#pragma unroll
    for (int sum = 0; sum < sums_of(P); ++sum)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s16x4 out[COUNT];
        planes_of_dz<P>(z[0] + 4 * c, sum, out);
#pragma unroll
        for (int plane = 0; plane < COUNT; ++plane)
          *reinterpret_cast<s16x4*>(d.dz + (sum * COUNT + plane) * d.plane + token * d.ldz + v + row0 + row_of(4 * c, lane)) = out[plane];
      }
  }
}
template <typename T, Planes P>
hipError_t start_few_dz(const FewArgs& a, const DzArgs& d, hipStream_t stream) {
  if (a.rows <= 16) few_grad_kernel<T, 2, 1, P><<<(unsigned)ceil_div(a.values, 32), 64 * kFewWaves, 0, stream>>>(a, d);
  else if (a.rows <= 32) few_grad_kernel<T, 4, 2, P><<<(unsigned)ceil_div(a.values, 64), 64 * kFewWaves, 0, stream>>>(a, d);
  else few_grad_kernel<T, 4, 4, P><<<dim3((unsigned)ceil_div(a.values, 64), (unsigned)ceil_div(a.rows, 64)), 64 * kFewWaves, 0, stream>>>(a, d);
  return hipGetLastError();
}

// dh: a piece of the vocabulary, cut into `splits` of `per` values that different workgroups sum, each into its own slot.
struct HiddenArgs {
  Side dz, w;
  Pairs pairs;           // of PLANES 1
  int tiles_m, tiles_n, rows, width, length, per;
  int first;             // the slots hold nothing yet
  float* slots;          // [splits][rows][width]
};
template <typename S, bool HALF, int PLANES>
__global__ __launch_bounds__(S::THREADS, S::GROUPS) void hidden_grad_kernel(HiddenArgs a) {
  extern __shared__ __align__(1024) unsigned char memory[];
  const Place t = place_of(blockIdx.x, a.tiles_m, a.tiles_n);
  const int begin = blockIdx.y * a.per, length = a.length - begin < a.per ? a.length - begin : a.per;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int row0 = t.m * S::BM + (wave % S::WM) * (32 * S::FM), col0 = t.n * S::BN + (wave / S::WM) * (32 * S::FN) + lane % 32;
  float* slot = a.slots + (long long)blockIdx.y * a.rows * a.width;
  f32x16 acc[S::FM][S::FN] = {}, none[S::FM / S::WN];
  product<S, HALF, false, true, PLANES, false>(a.dz, a.w, a.pairs, (long long)t.m * S::BM, (long long)t.n * S::BN, begin, length > 0 ? length : 0,
                                               memory, acc, none);
#pragma unroll
  for (int r = 0; r < S::FM; ++r)
#pragma unroll
    for (int j = 0; j < S::FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int row = row0 + 32 * r + row_of(e, lane), col = col0 + 32 * j;
        if (row >= a.rows || col >= a.width) continue;
        // One workgroup adds one value of a launch, so the order is that of the launches; nothing is waited for.  (Sums that go on from what the
        // slot holds 600 us a piece of 8192 x 8192 x 4096 with one plane of dz, loaded behind the products 684, stored 500.)
        float* to = slot + (long long)row * a.width + col;
        if (a.first) *to = acc[r][j][e];
        else unsafeAtomicAdd(to, acc[r][j][e]);
      }
}
// Slots in their order, for the rows that belong to somebody.
struct HiddenJoinArgs {
  const float* slots;
  int splits, rows, width, m;
  const int32_t* offsets;
  const float* up;       // [rows] or nullptr
  void* out;
  long long ldo;
};
template <typename T>
__global__ __launch_bounds__(256) void hidden_join_kernel(HiddenJoinArgs a) {
  const int lo = group_offset(a.offsets, 0, a.rows), hi = group_offset(a.offsets, a.offsets == nullptr ? 1 : a.m, a.rows);
  const long long stride = (long long)a.rows * a.width;
  for (int row = lo + blockIdx.y; row < hi; row += gridDim.y) {
    const float down = a.up != nullptr ? 1.f / a.up[row] : 1.f;   // (a power of two: exact)
    const float* from = a.slots + (long long)row * a.width;
    T* to = reinterpret_cast<T*>(a.out) + row * a.ldo;
    const int whole = a.width / 4 * 4;
    for (int col = (blockIdx.x * 256 + threadIdx.x) * 4; col < a.width; col += gridDim.x * 1024) {
      if (col < whole) {
        f32x4 sum = *reinterpret_cast<const f32x4_a4*>(from + col);
        for (int s = 1; s < a.splits; ++s) sum += *reinterpret_cast<const f32x4_a4*>(from + s * stride + col);
        typedef T t4 __attribute__((ext_vector_type(4)));
        typedef t4 unaligned __attribute__((aligned(sizeof(T))));
        t4 out;
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = (T)(sum[i] * down);
        *reinterpret_cast<unaligned*>(to + col) = out;
      } else {
        for (int i = col; i < a.width; ++i) {
          float sum = from[i];
          for (int s = 1; s < a.splits; ++s) sum += from[s * stride + i];
          to[i] = (T)(sum * down);
        }
      }
    }
  }
}

// dW of a piece of the vocabulary, a group's tokens from its offset on.
struct WeightArgs {
  Side dz, h;
  Pairs pairs;
  int tiles_m, tiles_n, rows, width, values;   // values: of the vocabulary in this piece
  const int32_t* offsets;
  const int* power;          // [m] of two that dz has been multiplied by, or nullptr
  const unsigned* columns;   // largest values of the columns of h that have been scaled by column_power(), or nullptr
  float *dweight, *dbias;   // at the piece's first value, or in slots; each may be nullptr
  long long ldw, ldb;
  int parts;                // of a group's tokens, that different workgroups sum
  long long slot;           // between two parts' sums
};
template <typename S, bool HALF>
__global__ __launch_bounds__(S::THREADS, S::GROUPS) void head_weight_grad_kernel(WeightArgs a) {
  extern __shared__ __align__(1024) unsigned char memory[];
  const Place t = place_of(blockIdx.x, a.tiles_m, a.tiles_n);
  const int g = blockIdx.y, lo = group_offset(a.offsets, g, a.rows), hi = group_offset(a.offsets, g + 1, a.rows);
  const int per = hi > lo ? ((hi - lo + a.parts - 1) / a.parts + kStep - 1) / kStep * kStep : 0, part = blockIdx.z;
  const int begin = min(lo + (long long)part * per, (long long)hi), end = min((long long)begin + per, (long long)hi);
  f32x16 acc[S::FM][S::FN] = {};
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, length = end > begin ? end - begin : 0;
  const int row0 = t.m * S::BM + (wave % S::WM) * (32 * S::FM), col0 = t.n * S::BN + (wave / S::WM) * (32 * S::FN) + lane % 32;
  const int down = HALF ? -a.power[g] : 0;
  if (a.dbias != nullptr && t.n == 0) {
    f32x16 sums[S::FM / S::WN] = {};
    product<S, HALF, true, true, HALF ? 2 : 1, true>(a.dz, a.h, a.pairs, (long long)t.m * S::BM, 0, begin, length, memory, acc, sums);
    if (lane % 32 == 0) {
#pragma unroll
      for (int r = 0; r < S::FM / S::WN; ++r)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int row = row0 + 32 * (S::WN * r + wave / S::WM) + row_of(e, lane);
          if (row < a.values) a.dbias[g * a.ldb + part * a.slot + row] = ldexpf(sums[r][e], down);
        }
    }
  } else {
    f32x16 none[S::FM / S::WN];
    product<S, HALF, true, true, HALF ? 2 : 1, false>(a.dz, a.h, a.pairs, (long long)t.m * S::BM, (long long)t.n * S::BN, begin, length, memory, acc, none);
  }
  if (a.dweight == nullptr) return;
  float* dw = a.dweight + g * a.ldw + part * a.slot;
  // Gradients are read when all layers have theirs: where rows are whole memory lines they go past the caches.
  const bool past = t.m * S::BM + S::BM <= a.values && t.n * S::BN + S::BN <= a.width && a.width % 32 == 0 && on_line(dw);
#pragma unroll
  for (int j = 0; j < S::FN; ++j) {
    const int col = col0 + 32 * j;
    const int back = HALF && a.columns != nullptr && col < a.width ? down - column_power(a.columns[(long long)g * a.width + col]) : down;   // (one step: in between it may leave float32's range)
    float* to = dw + (long long)row0 * a.width + col;
    if (past) {
#pragma unroll
      for (int r = 0; r < S::FM; ++r)
#pragma unroll
        for (int e = 0; e < 16; ++e) __builtin_nontemporal_store(HALF ? ldexpf(acc[r][j][e], back) : acc[r][j][e], to + (long long)(32 * r + row_of(e, lane)) * a.width);
      keep_apart();
    } else if (col < a.width) {
#pragma unroll
      for (int r = 0; r < S::FM; ++r)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (row0 + 32 * r + row_of(e, lane) < a.values) to[(long long)(32 * r + row_of(e, lane)) * a.width] = HALF ? ldexpf(acc[r][j][e], back) : acc[r][j][e];
    }
  }
}

// Parts in their order.
struct WeightJoinArgs {
  const float *dweight, *dbias;   // slots: parts `slot` apart, groups `group` apart
  long long slot, group, n;       // n: weights of a group in this piece
  int parts, values;
  float *out_w, *out_b;
  long long ldw, ldb;
};
__global__ __launch_bounds__(256) void weight_join_kernel(WeightJoinArgs a) {
  const long long all = (a.out_w != nullptr ? a.n : 0) + (a.out_b != nullptr ? a.values : 0), g = blockIdx.y;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
    const bool weights = a.out_w != nullptr && i < a.n;
    const long long at = weights ? i : i - (a.out_w != nullptr ? a.n : 0);
    const float* from = (weights ? a.dweight : a.dbias) + g * a.group + at;
    float sum = from[0];
#pragma unroll 8
    for (int part = 1; part < a.parts; ++part) sum += from[part * a.slot];
    (weights ? a.out_w + g * a.ldw : a.out_b + g * a.ldb)[at] = sum;
  }
}

// ---- launches

hipError_t allow(const void* kernel, int lds) { return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds); }

template <typename S, bool HALF>
hipError_t start_stats(const StatArgs& a, hipStream_t stream) {
  const auto kernel = logit_stats_kernel<S, HALF>;
  constexpr int lds = S::template LDS<1>;
  const hipError_t e = allow(reinterpret_cast<const void*>(kernel), lds);
  if (e != hipSuccess) return e;
  kernel<<<(unsigned)a.l.tiles_m * a.l.tiles_n, S::THREADS, lds, stream>>>(a);
  return hipGetLastError();
}
template <typename S, bool HALF, Planes P>
hipError_t start_dz(const DzArgs& a, hipStream_t stream) {
  const auto kernel = logit_grad_kernel<S, HALF, P>;
  constexpr int lds = std::max(S::template LDS<1>, S::DZ);
  const hipError_t e = allow(reinterpret_cast<const void*>(kernel), lds);
  if (e != hipSuccess) return e;
  kernel<<<(unsigned)a.l.tiles_m * a.l.tiles_n, S::THREADS, lds, stream>>>(a);
  return hipGetLastError();
}
template <typename S>
hipError_t start_dz(const DzArgs& a, int dtype, hipStream_t stream) {
  if (dtype == ZENO_F32) return start_dz<S, false, kBf16Three>(a, stream);
  return dtype == ZENO_F16 ? start_dz<S, true, kHalfTwo>(a, stream) : start_dz<S, false, kBf16TwoHalfTwo>(a, stream);
}
template <typename S, bool HALF, int PLANES>
hipError_t start_hidden(const HiddenArgs& a, int splits, hipStream_t stream) {
  const auto kernel = hidden_grad_kernel<S, HALF, PLANES>;
  constexpr int lds = S::template LDS<PLANES>;
  const hipError_t e = allow(reinterpret_cast<const void*>(kernel), lds);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)a.tiles_m * a.tiles_n, splits), S::THREADS, lds, stream>>>(a);
  return hipGetLastError();
}
template <typename S>
hipError_t start_hidden(const HiddenArgs& a, int dtype, int splits, hipStream_t stream) {
  if (dtype == ZENO_F32) return start_hidden<S, false, 1>(a, splits, stream);
  return dtype == ZENO_F16 ? start_hidden<S, true, 2>(a, splits, stream) : start_hidden<S, false, 2>(a, splits, stream);
}
template <typename S, bool HALF>
hipError_t start_weight(const WeightArgs& a, int m, hipStream_t stream) {
  const auto kernel = head_weight_grad_kernel<S, HALF>;
  constexpr int lds = S::template LDS<(HALF ? 2 : 1)>;
  const hipError_t e = allow(reinterpret_cast<const void*>(kernel), lds);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)a.tiles_m * a.tiles_n, m, a.parts), S::THREADS, lds, stream>>>(a);
  return hipGetLastError();
}

#define ZENO_STEP(expr)                          \
  do {                                           \
    const hipError_t zeno_step_error = (expr);   \
    if (zeno_step_error != hipSuccess) return zeno_step_error; \
  } while (0)

// The side of a matrix of `rows` rows: as it stands, or packed into `space`.
hipError_t side_of(const void* x, long long ld, int dtype, int rows, int width, u16* space, Side& s, hipStream_t stream) {
  s.extent = rows;
  if (as_it_is(x, ld, dtype, width)) {
    s.p = reinterpret_cast<const u16*>(x);
    s.ld = ld;
    s.plane = 0;
    return hipSuccess;
  }
  s.p = space;
  s.ld = padded_width(width);
  s.plane = (long long)rows * s.ld;
  return pack(x, ld, dtype, rows, width, space, stream);
}

}  // namespace

size_t linear_logprobs_workspace_bytes(int rows, int vocab, int width, int dtype) { return forward_plan(std::max(rows, 1), vocab, width, dtype).bytes; }

hipError_t launch_linear_logprobs(const LinearLogprobsArgs& a, void* workspace, hipStream_t stream) {
  const ForwardPlan p = forward_plan(a.rows, a.vocab, a.width, a.dtype);
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  const size_t bytes = a.dtype == ZENO_F32 ? 4 : 2;
  auto join = [&](const StatArgs& s, int t0, int rows, int slices) {
    const JoinArgs j = {s.part, s.part_u, s.label_logit, a.labels == nullptr ? nullptr : a.labels + t0, slices, rows, a.vocab,
                        a.logp == nullptr ? nullptr : a.logp + t0, a.entropy == nullptr ? nullptr : a.entropy + t0,
                        a.stats == nullptr ? nullptr : a.stats + 2 * (size_t)t0};
    int tokens = 1;   // a workgroup for every compute unit, up to whole memory lines
    while (tokens < 64 && rows / (2 * tokens) >= 256) tokens *= 2;
    logit_join_kernel<<<(unsigned)ceil_div(rows, tokens), kJoinThreads, 0, stream>>>(j, tokens);
    return hipGetLastError();
  };
  StatArgs s = {};
  s.part = reinterpret_cast<float2*>(ws + p.part);
  s.part_u = a.entropy != nullptr ? reinterpret_cast<float*>(ws + p.part_u) : nullptr;
  s.label_logit = reinterpret_cast<float*>(ws + p.label);
  if (p.few) {
    const FewArgs f = {a.hidden, a.weight, a.ldh, a.ldw, a.rows, a.vocab, a.width};
    s.l.vocab = a.vocab;
    s.l.bias = a.bias;
    s.l.labels = a.labels;
    ZENO_STEP(a.dtype == ZENO_F32 ? start_few<float>(f, s, stream) : a.dtype == ZENO_BF16 ? start_few<__bf16>(f, s, stream) : start_few<_Float16>(f, s, stream));
    return join(s, 0, a.rows, a.rows <= 16 ? ceil_div(a.vocab, 32) : ceil_div(a.vocab, 64) * 2);   // (what the workgroups have left)
  }
  const bool half = a.dtype == ZENO_F16, direct = as_it_is(a.weight, a.ldw, a.dtype, a.width);
  const int piece = direct ? a.vocab : p.piece;
  for (int t0 = 0; t0 < a.rows; t0 += p.block) {
    const int rows = std::min(p.block, a.rows - t0);
    LogitArgs& l = s.l;
    ZENO_STEP(side_of(reinterpret_cast<const unsigned char*>(a.hidden) + (size_t)t0 * a.ldh * bytes, a.ldh, a.dtype, rows, a.width,
                      reinterpret_cast<u16*>(ws + p.hidden), l.h, stream));
    l.pairs = pairs_of(planes_of(a.dtype), planes_of(a.dtype));
    l.width = padded_width(a.width);
    l.vocab = a.vocab;
    l.rows = rows;
    l.bias = a.bias;
    l.labels = a.labels == nullptr ? nullptr : a.labels + t0;
    int slices = 0;
    for (int v0 = 0; v0 < a.vocab; v0 += piece) {
      const int values = std::min(piece, a.vocab - v0);
      ZENO_STEP(side_of(reinterpret_cast<const unsigned char*>(a.weight) + (size_t)v0 * a.ldw * bytes, a.ldw, a.dtype, values, a.width,
                        reinterpret_cast<u16*>(ws + p.weight), l.w, stream));
      l.v0 = v0;
      s.slice0 = v0 / p.slice;
      const int side = p.wide ? kWideSide : kTileSide;
      l.tiles_m = ceil_div(values, side);
      l.tiles_n = ceil_div(rows, side);
      if (p.wide) ZENO_STEP(half ? (start_stats<WideTile, true>(s, stream)) : (start_stats<WideTile, false>(s, stream)));
      else ZENO_STEP(half ? (start_stats<ThirdTile, true>(s, stream)) : (start_stats<ThirdTile, false>(s, stream)));
      slices = s.slice0 + l.tiles_m * 2;
    }
    ZENO_STEP(join(s, t0, rows, slices));
  }
  return hipSuccess;
}

size_t linear_logprobs_backward_workspace_bytes(int rows, int vocab, int width, int dtype, int m) {
  return backward_plan(rows, vocab, width, dtype, m).bytes;
}

hipError_t launch_linear_logprobs_backward(const LinearLogprobsGradArgs& a, void* workspace, hipStream_t stream) {
  const BackwardPlan p = backward_plan(a.rows, a.vocab, a.width, a.dtype, a.m);
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  const size_t bytes = a.dtype == ZENO_F32 ? 4 : 2;
  const bool half = a.dtype == ZENO_F16, direct = as_it_is(a.weight, a.ldw, a.dtype, a.width);
  const int planes = planes_of(a.dtype);
  int* power = reinterpret_cast<int*>(ws + p.power);
  const bool convert = a.dtype == ZENO_BF16 && (a.dweight != nullptr || a.dbias != nullptr) && a.rows > 0;
  unsigned* columns = reinterpret_cast<unsigned*>(ws + p.columns);
  float* up = reinterpret_cast<float*>(ws + p.up);
  const ScaleArgs sc = {a.grad_logp, a.grad_entropy, a.labels, a.offsets, a.rows, planes == 3, power, up, columns, convert ? a.width : 0};
  grad_scale_kernel<<<a.m, 1024, 0, stream>>>(sc);
  ZENO_STEP(hipGetLastError());
  DzArgs d = {};
  LogitArgs& l = d.l;
  if (a.rows > 0)
    ZENO_STEP(side_of(a.hidden, a.ldh, a.dtype, a.rows, a.width, reinterpret_cast<u16*>(ws + p.hidden), l.h, stream));
  l.pairs = pairs_of(planes, planes);
  l.width = padded_width(a.width);
  l.vocab = a.vocab;
  l.rows = a.rows;
  l.bias = a.bias;
  l.labels = a.labels;
  Side hidden = l.h;   // as the weights' gradients take it
  if (convert) {
    const dim3 grid((unsigned)ceil_div(a.width, 512), (unsigned)ceil_div(a.rows, kColumnRows));
    hidden = {reinterpret_cast<const u16*>(ws + p.half), l.width, 0, a.rows};
    const ColumnArgs c = {l.h, a.width, a.m, a.rows, a.offsets, columns, reinterpret_cast<u16*>(ws + p.half)};
    column_max_kernel<<<grid, 1024, 0, stream>>>(c);
    column_half_kernel<<<grid, 1024, 0, stream>>>(c);
    ZENO_STEP(hipGetLastError());
  }
  d.stats = a.stats;
  d.grad_logp = a.grad_logp;
  d.entropy = a.entropy;
  d.grad_entropy = a.grad_entropy;
  d.up = up;
  d.dz = reinterpret_cast<u16*>(ws + p.dz);
  d.ldz = p.piece;
  d.plane = (long long)a.rows * p.piece;
  float* slots = reinterpret_cast<float*>(ws + p.slots);
  const int fine = a.dtype == ZENO_BF16 ? 2 : 0;   // the first plane that the float32 gradients take
  const u16* fine_dz = d.dz + fine * d.plane;
  for (int v0 = 0; v0 < a.vocab; v0 += p.piece) {
    const int values = std::min(p.piece, a.vocab - v0);
    auto weights = [&](int v) { return reinterpret_cast<const unsigned char*>(a.weight) + (size_t)v * a.ldw * bytes; };
    if (a.rows > 0 && p.few) {
      const FewArgs f = {a.hidden, weights(v0), a.ldh, a.ldw, a.rows, values, a.width};
      l.v0 = v0;
      ZENO_STEP(a.dtype == ZENO_F32 ? (start_few_dz<float, kBf16Three>(f, d, stream))
                                    : half ? (start_few_dz<_Float16, kHalfTwo>(f, d, stream)) : (start_few_dz<__bf16, kBf16TwoHalfTwo>(f, d, stream)));
    }
    // The weights of the piece: at once where they are read as they stand, or as many as are packed at a time.
    const bool products = a.rows > 0 && (!p.few || a.dhidden != nullptr);
    for (int s0 = 0; products && s0 < values; s0 += direct ? p.piece : p.pack) {
      const int here = std::min(direct ? p.piece : p.pack, values - s0);
      ZENO_STEP(side_of(weights(v0 + s0), a.ldw, a.dtype, here, a.width, reinterpret_cast<u16*>(ws + p.weight), l.w, stream));
      if (!p.few) {
        DzArgs part = d;
        part.dz = d.dz + s0;
        part.l.v0 = v0 + s0;
        const int side = p.wide_logits ? kWideSide : kTileSide;
        part.l.tiles_m = ceil_div(here, side);
        part.l.tiles_n = ceil_div(a.rows, side);
        ZENO_STEP(p.wide_logits ? start_dz<WideTile>(part, a.dtype, stream) : start_dz<ThirdTile>(part, a.dtype, stream));
      }
      if (a.dhidden != nullptr) {
        HiddenArgs h = {};
        h.dz = {d.dz + s0, d.ldz, d.plane, a.rows};
        h.w = l.w;
        h.w.extent = l.width;   // (across the contraction: columns)
        h.pairs = pairs_of(3, 3);
        const int tile = p.wide_hidden ? kWideSide : kTileSide;
        h.tiles_m = ceil_div(a.rows, tile);
        h.tiles_n = ceil_div(a.width, tile);
        h.rows = a.rows;
        h.width = a.width;
        h.length = here;
        h.per = ceil_div(ceil_div(here, p.splits), kStep) * kStep;
        h.first = v0 + s0 == 0;
        h.slots = slots;
        ZENO_STEP(p.wide_hidden ? start_hidden<WideTile>(h, a.dtype, p.splits, stream) : start_hidden<MidTile>(h, a.dtype, p.splits, stream));
      }
    }
    if (a.dweight != nullptr || a.dbias != nullptr) {
      WeightArgs w = {};
      w.dz = {fine_dz, d.ldz, d.plane, p.piece};
      w.h = hidden;
      w.h.extent = l.width;
      w.pairs = pairs_of(p.planes - fine, planes);
      w.columns = convert ? columns : nullptr;
      const int tile = p.wide_weight ? kWideSide : kTileSide;
      w.tiles_m = ceil_div(values, tile);
      w.tiles_n = a.dweight != nullptr ? ceil_div(a.width, tile) : 1;   // (the first ones take the bias's along)
      w.rows = a.rows;
      w.width = a.width;
      w.values = values;
      w.offsets = a.offsets;
      w.power = power;
      w.dweight = a.dweight != nullptr ? a.dweight + (long long)v0 * a.width : nullptr;
      w.dbias = a.dbias != nullptr ? a.dbias + v0 : nullptr;
      w.ldw = a.ldg;
      w.ldb = a.ldb;
      w.parts = p.parts;
      const WeightJoinArgs j = {reinterpret_cast<float*>(ws + p.sums), reinterpret_cast<float*>(ws + p.sums) + (long long)values * a.width,
                                a.m * (long long)values * (a.width + 1LL), (long long)values * (a.width + 1LL), (long long)values * a.width,
                                p.parts, values, w.dweight, w.dbias, a.ldg, a.ldb};
      if (p.parts > 1) {
        w.dweight = w.dweight != nullptr ? const_cast<float*>(j.dweight) : nullptr;
        w.dbias = w.dbias != nullptr ? const_cast<float*>(j.dbias) : nullptr;
        w.slot = j.slot;
        w.ldw = w.ldb = j.group;
      }
      if (p.wide_weight) ZENO_STEP(planes == 1 ? (start_weight<WideTile, true>(w, a.m, stream)) : (start_weight<WideTile, false>(w, a.m, stream)));
      else ZENO_STEP(planes == 1 ? (start_weight<ThirdTile, true>(w, a.m, stream)) : (start_weight<ThirdTile, false>(w, a.m, stream)));
      if (p.parts > 1) {
        weight_join_kernel<<<dim3((unsigned)std::min<long long>((j.n + values + 255) / 256, 2048), (unsigned)a.m), 256, 0, stream>>>(j);
        ZENO_STEP(hipGetLastError());
      }
    }
  }
  if (a.dhidden != nullptr && a.rows > 0) {
    const HiddenJoinArgs j = {slots, p.splits, a.rows, a.width, a.m, a.offsets, planes == 1 ? up : nullptr, a.dhidden, a.lddh};
    const dim3 grid((unsigned)std::min(ceil_div(a.width, 1024), 64), (unsigned)std::min(a.rows, 16384));
    if (a.dtype == ZENO_F32) hidden_join_kernel<float><<<grid, 256, 0, stream>>>(j);
    else if (half) hidden_join_kernel<_Float16><<<grid, 256, 0, stream>>>(j);
    else hidden_join_kernel<__bf16><<<grid, 256, 0, stream>>>(j);
    ZENO_STEP(hipGetLastError());
  }
  return hipSuccess;
}

}  // namespace zeno
