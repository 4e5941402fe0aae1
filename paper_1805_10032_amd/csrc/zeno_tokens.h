// Shared by the operators for models that answer with tokens (log probabilities, layer norm, activations in 8 bits, weight
// gradients, the score from log probabilities): element types, 128-bit access to rows at any element alignment, reductions.
#ifndef ZENO_TOKENS_H_
#define ZENO_TOKENS_H_

#include "zeno_internal.h"

namespace zeno {

// 16 bytes of a row.  Rows may start at any element: gfx950 takes 128-bit global accesses at any alignment, so there is one
// path for all of them.
template <typename T>
struct Wide {
  static constexpr int N = 16 / (int)sizeof(T);
  typedef T type __attribute__((ext_vector_type(N)));
  typedef type unaligned __attribute__((aligned(sizeof(T))));
};

template <typename T>
__device__ inline void load_wide(const T* p, float (&v)[Wide<T>::N]) {
  const typename Wide<T>::type raw = *reinterpret_cast<const typename Wide<T>::unaligned*>(p);
#pragma unroll
  for (int i = 0; i < Wide<T>::N; ++i) v[i] = (float)raw[i];
}

// The first n of N values, `fill` behind them: the end of a row.
template <typename T>
__device__ inline void load_part(const T* p, int n, float fill, float (&v)[Wide<T>::N]) {
#pragma unroll
  for (int i = 0; i < Wide<T>::N; ++i) v[i] = i < n ? (float)p[i] : fill;
}

template <typename T>
__device__ inline void store_wide(T* p, const float (&v)[Wide<T>::N]) {
  typename Wide<T>::type raw;
#pragma unroll
  for (int i = 0; i < Wide<T>::N; ++i) raw[i] = (T)v[i];
  *reinterpret_cast<typename Wide<T>::unaligned*>(p) = raw;
}

// Rows that start on a memory line may be written past the caches, whole lines at once, where the caches would keep them only to displace what
// the next operators read and to write them then.  Rows that do not start on one would be written in parts (a weight gradient 1000 columns wide 41 ->
// 45 us).
__device__ inline bool on_line(const void* p) { return (reinterpret_cast<unsigned long long>(p) & 127) == 0; }
// What the next launch reads back, gradients of activations and of logits, goes past the caches only where half of the 256 MB behind them would
// not hold it.  Gradient, weight gradient from it and product with the weights, ordinary / past, us: dlogits in bf16 17 MB 90 / 92, 34 MB 141 /
// 143, 134 MB 427 / 422, 537 MB 1149 / 1154; dx in bf16 17 MB 103 / 103, 134 MB 347 / 358.  The kernel again and again, with nothing that reads what
// it wrote: dx 134 MB 90 / 74, dlogits in float32 268 MB 100 / 82.  A whole iteration takes the same time either way.
constexpr long long kPastBytes = 128LL << 20;
// (or the compiler joins such a store with the ordinary one of the other branch)
__device__ inline void keep_apart() { asm volatile("" ::: "memory"); }
template <typename T>
__device__ inline void store_wide_past(T* p, const float (&v)[Wide<T>::N]) {
  typename Wide<T>::type raw;
#pragma unroll
  for (int i = 0; i < Wide<T>::N; ++i) raw[i] = (T)v[i];
  __builtin_nontemporal_store(raw, reinterpret_cast<typename Wide<T>::unaligned*>(p));
  keep_apart();
}

template <typename T>
__device__ inline void store_part(T* p, int n, const float (&v)[Wide<T>::N]) {
#pragma unroll
  for (int i = 0; i < Wide<T>::N; ++i)
    if (i < n) p[i] = (T)v[i];
}

// Reductions over the 64 lanes without LDS: neighbours by DPP inside rows of sixteen, rows by the lane swaps.  Every lane adds the same
// pairs, so all of them get the same bits.
template <int CTRL>
__device__ inline float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ inline int dpp_int(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;
template <typename F>
__device__ inline float wave_reduce(float v, F f) {
  v = f(v, dpp<kDppXor1>(v));
  v = f(v, dpp<kDppXor2>(v));
  v = f(v, dpp<kDppHalfMirror>(v));
  v = f(v, dpp<kDppMirror>(v));
  const unsigned u = __float_as_uint(v);
  const auto rows = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = f(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
  const unsigned w = __float_as_uint(v);
  const auto halves = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return f(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
}
__device__ inline float wave_sum_f(float v) {
  return wave_reduce(v, [](float a, float b) { return a + b; });
}
__device__ inline float wave_max_f(float v) {
  return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}

// Barrier of the NW waves that share a row.  One wave runs its LDS accesses in order, so only the compiler has to keep them so.
template <int NW>
__device__ inline void row_sync() {
  if (NW == 1) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    __builtin_amdgcn_wave_barrier();
  } else {
    __syncthreads();
  }
}

// ---- log probabilities (zeno_logprobs.hip)
struct LogprobsArgs {
  const void* logits;
  long long ldz;
  int dtype, rows, vocab;
  const int32_t* labels;
  float *logp, *entropy, *stats;
  int top;
  int32_t* top_index;
  float* top_logp;
};
size_t logprobs_workspace_bytes(int rows, int vocab, int top);
hipError_t launch_logprobs(const LogprobsArgs& a, void* workspace, hipStream_t stream);

struct LogprobsGradArgs {
  const void* logits;
  void* dlogits;
  long long ldz, ldd;
  int dtype, rows, vocab;
  const float* stats;
  const int32_t* labels;
  const float *grad_logp, *grad_entropy, *entropy;
  int top;
  const int32_t* top_index;
  const float* grad_top;
  bool large;   // dlogits: kPastBytes or more
};
hipError_t launch_logprobs_backward(const LogprobsGradArgs& a, hipStream_t stream);

// ---- activations in 8 bits (zeno_checkpoint.hip): e4m3 values, kCkptBlock columns share the scale 2^(byte - 127)
constexpr int kCkptBlock = 32;
__host__ __device__ inline int ckpt_blocks(int width) { return (width + kCkptBlock - 1) / kCkptBlock; }

// Exponent k of the scale for a block whose largest finite magnitude is `largest`: the smallest k >= -127 with largest <= 448 * 2^k
// (448 = 1.75 * 2^8 is e4m3's largest value).
__device__ inline int ckpt_exponent(float largest) {
  const unsigned bits = __float_as_uint(largest);
  const int k = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
  return k < -127 ? -127 : k;
}
__device__ inline float ckpt_scale(int k) { return __uint_as_float(k > -127 ? (unsigned)(k + 127) << 23 : 1u << 22); }

__device__ inline unsigned ckpt_pack4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
// N of a block's 32 columns, whose others the next 32 / N - 1 lanes hold, divided by the block's scale; returns its exponent k.  An
// infinity stays one and is packed as NaN; it does not enter the scale.  All lanes of a block take part.
template <int N>
__device__ inline int ckpt_quotients(const float (&v)[N], float (&q)[N]) {
  auto block_max = [](float m) {
    m = fmaxf(m, dpp<kDppXor1>(m));
    m = fmaxf(m, dpp<kDppXor2>(m));
    if (N == 4) m = fmaxf(m, dpp<kDppHalfMirror>(m));
    return m;
  };
  float largest = fabsf(v[0]);
#pragma unroll
  for (int j = 1; j < N; ++j) largest = fmaxf(largest, fabsf(v[j]));
  largest = block_max(largest);
  const float inf = __builtin_inff();
  if (!(largest < inf)) {   // (the lanes of a block agree)
    largest = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) largest = fabsf(v[j]) < inf ? fmaxf(largest, fabsf(v[j])) : largest;
    largest = block_max(largest);
  }
  const int k = ckpt_exponent(largest);
  const float scale = ckpt_scale(-k);   // -k lies in [-120, 127]: a normal scale, and the quotient is exact or far below the grid's first step
#pragma unroll
  for (int j = 0; j < N; ++j) q[j] = v[j] * scale;
  if (k >= 120) {
    // floats above 448 * 2^119: the grid's next step up may lie beyond float32's range
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (fabsf(v[j]) < inf) q[j] = fminf(fmaxf(q[j], -240.f), 240.f);
  }
  return k;
}
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <int N>
__device__ inline void ckpt_unpack(const unsigned* words, float scale, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(words[i / 4], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(words[i / 4], true);
    v[i] = lo.x * scale;
    v[i + 1] = lo.y * scale;
    v[i + 2] = hi.x * scale;
    v[i + 3] = hi.y * scale;
  }
}

hipError_t launch_checkpoint(const void* x, long long ldx, int dtype, int rows, int width, uint8_t* values, uint8_t* scales,
                             hipStream_t stream);
hipError_t launch_checkpoint_values(const uint8_t* values, const uint8_t* scales, int rows, int width, int dtype, void* out,
                                    long long ldo, hipStream_t stream);

// ---- layer norm (zeno_norm.hip)
struct NormArgs {
  const void* x;
  void* y;
  long long ldx, ldy;
  int dtype, rows, width;
  const float *weight, *bias;
  float eps;
  float *mean, *rstd;
  uint8_t *values, *scales;   // checkpoint of x, or nullptr
};
hipError_t launch_layer_norm(const NormArgs& a, hipStream_t stream);

struct NormGradArgs {
  const void *dy, *x;               // x == nullptr: the checkpoint
  const uint8_t *values, *scales;
  void* dx;                         // may be nullptr
  long long lddy, ldx, lddx;
  int dtype, rows, width;
  const float *mean, *rstd, *weight;
  int m;
  const int32_t* offsets;           // nullptr: all rows are one group's
  float *dweight, *dbias;           // may be nullptr
  long long ldw, ldb;
  bool large;                       // dx: kPastBytes or more
};
size_t layer_norm_workspace_bytes(int rows, int width, int m);
hipError_t launch_layer_norm_backward(const NormGradArgs& a, void* workspace, hipStream_t stream);

// Rows of group g: offsets as they stand in device memory, kept inside [0, rows] whatever they hold.
__device__ inline int group_offset(const int32_t* offsets, int g, int rows) {
  if (offsets == nullptr) return g == 0 ? 0 : rows;
  const int o = offsets[g];
  return o < 0 ? 0 : (o > rows ? rows : o);
}

// ---- weight gradients from a checkpoint (zeno_weight.hip)
struct WeightGradArgs {
  const void* dy;
  long long lddy;
  int dtype, rows, out, width;
  const uint8_t *values, *scales;
  int m;
  const int32_t* offsets;
  float *dweight, *dbias;           // dbias may be nullptr
  long long ldw, ldb;
};
bool weight_gradient_fits(int out, int width);   // one launch
size_t weight_gradient_workspace_bytes(int rows, int out, int width, int m);
hipError_t launch_weight_gradient(const WeightGradArgs& a, void* workspace, hipStream_t stream);

// ---- the score from log probabilities (zeno_score_tokens.hip)
size_t score_logprobs_workspace_bytes(int m, long long d);
hipError_t launch_score_logprobs(const float* G, long long ldg, int m, long long d, const float* logp_x, const float* logp,
                                 long long ldp, int n, const int32_t* labels, float rho, float* scores, void* workspace,
                                 hipStream_t stream);

}  // namespace zeno
#endif  // ZENO_TOKENS_H_
