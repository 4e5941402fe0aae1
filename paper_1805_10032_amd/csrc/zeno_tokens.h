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

template <typename T>
__device__ inline void store_part(T* p, int n, const float (&v)[Wide<T>::N]) {
#pragma unroll
  for (int i = 0; i < Wide<T>::N; ++i)
    if (i < n) p[i] = (T)v[i];
}

__device__ inline float wave_sum_f(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}
__device__ inline float wave_max_f(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
  return v;
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

// v / 2^k on the e4m3 grid, rounded to nearest even; an infinity or a NaN becomes NaN.  With the largest k (floats above 448 * 2^119) the
// grid's next step up may be beyond float32's range: values stop at the step below it.
__device__ inline float ckpt_quotient(float v, int k) {
  float q = v * ckpt_scale(-k);                        // -k lies in [-120, 127]: a normal scale, and the product is exact or tiny
  if (k >= 120) q = fminf(fmaxf(q, -240.f), 240.f);
  return fabsf(v) < __builtin_inff() ? q : __builtin_nanf("");
}
__device__ inline unsigned ckpt_pack4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
// the largest finite magnitude among |v|, `sofar`
__device__ inline float ckpt_larger(float sofar, float v) {
  const float a = fabsf(v);
  return a < __builtin_inff() ? fmaxf(sofar, a) : sofar;
}
template <int N>
__device__ inline void ckpt_unpack(const unsigned* words, float scale, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    v[i] = __builtin_amdgcn_cvt_f32_fp8(words[i / 4], 0) * scale;
    v[i + 1] = __builtin_amdgcn_cvt_f32_fp8(words[i / 4], 1) * scale;
    v[i + 2] = __builtin_amdgcn_cvt_f32_fp8(words[i / 4], 2) * scale;
    v[i + 3] = __builtin_amdgcn_cvt_f32_fp8(words[i / 4], 3) * scale;
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
