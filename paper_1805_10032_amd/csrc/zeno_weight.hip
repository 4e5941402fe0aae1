// Weight gradients of a linear layer from 8-bit activations, per group of rows (a worker's tokens):
//   dW_g[o][k] = sum_{t in g} dy[t][o] a[t][k],   db_g[o] = sum_{t in g} dy[t][o].
//
// A matrix product over tokens on the bf16 matrix cores.  An e4m3 value times its power-of-two scale has four significant bits: it is
// exact in bf16.  dy goes in as bf16 pieces: one for bf16, two for fp16 (11 bits), three for float32 (24 bits), so every product is
// exact and the only rounding is that of the float32 sums.
// Both operands have the tokens as their slow axis, and a lane of the matrix instruction wants eight tokens of one column: tiles
// stay as they are in LDS and the transposing LDS read turns four tokens x sixteen columns at a time.
#include "zeno_tokens.h"

namespace zeno {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 128;      // outputs x inputs of a workgroup; each of its four waves 64 x 64
constexpr int kTokens = 32;     // tokens of a stage
constexpr int kPitch = 160;     // bf16 of an LDS row: 64 bytes behind a multiple of 256, so four rows lie on different banks

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct Span {
  int begin, end;
};
__device__ inline Span piece_of(const WeightGradArgs& a, int g, int piece, int pieces) {
  const int b = group_offset(a.offsets, g, a.rows), e = group_offset(a.offsets, g + 1, a.rows);
  const int n = e > b ? e - b : 0;
  const int len = ((n + pieces - 1) / pieces + kTokens - 1) / kTokens * kTokens;
  const long long lo = b + (long long)len * piece, hi = lo + len;
  Span s;
  s.begin = (int)(lo < b + n ? lo : b + n);
  s.end = (int)(hi < b + n ? hi : b + n);
  return s;
}

// v as the sum of P bf16 pieces.
template <int P>
__device__ inline void split(float v, __bf16 (&piece)[P]) {
  const bool fin = fabsf(v) < __builtin_inff();
  // (a float above bf16's range leaves its rest to the second piece instead of rounding to infinity)
  piece[0] = (__bf16)(P > 1 && fin ? fminf(fmaxf(v, -3.38953139e38f), 3.38953139e38f) : v);
  float rest = v;
#pragma unroll
  for (int i = 1; i < P; ++i) {
    rest = fin ? rest - (float)piece[i - 1] : 0.f;
    piece[i] = (__bf16)rest;
  }
}

// Eight columns of a row as floats, zeros behind its end.
template <typename T>
__device__ inline void load8(const T* row, int col, int width, float (&v)[8]) {
  constexpr int N = Wide<T>::N;
#pragma unroll
  for (int h = 0; h < 8 / N; ++h) {
    float part[N];
    const int at = col + h * N;
    if (at + N <= width)
      load_wide(row + at, part);
    else
      load_part(row + at, width - at, 0.f, part);
#pragma unroll
    for (int j = 0; j < N; ++j) v[h * N + j] = part[j];
  }
}

// One operand of a matrix instruction: 32 columns from `col` on of 16 tokens, lane l column l % 32, tokens 8 (l / 32) + 0..7.
__device__ inline bf16x8 read_columns(const __bf16* tile, int col, int token, int lane) {
  const int at = (token + 8 * (lane / 32) + (lane % 16) / 4) * kPitch + col + 16 * ((lane / 16) % 2) + 4 * (lane % 4);
  typedef __attribute__((address_space(3))) s16x4* lds;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(tile + at));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(tile + at + 4 * kPitch));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, both);
}

template <typename T, int P>
__global__ __launch_bounds__(kThreads) void weight_grad_kernel(WeightGradArgs a, int tiles_in, int pieces, float* partial) {
  __shared__ __align__(16) __bf16 ys[P][kTokens * kPitch];
  __shared__ __align__(16) __bf16 as[kTokens * kPitch];
  __shared__ float bias_part[16][kTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
  const int o0 = (int)(blockIdx.x / tiles_in) * kTile, k0 = (int)(blockIdx.x % tiles_in) * kTile;
  const int g = blockIdx.y / pieces, piece = blockIdx.y % pieces;
  const Span span = piece_of(a, g, piece, pieces);
  const int blocks = ckpt_blocks(a.width);
  const int wo = 64 * (wave / 2), wk = 64 * (wave % 2);
  f32x16 acc[2][2] = {};
  float bias[8] = {};
  for (int t0 = span.begin; t0 < span.end; t0 += kTokens) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int token = tid / 16 + 16 * h, col = 8 * (tid % 16);
      const bool live = t0 + token < span.end;
      const long long row = live ? t0 + token : span.begin;
      float v[8];
      load8(reinterpret_cast<const T*>(a.dy) + row * a.lddy, o0 + col, live ? a.out : 0, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) bias[j] += v[j];
      bf16x8 plane[P];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        __bf16 p[P];
        split<P>(v[j], p);
#pragma unroll
        for (int i = 0; i < P; ++i) plane[i][j] = p[i];
      }
#pragma unroll
      for (int i = 0; i < P; ++i) *reinterpret_cast<bf16x8*>(&ys[i][token * kPitch + col]) = plane[i];
      bf16x8 kept = {};
      if (live && k0 + col < blocks * kCkptBlock) {
        const uint2 w = *reinterpret_cast<const uint2*>(a.values + row * ((long long)blocks * kCkptBlock) + k0 + col);
        const float s = ckpt_scale((int)a.scales[row * blocks + (k0 + col) / kCkptBlock] - 127);
        const bf16x2 q0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, s, false), q1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, s, true);
        const bf16x2 q2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, s, false), q3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, s, true);
        kept = {q0.x, q0.y, q1.x, q1.y, q2.x, q2.y, q3.x, q3.y};
      }
      *reinterpret_cast<bf16x8*>(&as[token * kPitch + col]) = kept;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTokens; t += 16) {
      bf16x8 x[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) x[j] = read_columns(as, wk + 32 * j, t, lane);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int p = P - 1; p >= 0; --p) {
          const bf16x8 y = read_columns(ys[p], wo + 32 * i, t, lane);
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, x[j], acc[i][j], 0, 0, 0);
        }
    }
    __syncthreads();
  }
  const long long n = (long long)a.out * a.width;
  float* dw = pieces == 1 ? a.dweight + g * a.ldw : partial + (long long)blockIdx.y * (n + a.out);
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int k = k0 + wk + 32 * j + lane % 32;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int o = o0 + wo + 32 * i + 8 * (e / 4) + 4 * (lane / 32) + e % 4;
        if (o < a.out && k < a.width) dw[(long long)o * a.width + k] = acc[i][j][e];
      }
    }
  if (k0 == 0 && a.dbias != nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) bias_part[tid / 16][8 * (tid % 16) + j] = bias[j];
    __syncthreads();
    if (tid < kTile && o0 + tid < a.out) {
      float sum = 0.f;
      for (int i = 0; i < 16; ++i) sum += bias_part[i][tid];
      float* db = pieces == 1 ? a.dbias + g * a.ldb : dw + n;
      db[o0 + tid] = sum;
    }
  }
}

// Wide tiles for long sums: 256 x 256 outputs a workgroup, 128 x 128 a wave, which halves what each matrix instruction reads from LDS
// (64 x 64 a wave asks for all of its bandwidth).  One workgroup a compute unit; stages alternate between two buffers, so the next
// one is fetched and converted while this one is multiplied.
constexpr int kWide = 256;
constexpr int kWidePitch = 288;   // bf16 of an LDS row, 64 bytes behind a multiple of 256

__device__ inline bf16x8 read_wide(const __bf16* tile, int col, int token, int lane) {
  const int at = (token + 8 * (lane / 32) + (lane % 16) / 4) * kWidePitch + col + 16 * ((lane / 16) % 2) + 4 * (lane % 4);
  typedef __attribute__((address_space(3))) s16x4* lds;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(tile + at));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(tile + at + 4 * kWidePitch));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, both);
}

// What a thread fetches of a stage: 8 columns of four tokens of dy, 16 of two tokens of the activations.
template <typename T>
struct Fetched {
  typename Wide<T>::type dy[4][8 / Wide<T>::N];
  uint4 a[2];
  uint8_t scale[2];
};

template <typename T>
__device__ inline void fetch(const WeightGradArgs& a, int t0, int end, int o0, int k0, int blocks, int tid, Fetched<T>& f) {
  constexpr int N = Wide<T>::N;
  const int last = end - 1;
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const int token = t0 + tid / 32 + 8 * h, col = o0 + 8 * (tid % 32);
    const T* p = reinterpret_cast<const T*>(a.dy) + (long long)(token < last ? token : last) * a.lddy + col;
    if (token < end && col + 8 <= a.out) {
#pragma unroll
      for (int i = 0; i < 8 / N; ++i) f.dy[h][i] = *reinterpret_cast<const typename Wide<T>::unaligned*>(p + i * N);
    } else {
#pragma unroll
      for (int i = 0; i < 8 / N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) f.dy[h][i][j] = token < end && col + i * N + j < a.out ? p[i * N + j] : (T)0.f;
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int token = t0 + tid / 16 + 16 * h, col = k0 + 16 * (tid % 16);
    f.a[h] = make_uint4(0, 0, 0, 0);
    f.scale[h] = 127;
    if (token < end && col < blocks * kCkptBlock) {
      f.a[h] = *reinterpret_cast<const uint4*>(a.values + (long long)token * (blocks * kCkptBlock) + col);
      f.scale[h] = a.scales[(long long)token * blocks + col / kCkptBlock];
    }
  }
}

__device__ inline bf16x8 widen8(unsigned x, unsigned y, float s) {
  const bf16x2 q0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, false), q1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, true);
  const bf16x2 q2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, s, false), q3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, s, true);
  return bf16x8{q0.x, q0.y, q1.x, q1.y, q2.x, q2.y, q3.x, q3.y};
}

template <typename T, int P>
struct WideStage {
  __bf16 y[P][kTokens * kWidePitch];
  __bf16 a[kTokens * kWidePitch];
};

template <typename T, int P>
__device__ inline void deposit(const Fetched<T>& f, WideStage<T, P>& st, int tid, float (&bias)[8]) {
  constexpr int N = Wide<T>::N;
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    bf16x8 plane[P];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = (float)f.dy[h][j / N][j % N];
      bias[j] += v;
      __bf16 p[P];
      split<P>(v, p);
#pragma unroll
      for (int i = 0; i < P; ++i) plane[i][j] = p[i];
    }
#pragma unroll
    for (int i = 0; i < P; ++i) *reinterpret_cast<bf16x8*>(&st.y[i][(tid / 32 + 8 * h) * kWidePitch + 8 * (tid % 32)]) = plane[i];
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float s = ckpt_scale((int)f.scale[h] - 127);
    __bf16* to = &st.a[(tid / 16 + 16 * h) * kWidePitch + 16 * (tid % 16)];
    *reinterpret_cast<bf16x8*>(to) = widen8(f.a[h].x, f.a[h].y, s);
    *reinterpret_cast<bf16x8*>(to + 8) = widen8(f.a[h].z, f.a[h].w, s);
  }
}

template <typename T, int P>
__global__ __launch_bounds__(kThreads, 1) void weight_grad_wide_kernel(WeightGradArgs a, int tiles_in) {
  extern __shared__ __align__(16) unsigned char memory[];
  WideStage<T, P>* stage = reinterpret_cast<WideStage<T, P>*>(memory);   // two of them
  const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
  const int o0 = (int)(blockIdx.x / tiles_in) * kWide, k0 = (int)(blockIdx.x % tiles_in) * kWide;
  const int g = blockIdx.y;
  const Span span = piece_of(a, g, 0, 1);
  const int blocks = ckpt_blocks(a.width);
  const int wo = 128 * (wave / 2), wk = 128 * (wave % 2);
  f32x16 acc[4][4] = {};
  float bias[8] = {};
  Fetched<T> f;
  const int stages = (span.end - span.begin + kTokens - 1) / kTokens;
  if (stages > 0) {
    fetch<T>(a, span.begin, span.end, o0, k0, blocks, tid, f);
    deposit<T, P>(f, stage[0], tid, bias);
    if (stages > 1) fetch<T>(a, span.begin + kTokens, span.end, o0, k0, blocks, tid, f);
  }
  __syncthreads();
  for (int i = 0; i < stages; ++i) {
    const WideStage<T, P>& st = stage[i & 1];
#pragma unroll
    for (int t = 0; t < kTokens; t += 16) {
      bf16x8 x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = read_wide(st.a, wk + 32 * j, t, lane);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int p = P - 1; p >= 0; --p) {
          const bf16x8 y = read_wide(st.y[p], wo + 32 * r, t, lane);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[r][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, x[j], acc[r][j], 0, 0, 0);
        }
      if (t == 0 && i + 1 < stages) {
        deposit<T, P>(f, stage[(i + 1) & 1], tid, bias);
        if (i + 2 < stages) fetch<T>(a, span.begin + (i + 2) * kTokens, span.end, o0, k0, blocks, tid, f);
      }
    }
    __syncthreads();
  }
  float* dw = a.dweight + g * a.ldw;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = k0 + wk + 32 * j + lane % 32;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int o = o0 + wo + 32 * r + 8 * (e / 4) + 4 * (lane / 32) + e % 4;
        if (o < a.out && k < a.width) dw[(long long)o * a.width + k] = acc[r][j][e];
      }
    }
  if (k0 == 0 && a.dbias != nullptr) {
    float (*part)[kWide] = reinterpret_cast<float (*)[kWide]>(memory);   // [8][256]; behind the last barrier nobody reads a stage
#pragma unroll
    for (int j = 0; j < 8; ++j) part[tid / 32][8 * (tid % 32) + j] = bias[j];
    __syncthreads();
    if (o0 + tid < a.out) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += part[i][tid];
      a.dbias[g * a.ldb + o0 + tid] = sum;
    }
  }
}

// The pieces of a group's tokens, in order.
__global__ __launch_bounds__(kThreads) void weight_grad_join_kernel(WeightGradArgs a, int pieces, const float* __restrict__ partial) {
  const long long n = (long long)a.out * a.width, all = n + (a.dbias != nullptr ? a.out : 0), stride = n + a.out;
  const int g = blockIdx.y;
  const float* p = partial + (long long)g * pieces * stride;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < all; i += (long long)gridDim.x * kThreads) {
    float sum = 0.f;
    for (int s = 0; s < pieces; ++s) sum += p[s * stride + i];
    if (i < n)
      a.dweight[g * a.ldw + i] = sum;
    else
      a.dbias[g * a.ldb + i - n] = sum;
  }
}

long long tiles_of(int out, int width) { return (long long)ceil_div(out, kTile) * ceil_div(width, kTile); }

// Pieces that a group's tokens are cut into: where the output tiles alone leave most of the chip idle.
int pieces_of(int rows, int out, int width, int m) {
  const long long tiles = tiles_of(out, width) * m;
  long long pieces = 512 / tiles;
  const long long most = rows / m / 256;
  if (pieces > most) pieces = most;
  return pieces < 1 ? 1 : (int)pieces;
}

bool wide_tiles(int rows, int out, int width, int m) {
  return out > kTile && width > kTile && (long long)ceil_div(out, kWide) * ceil_div(width, kWide) * m >= 256 && rows / m >= 64;
}

template <typename T, int P>
hipError_t start_wide(const WeightGradArgs& a, hipStream_t stream) {
  const size_t lds = 2 * sizeof(WideStage<T, P>);
  const auto kernel = weight_grad_wide_kernel<T, P>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  const int tiles_in = ceil_div(a.width, kWide);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles_in * (long long)ceil_div(a.out, kWide)), a.m), dim3(kThreads), lds, stream, a, tiles_in);
  return hipGetLastError();
}

}  // namespace

bool weight_gradient_fits(int out, int width) { return tiles_of(out, width) * kThreads < (1LL << 31); }

size_t weight_gradient_workspace_bytes(int rows, int out, int width, int m) {
  const int pieces = pieces_of(rows, out, width, m);
  if (pieces == 1) return 256;
  return align_up((size_t)m * pieces * ((size_t)out * width + out) * sizeof(float), 256);
}

hipError_t launch_weight_gradient(const WeightGradArgs& a, void* workspace, hipStream_t stream) {
  const int pieces = pieces_of(a.rows, a.out, a.width, a.m);
  float* partial = reinterpret_cast<float*>(workspace);
  if (wide_tiles(a.rows, a.out, a.width, a.m)) {
    if (a.dtype == ZENO_F32) return start_wide<float, 3>(a, stream);
    if (a.dtype == ZENO_BF16) return start_wide<__bf16, 1>(a, stream);
    return start_wide<_Float16, 2>(a, stream);
  }
  const dim3 grid((unsigned)tiles_of(a.out, a.width), a.m * pieces), block(kThreads);
  const int tiles_in = ceil_div(a.width, kTile);
  switch (a.dtype) {
    case ZENO_F32: hipLaunchKernelGGL((weight_grad_kernel<float, 3>), grid, block, 0, stream, a, tiles_in, pieces, partial); break;
    case ZENO_BF16: hipLaunchKernelGGL((weight_grad_kernel<__bf16, 1>), grid, block, 0, stream, a, tiles_in, pieces, partial); break;
    default: hipLaunchKernelGGL((weight_grad_kernel<_Float16, 2>), grid, block, 0, stream, a, tiles_in, pieces, partial); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || pieces == 1) return e;
  const long long n = (long long)a.out * a.width + a.out, blocks = (n + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(weight_grad_join_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096), a.m), block, 0, stream, a, pieces, partial);
  return hipGetLastError();
}

}  // namespace zeno
