// Activations in 8 bits: blocks of 32 columns of a row share a power-of-two scale, so that dividing by it is exact and the only
// rounding is the one to the e4m3 grid (half a step: 2^-4 of a value, or 2^-10 of the scale for the smallest).
// Rows of values are padded with zeros to whole blocks: their words are aligned whatever the width.
#include "zeno_tokens.h"

namespace zeno {
namespace {

constexpr int kThreads = 256;

// A thread takes 8 columns: four threads share a block, whose largest magnitude two lane exchanges find.  Bound by memory: 16384 x 4096 bf16
// 40 us (5.1 TB/s; plain streams of two reads and a write reach 6.4).
template <typename T>
__global__ __launch_bounds__(kThreads) void checkpoint_kernel(const T* __restrict__ x, long long ldx, int rows, int width, int blocks,
                                                              uint8_t* __restrict__ values, uint8_t* __restrict__ scales) {
  const long long per_row = 4LL * blocks, total = per_row * rows;
  for (long long base = (long long)blockIdx.x * kThreads; base < total; base += (long long)gridDim.x * kThreads) {
    const long long i = base + threadIdx.x;
    const bool live = i < total;   // (whole blocks: four neighbours live and die together)
    const long long row = live ? i / per_row : 0;
    const int col = live ? (int)(i % per_row) * 8 : 0;
    float v[8];
    const T* p = x + row * ldx + col;
    constexpr int N = Wide<T>::N;
#pragma unroll
    for (int h = 0; h < 8 / N; ++h) {
      float part[N];
      if (col + (h + 1) * N <= width)
        load_wide(p + h * N, part);
      else
        load_part(p + h * N, width - col - h * N, 0.f, part);
#pragma unroll
      for (int j = 0; j < N; ++j) v[h * N + j] = part[j];
    }
    float q[8];
    const int k = ckpt_quotients<8>(v, q);
    if (live) {
      uint2 w;
      w.x = ckpt_pack4(q[0], q[1], q[2], q[3]);
      w.y = ckpt_pack4(q[4], q[5], q[6], q[7]);
      *reinterpret_cast<uint2*>(values + row * (blocks * 32LL) + col) = w;
      if ((threadIdx.x & 3) == 0) scales[row * blocks + col / 32] = (uint8_t)(k + 127);
    }
  }
}

template <typename T>
__device__ inline float largest_of();
template <>
__device__ inline float largest_of<float>() { return 3.402823466e38f; }
template <>
__device__ inline float largest_of<__bf16>() { return 3.38953139e38f; }
template <>
__device__ inline float largest_of<_Float16>() { return 65504.f; }

// The way back: 16384 x 4096 bf16 31 us (6.5 TB/s).
template <typename T>
__global__ __launch_bounds__(kThreads) void checkpoint_values_kernel(const uint8_t* __restrict__ values,
                                                                     const uint8_t* __restrict__ scales, int rows, int width,
                                                                     int blocks, T* __restrict__ out, long long ldo) {
  const long long per_row = 4LL * blocks, total = per_row * rows;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < total; i += (long long)gridDim.x * kThreads) {
    const long long row = i / per_row;
    const int col = (int)(i % per_row) * 8;
    const uint2 w = *reinterpret_cast<const uint2*>(values + row * (blocks * 32LL) + col);
    const unsigned words[2] = {w.x, w.y};
    float v[8];
    ckpt_unpack(words, ckpt_scale((int)scales[row * blocks + col / 32] - 127), v);
    // a value just below the type's largest may have been rounded up past it
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (fabsf(v[j]) > largest_of<T>()) v[j] = copysignf(largest_of<T>(), v[j]);
    constexpr int N = Wide<T>::N;
#pragma unroll
    for (int h = 0; h < 8 / N; ++h) {
      float part[N];
#pragma unroll
      for (int j = 0; j < N; ++j) part[j] = v[h * N + j];
      const int at = col + h * N;
      if (at + N <= width)
        store_wide(out + row * ldo + at, part);
      else
        store_part(out + row * ldo + at, width - at, part);
    }
  }
}

unsigned grid_for(int rows, int width) {
  const long long blocks = (4LL * ckpt_blocks(width) * rows + kThreads - 1) / kThreads;
  return (unsigned)(blocks < 8192 ? blocks : 8192);
}

}  // namespace

hipError_t launch_checkpoint(const void* x, long long ldx, int dtype, int rows, int width, uint8_t* values, uint8_t* scales,
                             hipStream_t stream) {
  const dim3 grid(grid_for(rows, width)), block(kThreads);
  const int blocks = ckpt_blocks(width);
  if (dtype == ZENO_F32)
    hipLaunchKernelGGL(checkpoint_kernel<float>, grid, block, 0, stream, reinterpret_cast<const float*>(x), ldx, rows, width, blocks,
                       values, scales);
  else if (dtype == ZENO_BF16)
    hipLaunchKernelGGL(checkpoint_kernel<__bf16>, grid, block, 0, stream, reinterpret_cast<const __bf16*>(x), ldx, rows, width, blocks,
                       values, scales);
  else
    hipLaunchKernelGGL(checkpoint_kernel<_Float16>, grid, block, 0, stream, reinterpret_cast<const _Float16*>(x), ldx, rows, width,
                       blocks, values, scales);
  return hipGetLastError();
}

hipError_t launch_checkpoint_values(const uint8_t* values, const uint8_t* scales, int rows, int width, int dtype, void* out,
                                    long long ldo, hipStream_t stream) {
  const dim3 grid(grid_for(rows, width)), block(kThreads);
  const int blocks = ckpt_blocks(width);
  if (dtype == ZENO_F32)
    hipLaunchKernelGGL(checkpoint_values_kernel<float>, grid, block, 0, stream, values, scales, rows, width, blocks,
                       reinterpret_cast<float*>(out), ldo);
  else if (dtype == ZENO_BF16)
    hipLaunchKernelGGL(checkpoint_values_kernel<__bf16>, grid, block, 0, stream, values, scales, rows, width, blocks,
                       reinterpret_cast<__bf16*>(out), ldo);
  else
    hipLaunchKernelGGL(checkpoint_values_kernel<_Float16>, grid, block, 0, stream, values, scales, rows, width, blocks,
                       reinterpret_cast<_Float16*>(out), ldo);
  return hipGetLastError();
}

}  // namespace zeno
