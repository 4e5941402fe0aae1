// Definition 2 from log probabilities: score_i = mean_t (log p_t at x - gamma u_i  -  log p_t at x) - rho ||u_i||^2.
// One pass over G in float64 sums per (row, slice of columns), then one workgroup a row for the tokens and the slices.
#include "zeno_tokens.h"

namespace zeno {
namespace {

constexpr int kThreads = 256;

template <int THREADS>
__device__ inline double block_sum(double v, double* shared) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x / 64] = v;
  __syncthreads();
  double s = 0.0;
  for (int i = 0; i < THREADS / 64; ++i) s += shared[i];
  __syncthreads();
  return s;
}

// Bound by memory: 100 rows of 14.7 M 905 us (6.5 TB/s; the same read stream alone reaches 6.9), 20 rows of 1.58 M 19.5 us (6.5 TB/s).
__global__ __launch_bounds__(kThreads) void row_norms_kernel(const float* __restrict__ G, long long ldg, long long d, int slices,
                                                             long long slice_len, double* __restrict__ partial) {
  __shared__ double shared[kThreads / 64];
  const int slice = blockIdx.x, i = blockIdx.y;
  const long long lo = slice * slice_len, hi = lo + slice_len < d ? lo + slice_len : d;
  const float* g = G + (long long)i * ldg;
  double a0 = 0.0, a1 = 0.0;
  for (long long c = lo + 4LL * threadIdx.x; c < hi; c += 4 * kThreads) {
    if (c + 4 <= hi) {
      const f32x4 v = load_stream4(g + c);
      a0 += (double)v.x * v.x + (double)v.z * v.z;
      a1 += (double)v.y * v.y + (double)v.w * v.w;
    } else {
      for (long long j = c; j < hi; ++j) a0 += (double)g[j] * g[j];
    }
  }
  const double s = block_sum<kThreads>(a0 + a1, shared);
  if (threadIdx.x == 0) partial[(long long)i * slices + slice] = s;
}

// 4 us with 64 tokens, 5.3 us with 4096: a launch and its round trips.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void score_logprobs_kernel(const float* __restrict__ logp_x, const float* __restrict__ logp,
                                                                 long long ldp, int n, const int32_t* __restrict__ labels,
                                                                 const double* __restrict__ partial, int slices, float rho,
                                                                 float* __restrict__ scores) {
  __shared__ double shared[THREADS / 64];
  const int i = blockIdx.x;
  const float* lp = logp + (long long)i * ldp;
  double gain = 0.0, norm = 0.0, counted = 0.0;
#pragma unroll 4
  for (long long t = threadIdx.x; t < n; t += THREADS) {
    const bool counts = labels == nullptr || labels[t] != -1;
    const double d = (double)lp[t] - (double)logp_x[t];
    gain += counts ? d : 0.0;
    counted += counts ? 1.0 : 0.0;
  }
  for (int s = threadIdx.x; s < slices; s += THREADS) norm += partial[(long long)i * slices + s];
  gain = block_sum<THREADS>(gain, shared);
  norm = block_sum<THREADS>(norm, shared);
  counted = block_sum<THREADS>(counted, shared);
  if (threadIdx.x == 0) scores[i] = (float)((counted > 0.0 ? gain / counted : 0.0) - (double)rho * norm);
}

// Slices of a row: enough workgroups for the chip, at least 16 KiB each.
int norm_slices(int m, long long d) {
  long long want = (8192 + m - 1) / m;
  const long long most = (d + 4095) / 4096;
  if (want > most) want = most;
  return (int)(want < 1024 ? want : 1024);
}

}  // namespace

size_t score_logprobs_workspace_bytes(int m, long long d) {
  return align_up((size_t)m * norm_slices(m, d) * sizeof(double), 256);
}

hipError_t launch_score_logprobs(const float* G, long long ldg, int m, long long d, const float* logp_x, const float* logp,
                                 long long ldp, int n, const int32_t* labels, float rho, float* scores, void* workspace,
                                 hipStream_t stream) {
  const int slices = norm_slices(m, d);
  const long long unit = 4 * kThreads;
  const long long slice_len = ((d + slices - 1) / slices + unit - 1) / unit * unit;
  double* partial = reinterpret_cast<double*>(workspace);
  hipLaunchKernelGGL(row_norms_kernel, dim3(slices, m), dim3(kThreads), 0, stream, G, ldg, d, slices, slice_len, partial);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (3 candidates, 12527 tokens: 20 us with 256 threads a candidate)
  if (n > 1024)
    hipLaunchKernelGGL(score_logprobs_kernel<1024>, dim3(m), dim3(1024), 0, stream, logp_x, logp, ldp, n, labels, partial, slices, rho, scores);
  else
    hipLaunchKernelGGL(score_logprobs_kernel<256>, dim3(m), dim3(256), 0, stream, logp_x, logp, ldp, n, labels, partial, slices, rho, scores);
  return hipGetLastError();
}

}  // namespace zeno
