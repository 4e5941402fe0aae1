// Layer norm and its backward pass; the weights' gradients are summed per group of rows (a worker's tokens).
//
//   xh = (x - mean) rstd,  y = weight xh + bias,  rstd = 1 / sqrt(var + eps)
//   a = weight dy,  dx = rstd (a - mean(a) - xh mean(a xh)),  dweight_g = sum_{rows of g} dy xh,  dbias_g = sum dy
//
// A row stays in registers between its statistics and its result: x is read once.  Threads own columns: the weights are read once into LDS,
// and the sums of their gradients stay in registers from row to row.  The variance is the mean of squared differences from the mean, not
// the difference of two large sums.
#include "zeno_tokens.h"

#include <type_traits>

namespace zeno {
namespace {

// NW waves for a row; a workgroup has four waves at least, of which one-wave rows use one each.
template <int NW>
struct Shape {
  static constexpr int TPR = 64 * NW, THREADS = NW < 4 ? 256 : TPR, RPB = THREADS / TPR;
  // Which of the workgroup's rows is a thread's (the same for a wave, so that a row's address needs no registers of the lanes).
  static __device__ inline int slot() { return RPB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : 0; }
};

// Sums over the threads of a row.  The buffers alternate from row to row, so one barrier is enough: a buffer is written again
// behind the barrier of the row between, which every wave reaches after it has read it.
template <int NW>
__device__ inline void row_sums2(float& a, float& b, float (*buf)[2], int wave) {
  a = wave_sum_f(a);
  b = wave_sum_f(b);
  if (NW > 1) {
    if ((threadIdx.x & 63) == 0) {
      buf[wave][0] = a;
      buf[wave][1] = b;
    }
    __syncthreads();
    a = buf[0][0];
    b = buf[0][1];
#pragma unroll
    for (int i = 1; i < NW; ++i) {
      a += buf[i][0];
      b += buf[i][1];
    }
  }
}
template <int NW>
__device__ inline float row_sum1(float a, float (*buf)[2], int wave) {
  a = wave_sum_f(a);
  if (NW > 1) {
    if ((threadIdx.x & 63) == 0) buf[wave][0] = a;
    __syncthreads();
    a = buf[0][0];
#pragma unroll
    for (int i = 1; i < NW; ++i) a += buf[i][0];
  }
  return a;
}

template <typename T>
__device__ inline void load_cols(const T* row, int col, int width, float (&v)[Wide<T>::N]) {
  if (col + Wide<T>::N <= width)
    load_wide(row + col, v);
  else
    load_part(row + col, width - col, 0.f, v);
}
template <typename T>
__device__ inline void store_cols(T* row, int col, int width, const float (&v)[Wide<T>::N]) {
  if (col + Wide<T>::N <= width)
    store_wide(row + col, v);
  else
    store_part(row + col, width - col, v);
}
template <int N>
__device__ inline void load_params(const float* p, int col, int width, float (&v)[N]) {
  typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
  if (p != nullptr && col + N <= width) {
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const f4 q = *reinterpret_cast<const f4*>(p + col + j);
      v[j] = q.x;
      v[j + 1] = q.y;
      v[j + 2] = q.z;
      v[j + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = p != nullptr && col + j < width ? p[col + j] : 0.f;
  }
}

template <typename T>
__device__ inline void store_cols_past(bool past, T* row, int col, int width, const float (&v)[Wide<T>::N]) {
  if (past && col + Wide<T>::N <= width)
    store_wide_past(row + col, v);
  else
    store_cols(row, col, width, v);
}
// The 8-bit copy of N columns of a row (a block's columns lie in neighbouring lanes).  Every lane of the wave takes part.
template <int N>
__device__ inline void keep_cols(const float (&v)[N], int col, int width, int blocks, uint8_t* values, uint8_t* scales, long long row) {
  float q[N];
  const int k = ckpt_quotients<N>(v, q);
  if (col < blocks * kCkptBlock) {
    uint8_t* p = values + row * ((long long)blocks * kCkptBlock) + col;
#pragma unroll
    for (int j = 0; j < N; j += 4) *reinterpret_cast<unsigned*>(p + j) = ckpt_pack4(q[j], q[j + 1], q[j + 2], q[j + 3]);
    if (col % kCkptBlock == 0) scales[row * blocks + col / kCkptBlock] = (uint8_t)(k + 127);
  }
}

// Keeps the compiler from holding the unpacked values of a row from one pass over it to the next: unpacking again costs an instruction a
// value, holding them costs the registers of a second workgroup.
template <typename V>
__device__ inline void unpack_again(V& v) {
  asm volatile("" : "+v"(v));
}

// A thread's part of a row as it lies in memory: CH 16-byte pieces, the c-th at column (c * TPR + tid) * N.  Pieces behind the row's end
// are its first columns once more, and one that the end cuts is the row's last N columns: so all of them are whole loads behind no
// branch, and cut() puts the right values (and zeros) in their place when they are used.
template <typename T, int TPR, int CH>
struct RowPart {
  typename Wide<T>::type raw[CH];
  __device__ inline void load(const T* row, int tid, int width) {
    constexpr int N = Wide<T>::N;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * TPR + tid) * N;
      if (TPR * CH == 64 && width < N) {   // (wider launches have wider rows)
#pragma unroll
        for (int j = 0; j < N; ++j) raw[c][j] = row[j < width ? j : 0];
      } else {
        const unsigned at = col + N <= width ? col : (col < width ? width - N : 0);
        raw[c] = *reinterpret_cast<const typename Wide<T>::unaligned*>(reinterpret_cast<const char*>(row) + at * (unsigned)sizeof(T));
      }
    }
  }
  __device__ inline void again() {
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (CH * Wide<T>::N >= 32) unpack_again(raw[c]);
  }
  __device__ inline void get(int c, int tid, int width, float (&v)[Wide<T>::N]) const {
    constexpr int N = Wide<T>::N;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = (float)raw[c][j];
    if ((c + 1) * TPR * N > width) cut<N>((c * TPR + tid) * N, width, v);
  }
  __device__ inline void centred(int c, int tid, int width, float mean, float (&v)[Wide<T>::N]) const {
    get(c, tid, width, v);
#pragma unroll
    for (int j = 0; j < Wide<T>::N; ++j) v[j] -= mean;
  }
  template <int N>
  static __device__ inline void cut(int col, int width, float (&v)[N]) {
    const int have = width - col;   // columns of this piece
    if (have >= N) return;
    const int shift = width < N ? 0 : N - width % N;
#pragma unroll
    for (int by = N / 2; by > 0; by /= 2)
      if (shift & by) {
#pragma unroll
        for (int j = 0; j + by < N; ++j) v[j] = v[j + by];
      }
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j >= have) v[j] = 0.f;
  }
};

// Weights in LDS, in the order in which the lanes read them: four floats a lane next to the neighbour's.
template <int N, int TPR, int CH>
struct Params {
  static constexpr int SIZE = CH * N * TPR;
  __device__ static inline void fill(float* to, const float* from, int width) {
    for (int i = threadIdx.x; i < SIZE; i += blockDim.x) {
      const int j = i % 4, lane = i / 4 % TPR, h = i / (4 * TPR) % (N / 4), c = i / (4 * TPR) / (N / 4);
      const int col = (c * TPR + lane) * N + 4 * h + j;
      to[i] = from != nullptr && col < width ? from[col] : 0.f;
    }
  }
  __device__ static inline void get(const float* p, int c, int tid, float (&v)[N]) {
#pragma unroll
    for (int h = 0; h < N / 4; ++h) {
      const float4 q = *reinterpret_cast<const float4*>(p + ((c * (N / 4) + h) * TPR + tid) * 4);
      v[4 * h] = q.x;
      v[4 * h + 1] = q.y;
      v[4 * h + 2] = q.z;
      v[4 * h + 3] = q.w;
    }
  }
};

// The next row is on its way while a row is reduced (the one after it as well: 72 -> 75 us).  Bound by memory and by what a row's two
// reductions leave idle.  16384 x 4096 bf16 with a checkpoint 63 us (5.3 TB/s; plain streams of this mix reach 6.2), without one 51 us (5.3 TB/s);
// 5003 x 1001 float32 11.5 us (3.5 TB/s), a launch and two round trips; 7634 x 6144 bf16 49 us, with a quarter of the threads idle.
template <typename T, int NW, int CH>
__global__ __launch_bounds__(Shape<NW>::THREADS) void norm_kernel(NormArgs a) {
  constexpr int N = Wide<T>::N, TPR = Shape<NW>::TPR, RPB = Shape<NW>::RPB;
  typedef Params<N, TPR, CH> P;
  __shared__ float buf[2][NW][2];
  __shared__ __align__(16) float weight[P::SIZE], bias[P::SIZE];
  const int tid = threadIdx.x % TPR, slot = Shape<NW>::slot(), wave = tid / 64;
  const int blocks = ckpt_blocks(a.width);
  const float inv = 1.f / (float)a.width;
  P::fill(weight, a.weight, a.width);
  P::fill(bias, a.bias, a.width);
  __syncthreads();
  const long long step = (long long)gridDim.x * RPB;
  long long row = (long long)blockIdx.x * RPB + slot;
  if (row >= a.rows) return;
  const T* x = reinterpret_cast<const T*>(a.x);
  RowPart<T, TPR, CH> now, next;
  now.load(x + row * a.ldx, tid, a.width);
  for (; row < a.rows; row += step) {
    next.load(x + (row + step < a.rows ? row + step : row) * a.ldx, tid, a.width);
    float sum = 0.f, v[N];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      now.get(c, tid, a.width, v);
#pragma unroll
      for (int j = 0; j < N; ++j) sum += v[j];
    }
    const float mean = row_sum1<NW>(sum, buf[0], wave) * inv;
    float sq = 0.f;
    now.again();
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      now.get(c, tid, a.width, v);
      const int have = a.width - (c * TPR + tid) * N;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float d = v[j] - mean;
        if ((c + 1) * TPR * N <= a.width || j < have) sq = fmaf(d, d, sq);
      }
    }
    const float var = row_sum1<NW>(sq, buf[1], wave) * inv;
    const float rstd = 1.f / sqrtf(var + a.eps);
    T* y = reinterpret_cast<T*>(a.y) + row * a.ldy;
    now.again();
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * TPR + tid) * N;
      now.get(c, tid, a.width, v);
      if (a.values != nullptr) keep_cols<N>(v, col, a.width, blocks, a.values, a.scales, row);
      float w[N], b[N];
      P::get(weight, c, tid, w);
      P::get(bias, c, tid, b);
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = fmaf((v[j] - mean) * rstd, w[j], b[j]);
      store_cols(y, col, a.width, v);
    }
    if (tid == 0) {
      if (a.mean != nullptr) a.mean[row] = mean;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
    now = next;
  }
}

// The pieces of a row that 1024 threads go over: f(column, whole), whole pieces AT_ONCE at a time so that their loads are on their way
// together, then the one that the row's end cuts.
template <int N, int AT_ONCE, typename F>
__device__ inline void over_row(int width, int tid, F f) {
  constexpr int TPR = 1024;
  const int whole = width / (TPR * N);
#pragma unroll AT_ONCE
  for (int c = 0; c < whole; ++c) f((c * TPR + tid) * N, std::true_type());
  if (whole * TPR * N < width) f((whole * TPR + tid) * N, std::false_type());
}
template <bool WHOLE, typename T>
__device__ inline void load_cols(const T* row, int col, int width, float (&v)[Wide<T>::N]) {
  if (WHOLE)
    load_wide(row + col, v);
  else
    load_cols(row, col, width, v);
}

// Rows too wide for the registers: read once for the mean, once for the variance and once for the result, from the caches
// where they hold the row.  2000 x 40000 bf16: 100 us (3.2 TB/s of one read and one write; piece after piece 333 us).
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  constexpr int N = Wide<T>::N;
  __shared__ float buf[2][16][2];
  const int tid = threadIdx.x, wave = tid / 64;
  const int blocks = ckpt_blocks(a.width);
  const float inv = 1.f / (float)a.width;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* __restrict__ x = reinterpret_cast<const T*>(a.x) + row * a.ldx;
    T* __restrict__ y = reinterpret_cast<T*>(a.y) + row * a.ldy;
    float sum = 0.f, sq = 0.f;
    over_row<N, 4>(a.width, tid, [&](int col, auto whole) __attribute__((always_inline)) {
      float v[N];
      load_cols<decltype(whole)::value>(x, col, a.width, v);
#pragma unroll
      for (int j = 0; j < N; ++j) sum += v[j];
    });
    const float mean = row_sum1<16>(sum, buf[0], wave) * inv;
    over_row<N, 4>(a.width, tid, [&](int col, auto whole) __attribute__((always_inline)) {
      float v[N];
      load_cols<decltype(whole)::value>(x, col, a.width, v);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float d = v[j] - mean;
        if (decltype(whole)::value || col + j < a.width) sq = fmaf(d, d, sq);
      }
    });
    const float rstd = 1.f / sqrtf(row_sum1<16>(sq, buf[1], wave) * inv + a.eps);
    // (one: a checkpoint's blocks are found by exchanges between lanes, which keep their order)
    over_row<N, 1>(a.width, tid, [&](int col, auto whole) __attribute__((always_inline)) {
      float v[N], w[N], b[N];
      load_cols<decltype(whole)::value>(x, col, a.width, v);
      if (a.values != nullptr) keep_cols<N>(v, col, a.width, blocks, a.values, a.scales, row);
      load_params(a.weight, col, a.width, w);
      load_params(a.bias, col, a.width, b);
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = fmaf((v[j] - mean) * rstd, w[j], b[j]);
      store_cols(y, col, a.width, v);
    });
    if (tid == 0) {
      if (a.mean != nullptr) a.mean[row] = mean;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
  }
}

// ---- backward.  Workgroup c takes rows [c * chunk, (c + 1) * chunk), whatever groups they belong to: the work is even however ragged
// the groups are.  Its sums for group g go to slot c + g: walking down the rows, every new piece raises c or g, so no two pieces share
// a slot, and a group's slots are its chunks' numbers plus g.  Sums are added in that order: the same bits every time.
struct Pieces {
  float* partial;   // [chunks + m][2][width]
  int chunk, chunks;
};

__device__ inline int first_group(const int32_t* offsets, int m, int row, int rows) {
  int g = 0;
  if (offsets == nullptr) return 0;
  for (int i = 0; i < m; i += blockDim.x) {
    const int at = i + (int)threadIdx.x;
    g += __syncthreads_count(at < m && group_offset(offsets, at + 1, rows) <= row);
  }
  return __builtin_amdgcn_readfirstlane(g);
}

// xh of N columns, from the row itself or from its checkpoint
template <typename T, bool KEPT, bool WHOLE>
__device__ inline void load_xh(const NormGradArgs& a, long long row, int col, int blocks, float mean, float rstd, float (&v)[Wide<T>::N]) {
  constexpr int N = Wide<T>::N;
  if (KEPT) {
    if (WHOLE || col < blocks * kCkptBlock) {
      unsigned words[N / 4];
      const uint8_t* p = a.values + row * ((long long)blocks * kCkptBlock) + col;
#pragma unroll
      for (int j = 0; j < N / 4; ++j) words[j] = reinterpret_cast<const unsigned*>(p)[j];
      ckpt_unpack(words, ckpt_scale((int)a.scales[row * blocks + col / kCkptBlock] - 127), v);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = 0.f;
    }
  } else {
    load_cols<WHOLE>(reinterpret_cast<const T*>(a.x) + row * a.ldx, col, a.width, v);
  }
  // (0 behind the row's end, also where mean rstd is out of range: infinity times dy's 0 would be NaN)
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = WHOLE || col + j < a.width ? (v[j] - mean) * rstd : 0.f;
}

// The same of a checkpoint, whose rows end with zeros in whole blocks.
template <typename T, int TPR, int CH>
struct KeptPart {
  unsigned words[CH][Wide<T>::N / 4];
  uint8_t scale[CH];
  __device__ inline void load(const uint8_t* values, const uint8_t* scales, long long row, int blocks, int tid) {
    constexpr int N = Wide<T>::N;
    const uint8_t* v = values + row * ((long long)blocks * kCkptBlock);
    const uint8_t* s = scales + row * blocks;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * TPR + tid) * N;
      const unsigned at = col < blocks * kCkptBlock ? col : 0;
#pragma unroll
      for (int j = 0; j < N / 4; ++j) words[c][j] = reinterpret_cast<const unsigned*>(v + at)[j];
      scale[c] = s[at / kCkptBlock];
    }
  }
  __device__ inline void again() {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < Wide<T>::N / 4; ++j)
        if (CH * Wide<T>::N >= 32) unpack_again(words[c][j]);
  }
  // (q scale is exact, and so is the difference where it cancels)
  __device__ inline void centred(int c, int, int, float mean, float (&v)[Wide<T>::N]) const {
    const float s = ckpt_scale((int)scale[c] - 127);
#pragma unroll
    for (int i = 0; i < Wide<T>::N; i += 4) {
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(words[c][i / 4], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(words[c][i / 4], true);
      v[i] = fmaf(lo.x, s, -mean);
      v[i + 1] = fmaf(lo.y, s, -mean);
      v[i + 2] = fmaf(hi.x, s, -mean);
      v[i + 3] = fmaf(hi.y, s, -mean);
    }
  }
};
template <typename T, int TPR, int CH, bool KEPT>
struct GradRow {
  RowPart<T, TPR, CH> dy;
  typename std::conditional<KEPT, KeptPart<T, TPR, CH>, RowPart<T, TPR, CH>>::type x;
  float mean, rstd;
  __device__ inline void load(const NormGradArgs& a, long long row, int blocks, int tid) {
    dy.load(reinterpret_cast<const T*>(a.dy) + row * a.lddy, tid, a.width);
    if constexpr (KEPT)
      x.load(a.values, a.scales, row, blocks, tid);
    else
      x.load(reinterpret_cast<const T*>(a.x) + row * a.ldx, tid, a.width);
    mean = a.mean[row];
    rstd = a.rstd[row];
  }
};

//
// A row's two sums and its result take two passes over its registers, which hold it as it lies in memory: unpacking it twice costs less than
// the registers of the values.  16384 x 4096 bf16: 82 us from a checkpoint (4.1 TB/s; the
// vector pipes are busy for 39 %, waves wait for 44 % of their time, at one barrier a row and for the memory); 5003 x 1001 float32
// 20 us (3.0 TB/s), 313 chunks that each add up four waves' sums.
template <typename T, int NW, int CH, bool KEPT>
__global__ __launch_bounds__(Shape<NW>::THREADS) void norm_grad_kernel(NormGradArgs a, Pieces p) {
  constexpr int N = Wide<T>::N, TPR = Shape<NW>::TPR, RPB = Shape<NW>::RPB;
  typedef Params<N, TPR, CH> P;
  __shared__ float buf[2][NW][2];
  __shared__ __align__(16) float weight[P::SIZE];
  __shared__ float joined[RPB > 1 ? 2 * CH * N * 64 : 1];
  const int tid = threadIdx.x % TPR, slot = Shape<NW>::slot(), wave = tid / 64;
  const int blocks = ckpt_blocks(a.width);
  const float inv = 1.f / (float)a.width;
  const int r0 = blockIdx.x * p.chunk, r1 = a.rows - r0 < p.chunk ? a.rows : r0 + p.chunk;
  P::fill(weight, a.weight, a.width);
  if (a.offsets == nullptr) __syncthreads();   // (or the search for the first group has one)
  // (16384 x 4096 bf16 85 -> 82 us, the next forward pass 68 -> 63; for rows of one wave the test costs what it may bring)
  const bool past = NW >= 4 && a.large && on_line(a.dx) && a.lddx * (long long)sizeof(T) % 128 == 0;
  int parity = 0;
  for (int g = first_group(a.offsets, a.m, r0, a.rows); g < a.m; ++g) {
    const int begin = group_offset(a.offsets, g, a.rows), end = group_offset(a.offsets, g + 1, a.rows);
    if (begin >= r1) break;
    const int lo = begin > r0 ? begin : r0, hi = end < r1 ? end : r1;
    if (lo >= hi) continue;
    float dw[CH][N], db[CH][N];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < N; ++j) dw[c][j] = db[c][j] = 0.f;
    // Two rows are on their way while a third is reduced (one: 92 instead of 84 us at 4096 bf16 columns).  With more values a thread there
    // are registers for one, and with 32 values and eight waves for none, where a row that is on its way would be spilled (2000 x 12000
    // fp32: 89 us, 189 with one).
    constexpr int AHEAD = CH * N <= 16 ? 2 : NW == 8 && CH * N >= 32 ? 0 : 1;
    GradRow<T, TPR, CH, KEPT> now, next, after;
    if (lo + slot < hi) {
      if (AHEAD > 0) now.load(a, lo + slot, blocks, tid);
      if (AHEAD == 2) next.load(a, lo + slot + RPB < hi ? lo + slot + RPB : lo + slot, blocks, tid);
    }
    for (int row = lo + slot; row < hi; row += RPB) {
      if (AHEAD == 2) after.load(a, row + 2 * RPB < hi ? row + 2 * RPB : row, blocks, tid);
      if (AHEAD == 0) now.load(a, row, blocks, tid);
      if (AHEAD == 1) next.load(a, row + RPB < hi ? row + RPB : row, blocks, tid);
      const float mean = now.mean, rstd = now.rstd;
      // x - mean in the row's sum, and rstd behind it: columns behind the row's end, where dy is 0, hold -mean, which is finite where
      // mean rstd need not be
      float c1 = 0.f, c2 = 0.f, d[N], u[N], w[N];
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        now.dy.get(c, tid, a.width, d);
        now.x.centred(c, tid, a.width, mean, u);
        P::get(weight, c, tid, w);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          db[c][j] += d[j];
          dw[c][j] = fmaf(d[j], u[j] * rstd, dw[c][j]);
          const float t = d[j] * w[j];
          c1 += t;
          c2 = fmaf(t, u[j], c2);
        }
      }
      if (a.dx != nullptr) {
        row_sums2<NW>(c1, c2, buf[parity], wave);
        parity ^= 1;
        c1 *= inv * -rstd;
        c2 = rstd == 0.f ? 0.f : c2 * rstd * (inv * -rstd);   // (a variance out of range: the sum may be, too)
        T* dx = reinterpret_cast<T*>(a.dx) + (long long)row * a.lddx;
        now.dy.again();
        now.x.again();
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          now.dy.get(c, tid, a.width, d);
          now.x.centred(c, tid, a.width, mean, u);
          P::get(weight, c, tid, w);
#pragma unroll
          for (int j = 0; j < N; ++j) d[j] = fmaf(d[j] * w[j], rstd, fmaf(u[j] * rstd, c2, c1));
          store_cols_past(past, dx, (c * TPR + tid) * N, a.width, d);
        }
      }
      if (AHEAD > 0) now = next;
      if (AHEAD == 2) next = after;
    }
    float* out = p.partial + (long long)(blockIdx.x + g) * 2 * a.width;
    if (RPB > 1) {
      // the waves' sums, one wave after the other
      for (int s = 0; s < RPB; ++s) {
        if (slot == s) {
#pragma unroll
          for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < N; ++j) {
              const int at = (c * N + j) * 64 + tid;
              joined[at] = s == 0 ? dw[c][j] : joined[at] + dw[c][j];
              joined[CH * N * 64 + at] = s == 0 ? db[c][j] : joined[CH * N * 64 + at] + db[c][j];
            }
        }
        __syncthreads();
      }
      for (int i = threadIdx.x; i < a.width; i += Shape<NW>::THREADS) {
        const int c = i / (64 * N), lane = i / N % 64, at = (c * N + i % N) * 64 + lane;
        out[i] = joined[at];
        out[a.width + i] = joined[CH * N * 64 + at];
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + tid) * N;
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (col + j < a.width) {
            out[col + j] = dw[c][j];
            out[a.width + col + j] = db[c][j];
          }
      }
    }
  }
}

// Rows too wide for the registers: dx from two reads of the row (2000 x 40000 bf16, both kernels and the join: 299 us, from a checkpoint 254) ...
template <typename T, bool KEPT>
__global__ __launch_bounds__(1024) void norm_grad_long_dx_kernel(NormGradArgs a) {
  constexpr int N = Wide<T>::N;
  __shared__ float buf[2][16][2];
  const int tid = threadIdx.x, wave = tid / 64;
  const int blocks = ckpt_blocks(a.width);
  const float inv = 1.f / (float)a.width;
  const int first = group_offset(a.offsets, 0, a.rows), last = group_offset(a.offsets, a.offsets == nullptr ? 1 : a.m, a.rows);
  int parity = 0;
  for (long long row = first + (long long)blockIdx.x; row < last; row += gridDim.x) {
    const float mean = a.mean[row], rstd = a.rstd[row];
    const T* dy = reinterpret_cast<const T*>(a.dy) + row * a.lddy;
    T* dx = reinterpret_cast<T*>(a.dx) + row * a.lddx;
    float c1 = 0.f, c2 = 0.f;
    over_row<N, 4>(a.width, tid, [&](int col, auto whole) __attribute__((always_inline)) {
      float xh[N], d[N], w[N];
      load_cols<decltype(whole)::value>(dy, col, a.width, d);
      load_xh<T, KEPT, decltype(whole)::value>(a, row, col, blocks, mean, rstd, xh);
      load_params(a.weight, col, a.width, w);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        c1 = fmaf(d[j], w[j], c1);
        c2 = fmaf(d[j] * w[j], xh[j], c2);
      }
    });
    row_sums2<16>(c1, c2, buf[parity], wave);
    parity ^= 1;
    c1 *= inv;
    c2 *= inv;
    // (dx may be dy: a piece's loads come before its store)
    over_row<N, 4>(a.width, tid, [&](int col, auto whole) __attribute__((always_inline)) {
      float xh[N], d[N], w[N];
      load_cols<decltype(whole)::value>(dy, col, a.width, d);
      load_xh<T, KEPT, decltype(whole)::value>(a, row, col, blocks, mean, rstd, xh);
      load_params(a.weight, col, a.width, w);
#pragma unroll
      for (int j = 0; j < N; ++j) d[j] = rstd * (d[j] * w[j] - fmaf(xh[j], c2, c1));
      store_cols(dx, col, a.width, d);
    });
  }
}

// ... and the weights' gradients by columns: 1024 threads' columns of the rows of a chunk, four rows on their way together.
template <typename T, bool KEPT, bool WHOLE>
__device__ inline void long_weights(const NormGradArgs& a, int lo, int hi, int col, int blocks, float (&dw)[Wide<T>::N], float (&db)[Wide<T>::N]) {
  constexpr int N = Wide<T>::N;
#pragma unroll 4
  for (int row = lo; row < hi; ++row) {
    float d[N], xh[N];
    load_cols<WHOLE>(reinterpret_cast<const T*>(a.dy) + (long long)row * a.lddy, col, a.width, d);
    load_xh<T, KEPT, WHOLE>(a, row, col, blocks, a.mean[row], a.rstd[row], xh);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      db[j] += d[j];
      dw[j] = fmaf(d[j], xh[j], dw[j]);
    }
  }
}
template <typename T, bool KEPT>
__global__ __launch_bounds__(1024) void norm_grad_long_weights_kernel(NormGradArgs a, Pieces p) {
  constexpr int N = Wide<T>::N;
  const int blocks = ckpt_blocks(a.width);
  const int col = (int)(blockIdx.y * 1024 + threadIdx.x) * N;
  const int r0 = blockIdx.x * p.chunk, r1 = a.rows - r0 < p.chunk ? a.rows : r0 + p.chunk;
  for (int g = first_group(a.offsets, a.m, r0, a.rows); g < a.m; ++g) {
    const int begin = group_offset(a.offsets, g, a.rows), end = group_offset(a.offsets, g + 1, a.rows);
    if (begin >= r1) break;
    const int lo = begin > r0 ? begin : r0, hi = end < r1 ? end : r1;
    if (lo >= hi) continue;
    float dw[N], db[N];
#pragma unroll
    for (int j = 0; j < N; ++j) dw[j] = db[j] = 0.f;
    if (col + N <= a.width)
      long_weights<T, KEPT, true>(a, lo, hi, col, blocks, dw, db);
    else
      long_weights<T, KEPT, false>(a, lo, hi, col, blocks, dw, db);
    float* out = p.partial + (long long)(blockIdx.x + g) * 2 * a.width;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (col + j < a.width) {
        out[col + j] = dw[j];
        out[a.width + col + j] = db[j];
      }
  }
}

// A group's gradient: its slots.  64 columns (of weights and biases together) a workgroup; a wave takes every so-manieth slot, and the waves'
// sums are added in their order.  33 groups of 1001 columns 4 us, 64 of 4096 (19 MB) 10 us; eight loads a thread on their way instead of four
// change neither.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(64 * kJoinWaves) void norm_grad_join_kernel(Pieces p, const int32_t* offsets, int rows, int width,
                                                                         float* __restrict__ dweight, float* __restrict__ dbias,
                                                                         long long ldw, long long ldb) {
  __shared__ float shared[kJoinWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, waves = blockDim.x / 64, g = blockIdx.y;
  const long long col = (long long)blockIdx.x * 64 + lane;
  const int begin = group_offset(offsets, g, rows), end = group_offset(offsets, g + 1, rows);
  float sum = 0.f;
  if (begin < end && col < 2LL * width) {
    const int c1 = (end - 1) / p.chunk;
#pragma unroll 4
    for (int c = begin / p.chunk + wave; c <= c1; c += waves) sum += p.partial[(long long)(c + g) * 2 * width + col];
  }
  shared[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && col < 2LL * width) {
    for (int w = 1; w < waves; ++w) sum += shared[w][lane];
    if (col < width) {
      if (dweight != nullptr) dweight[g * ldw + col] = sum;
    } else if (dbias != nullptr) {
      dbias[g * ldb + col - width] = sum;
    }
  }
}

// Rows of a chunk: 512 chunks of a large batch, two workgroups a compute unit (16384 x 4096 bf16 from a checkpoint: 84 us; 256 chunks 93,
// 768 105, because a third workgroup does not fit beside two); at least 16 rows, where the
// partial sums (8 bytes a column and chunk) are a tenth of what the rows themselves move, unless that leaves most of the chip without work.
int chunk_rows(int rows) {
  const int many = ceil_div(rows, 512), few = ceil_div(rows, 256);
  int c = few < 16 ? few : 16;
  if (many > c) c = many;
  return c < 1 ? 1 : c;
}

Pieces pieces_for(int rows, void* workspace) {
  Pieces p;
  p.partial = reinterpret_cast<float*>(workspace);
  p.chunk = chunk_rows(rows);
  p.chunks = ceil_div(rows, p.chunk);
  return p;
}

// The narrowest launch that holds a row: waves a row and 16-byte pieces a thread.  0 waves: the kernels for long rows, beyond 16384
// columns, whose weights and biases no longer fit LDS.  Beyond 512 threads' rows the backward pass takes more pieces a thread where the
// forward pass takes more threads: its sums stay in registers, of which 1024 threads have 128 each (4000 x 12000 bf16: 410 us).
void pick_shape(int width, int per_load, bool backward, int* nw, int* ch) {
  static const int shapes[][2] = {{1, 1}, {1, 2}, {1, 4}, {4, 2}, {8, 2}, {8, 4}, {8, 8}};
  for (const auto& s : shapes)
    if (64 * s[0] * s[1] * per_load <= 16384 && width <= 64 * s[0] * s[1] * per_load) {
      const bool spread = !backward && s[1] > 2 && s[0] > 1;
      *nw = spread ? 16 : s[0];
      *ch = spread ? s[1] / 2 : s[1];
      return;
    }
  *nw = 0;
  *ch = 0;
}

template <typename T, int NW, int CH>
void start_norm(const NormArgs& a, hipStream_t stream) {
  const long long need = ((long long)a.rows + Shape<NW>::RPB - 1) / Shape<NW>::RPB;
  const long long most = 256LL * 1024 / Shape<NW>::THREADS;   // what the chip holds with the weights in LDS: more workgroups would only fill it again
  hipLaunchKernelGGL((norm_kernel<T, NW, CH>), dim3((unsigned)(need < most ? need : most)), dim3(Shape<NW>::THREADS), 0, stream, a);
}

template <typename T>
hipError_t launch_norm_type(const NormArgs& a, hipStream_t stream) {
  int nw, ch;
  pick_shape(a.width, Wide<T>::N, false, &nw, &ch);
  if (nw == 1 && ch == 1) start_norm<T, 1, 1>(a, stream);
  else if (nw == 1 && ch == 2) start_norm<T, 1, 2>(a, stream);
  else if (nw == 1 && ch == 4) start_norm<T, 1, 4>(a, stream);
  else if (nw == 4 && ch == 2) start_norm<T, 4, 2>(a, stream);
  else if (nw == 8) start_norm<T, 8, 2>(a, stream);
  else if (nw == 16 && ch == 2) start_norm<T, 16, 2>(a, stream);
  else if (nw == 16) start_norm<T, 16, 16 / Wide<T>::N>(a, stream);   // (four pieces: float32 alone)
  else hipLaunchKernelGGL(norm_long_kernel<T>, dim3(a.rows < 512 ? a.rows : 512), dim3(1024), 0, stream, a);
  return hipGetLastError();
}

template <typename T, int NW, int CH, bool KEPT>
void start_grad(const NormGradArgs& a, const Pieces& p, hipStream_t stream) {
  hipLaunchKernelGGL((norm_grad_kernel<T, NW, CH, KEPT>), dim3(p.chunks), dim3(Shape<NW>::THREADS), 0, stream, a, p);
}

template <typename T, bool KEPT>
hipError_t launch_grad_type(const NormGradArgs& a, const Pieces& p, hipStream_t stream) {
  int nw, ch;
  pick_shape(a.width, Wide<T>::N, true, &nw, &ch);
  if (a.rows == 0) {
    // (no rows: the groups' gradients are zero)
  } else if (nw == 1 && ch == 1) start_grad<T, 1, 1, KEPT>(a, p, stream);
  else if (nw == 1 && ch == 2) start_grad<T, 1, 2, KEPT>(a, p, stream);
  else if (nw == 1 && ch == 4) start_grad<T, 1, 4, KEPT>(a, p, stream);
  else if (nw == 4 && ch == 2) start_grad<T, 4, 2, KEPT>(a, p, stream);
  else if (nw == 8 && ch == 2) start_grad<T, 8, 2, KEPT>(a, p, stream);
  else if (nw == 8 && ch == 4) start_grad<T, 8, 4, KEPT>(a, p, stream);
  else if (nw == 8) start_grad<T, 8, 32 / Wide<T>::N, KEPT>(a, p, stream);   // (eight pieces: float32 alone)
  else {
    // (the weights' gradients first: dx may be dy)
    if (a.dweight != nullptr || a.dbias != nullptr) {
      hipLaunchKernelGGL((norm_grad_long_weights_kernel<T, KEPT>), dim3(p.chunks, ceil_div(a.width, 1024 * Wide<T>::N)), dim3(1024), 0,
                         stream, a, p);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (a.dx != nullptr)
      hipLaunchKernelGGL((norm_grad_long_dx_kernel<T, KEPT>), dim3(a.rows < 512 ? a.rows : 512), dim3(1024), 0, stream, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (a.dweight == nullptr && a.dbias == nullptr)) return e;
  const int waves = p.chunks / a.m > 32 ? kJoinWaves : 4;   // (170 slots for four waves: 20 us)
  hipLaunchKernelGGL(norm_grad_join_kernel, dim3(ceil_div(2LL * a.width, 64), a.m), dim3(64 * waves), 0, stream, p, a.offsets, a.rows,
                     a.width, a.dweight, a.dbias, a.ldw, a.ldb);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_layer_norm(const NormArgs& a, hipStream_t stream) {
  switch (a.dtype) {
    case ZENO_F32: return launch_norm_type<float>(a, stream);
    case ZENO_BF16: return launch_norm_type<__bf16>(a, stream);
    default: return launch_norm_type<_Float16>(a, stream);
  }
}

size_t layer_norm_workspace_bytes(int rows, int width, int m) {
  const Pieces p = pieces_for(rows, nullptr);
  return align_up((size_t)(p.chunks + m) * 2 * width * sizeof(float), 256);
}

hipError_t launch_layer_norm_backward(const NormGradArgs& a, void* workspace, hipStream_t stream) {
  const Pieces p = pieces_for(a.rows, workspace);
  const bool kept = a.x == nullptr;
  switch (a.dtype) {
    case ZENO_F32: return kept ? launch_grad_type<float, true>(a, p, stream) : launch_grad_type<float, false>(a, p, stream);
    case ZENO_BF16: return kept ? launch_grad_type<__bf16, true>(a, p, stream) : launch_grad_type<__bf16, false>(a, p, stream);
    default: return kept ? launch_grad_type<_Float16, true>(a, p, stream) : launch_grad_type<_Float16, false>(a, p, stream);
  }
}

}  // namespace zeno
