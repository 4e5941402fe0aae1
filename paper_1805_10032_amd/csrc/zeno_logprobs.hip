// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and their gradient.
//
// With M = max z and s = sum exp(z - M):   log p_j = (z_j - M) - log s,   H = log s - (1/s) sum exp(z - M) (z - M).
// One pass over a row: every thread keeps a reference c (in units of log2, within one of its running maximum) and the sums of
// 2^(L z - c) and of 2^(L z - c) (L z - c), L = log2 e, so a value costs one FMA and one exponential.
#include "zeno_tokens.h"

#include <float.h>

#include <algorithm>

namespace zeno {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kThreads = 256;
constexpr int kNarrow = 256;       // values of a row that sixteen lanes hold
constexpr int kCandidates = 512;   // top values are chosen from at most so many
constexpr int kMaxParts = 64;      // workgroups that share a row

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// (written out: fmaxf would first quiet every operand that might be a signalling NaN, an instruction a value; such a NaN takes the value
// beside it out of the maximum, so a thread that has met a NaN, as its sum shows, looks for its maxima again)
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
template <int N>
__device__ inline float max_of(const float (&v)[N], float m) {
#pragma unroll
  for (int j = 0; j < N; j += 2) m = max3(v[j], v[j + 1], m);
  return m;
}
__device__ inline float finite(float x) { return fminf(fmaxf(x, -FLT_MAX), FLT_MAX); }

// What a row, or a part of it, comes to: s and t relative to the largest logit M.
struct RowSums {
  float M, s, t;   // max, sum 2^(L(z-M)), sum 2^(L(z-M)) L(z-M)
};

// A thread's sums relative to a reference that is `delta` lower (delta = old reference - new one).  What lies 2^-100 below the new
// reference adds nothing to it, and is left out rather than scaled: a thread that has met nothing but masks of a size where the reference
// L z has no fraction left holds 2^(its rounding) there, up to infinity, which 0 would make NaN.  (Infinity would last through steps of
// less than 100, but from 2^31, where the rounding reaches 128, down to ordinary logits there are more of them than a thread has pieces.  The
// sums are NaN only next to a NaN.)
template <bool ENT>
__device__ inline void move_by(float& s, float& t, float delta) {
  if (delta > -100.f) {
    const float r = exp2_fast(delta);
    if (ENT) t = r * fmaf(s, delta, t);
    s *= r;
  } else {
    s = s == s ? 0.f : s;
    if (ENT) t = s;
  }
}

// The sums of two parts relative to M >= part.M.
__device__ inline void move_to(RowSums& p, float M) {
  if (p.s != 0.f && p.M < M) {
    const float delta = fmaxf((p.M - M) * kLog2e, -1e4f), r = exp2_fast(delta);
    p.t = r * fmaf(p.s, delta, p.t);
    p.s *= r;
  }
  p.M = M;
}

// A row whose logits are all -inf has no distribution: nothing can be drawn from it.
__device__ inline bool is_empty(float M, float s) { return M == -__builtin_inff() && s == 0.f; }

__device__ inline float log_prob(float z, float M, float log_s, bool empty) {
  return empty ? -__builtin_inff() : (z - M) - log_s;
}

__device__ inline float clean(float z) { return z != z ? -__builtin_inff() : z; }   // a NaN ranks as -inf
template <int N>
__device__ inline float clean_max_of(const float (&v)[N], float m) {
#pragma unroll
  for (int j = 0; j < N; ++j) m = fmaxf(m, clean(v[j]));
  return m;
}

// Writes what a row gives, except its alternatives.  One thread.
template <typename T>
__device__ inline void finish_row(const LogprobsArgs& a, int row, RowSums r, float* log_s_out) {
  if (r.M == __builtin_inff()) r.s = __builtin_nanf("");   // inf - inf
  const bool empty = is_empty(r.M, r.s);
  const float log_s = empty ? 0.f : logf(r.s);
  if (a.stats) {
    a.stats[2LL * row] = r.M;
    a.stats[2LL * row + 1] = log_s;
  }
  if (a.entropy) a.entropy[row] = empty ? 0.f : log_s - kLn2 * (r.t / r.s);
  if (a.logp) {
    const int y = a.labels[row];
    float lp = 0.f;   // label -1: the token does not count
    if (y != -1)
      lp = y >= 0 && y < a.vocab
               ? log_prob((float)reinterpret_cast<const T*>(a.logits)[(long long)row * a.ldz + y], r.M, log_s, empty)
               : __builtin_nanf("");
    a.logp[row] = lp;
  }
  *log_s_out = log_s;
}

// NW waves for a row (or a part of it): a workgroup is four rows of one wave each, or one row of four or sixteen.
template <int NW>
struct Shape {
  static constexpr int TPR = 64 * NW, ROWS = NW == 1 ? 4 : 1, THREADS = TPR * ROWS, WAVES = THREADS / 64;
  // maxima that a thread keeps of its share of the row, for the search of the top values
  static constexpr int GROUPS = NW == 16 ? 4 : 16;
};
template <typename T, int NW, bool TOP>
struct Shared {
  static constexpr int TPR = 64 * NW, ROWS = Shape<NW>::ROWS, WAVES = Shape<NW>::WAVES, GROUPS = Shape<NW>::GROUPS;
  float wave_max[WAVES], wave_s[WAVES], wave_t[WAVES];
  float log_s[ROWS];
  float group_max[TOP ? ROWS : 1][TOP ? GROUPS : 1][TOP ? TPR : 1];
  __align__(16) float thread_max[TOP ? ROWS : 1][TOP ? TPR : 4];
  int count[ROWS], ties[WAVES];
  float cand_val[TOP ? ROWS : 1][TOP ? kCandidates : 1];
  int cand_idx[TOP ? ROWS : 1][TOP ? kCandidates : 1];
  float best_val[WAVES];
  int best_idx[WAVES];
};

template <typename T>
__device__ inline void load_at(const T* row, int n, int i, float (&v)[Wide<T>::N]) {
  if (i + Wide<T>::N <= n)
    load_wide(row + i, v);
  else
    load_part(row + i, n - i, -__builtin_inff(), v);
}

// The k largest of row[0..n), ties to the lower index, in order, handed to put(rank, value, index).  k <= n, k <= TPR.
// Every thread kept the maxima of kGroups groups of its values while it read the row.  The k-th largest of 64 lanes' maxima is no larger
// than the k-th largest value, so only groups that reach it are read again: about k of them.
template <typename T, int NW, typename Put>
__device__ inline void top_values(Shared<T, NW, true>& sh, int slot, const T* row, int n, int iters, int per_group, int k, int tid,
                                  Put put) {
  constexpr int N = Wide<T>::N, TPR = 64 * NW;
  const int lane = tid & 63, wave = slot * NW + tid / 64;   // (tid counts from the row's first thread)
  if (tid == 0) sh.count[slot] = 0;
  float mine = sh.thread_max[slot][lane];   // of the lane's threads in all waves: 64 maxima bound the k-th value about as well as 256
#pragma unroll
  for (int w = 1; w < NW; ++w) mine = fmaxf(mine, sh.thread_max[slot][64 * w + lane]);
  row_sync<NW>();
  if (tid < 64) sh.thread_max[slot][lane] = mine;
  row_sync<NW>();
  int larger = 0;
#pragma unroll
  for (int i = 0; i < 64; i += 4) {
    const float4 o = *reinterpret_cast<const float4*>(&sh.thread_max[slot][i]);
    larger += (o.x > mine ? 1 : 0) + (o.y > mine ? 1 : 0) + (o.z > mine ? 1 : 0) + (o.w > mine ? 1 : 0);
  }
  const float tau = -wave_max_f(larger < k ? -mine : -__builtin_inff());   // the smallest of those that fewer than k exceed: the k-th
  float v[N];
  auto collect = [&](bool ties) {
    for (int g = 0; g * per_group < iters; ++g) {
      if (sh.group_max[slot][g][tid] < tau) continue;
      for (int it = g * per_group; it < iters && it < (g + 1) * per_group; ++it) {
        const int at = (it * TPR + tid) * N;
        if (at >= n) break;
        load_at(row, n, at, v);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float c = clean(v[j]);
          if (at + j < n && (ties ? c >= tau : c > tau)) {
            const int pos = atomicAdd(&sh.count[slot], 1);
            if (pos < kCandidates) {
              sh.cand_val[slot][pos] = c;
              sh.cand_idx[slot][pos] = at + j;
            }
          }
        }
      }
    }
  };
  collect(true);
  row_sync<NW>();
  int found = sh.count[slot];
  if (found > kCandidates) {
    // Many values equal to tau (masked rows, rows of few values): only the larger ones, then the first of the equal ones.
    row_sync<NW>();
    if (tid == 0) sh.count[slot] = 0;
    row_sync<NW>();
    collect(false);
    row_sync<NW>();
    found = sh.count[slot];
    if (found > kCandidates) {
      // The largest values crowd in the shares of few threads: one pass over the row for each of the k.
      float last = __builtin_inff();
      int last_idx = -1;
      for (int r = 0; r < k; ++r) {
        float bv = 0.f;
        int bi = -1;
        for (int it = 0; it < iters; ++it) {
          const int at = (it * TPR + tid) * N;
          if (at >= n) break;
          load_at(row, n, at, v);
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const float c = clean(v[j]);
            const bool after = c < last || (c == last && at + j > last_idx);
            if (at + j < n && after && (bi < 0 || c > bv)) {
              bv = c;
              bi = at + j;
            }
          }
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
          const float ov = __shfl_xor(bv, off, 64);
          const int oi = __shfl_xor(bi, off, 64);
          if (oi >= 0 && (bi < 0 || ov > bv || (ov == bv && oi < bi))) {
            bv = ov;
            bi = oi;
          }
        }
        if (NW > 1) {
          if (lane == 0) {
            sh.best_val[wave] = bv;
            sh.best_idx[wave] = bi;
          }
          __syncthreads();
          for (int w = 0; w < NW; ++w) {
            const float ov = sh.best_val[w];
            const int oi = sh.best_idx[w];
            if (oi >= 0 && (bi < 0 || ov > bv || (ov == bv && oi < bi))) {
              bv = ov;
              bi = oi;
            }
          }
          __syncthreads();
        }
        if (tid == 0) put(r, bv, bi);
        last = bv;
        last_idx = bi;
      }
      return;
    }
    if (found < k) {
      // the first (k - found) values equal to tau, in order of their index
      int have = found;
      for (int it = 0; it < iters && have < k; ++it) {
        const int at = (it * TPR + tid) * N;
        int eq = 0;
        if (at < n) {
          load_at(row, n, at, v);
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (at + j < n && clean(v[j]) == tau) eq |= 1 << j;
        }
        const int cnt = __popc(eq);
        int before = cnt;   // inclusive prefix over the lanes
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
          const int o = __shfl_up(before, off, 64);
          if (lane >= off) before += o;
        }
        int total = __shfl(before, 63, 64);
        before -= cnt;
        if (NW > 1) {
          if (lane == 0) sh.ties[wave] = total;
          __syncthreads();
          total = 0;
          for (int w = 0; w < NW; ++w) {
            if (w < wave) before += sh.ties[w];
            total += sh.ties[w];
          }
          __syncthreads();
        }
        int pos = have + before;
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (eq >> j & 1) {
            if (pos < k) {
              sh.cand_val[slot][pos] = tau;
              sh.cand_idx[slot][pos] = at + j;
            }
            ++pos;
          }
        have += total;
      }
      found = have < k ? have : k;
      row_sync<NW>();
    }
  }
  for (int i = tid; i < found; i += TPR) {
    const float c = sh.cand_val[slot][i];
    const int ci = sh.cand_idx[slot][i];
    int better = 0;
    for (int j = 0; j < found; ++j) {
      const float o = sh.cand_val[slot][j];
      better += (o > c || (o == c && sh.cand_idx[slot][j] < ci)) ? 1 : 0;
    }
    if (better < k) put(better, c, ci);
  }
}

// Partial results of a row that several workgroups share.
struct Parts {
  float* sums;   // [rows][parts][3]
  float* val;    // [rows][parts][top]
  int* idx;      // (-1: the part has fewer values)
  int parts;     // 1: the kernel writes the results itself
  int len;       // values of a part
};

// Reads every logit once; the alternatives are found in a second look at the few pieces whose maximum is large enough.  8192 x 32768 bf16 with
// entropy: 95 us (5.6 TB/s): the vector pipes are busy for 75 % of it, an FMA and an exponential at a quarter of the rate for every value
// and two more for the entropy.  2047 x 50257 float32 with five alternatives and entropy: 80 us (5.1 TB/s).  One row of 32000 with eight: 10 us,
// the round trips of the row's loads, two reductions over sixteen waves, the candidates and their ranks, one behind the other.
template <typename T, int NW, bool TOP, bool ENT>
__global__ __launch_bounds__(Shape<NW>::THREADS) void logprobs_kernel(LogprobsArgs a, Parts w) {
  constexpr int N = Wide<T>::N, TPR = 64 * NW, RPB = Shape<NW>::ROWS;
  __shared__ Shared<T, NW, TOP> sh;
  const int slot = threadIdx.x / TPR, tid = threadIdx.x % TPR, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int part = blockIdx.y;
  const int begin = part * w.len;
  const int n = a.vocab - begin < w.len ? a.vocab - begin : w.len;
  const int iters = (n + TPR * N - 1) / (TPR * N);
  const int per_group = (iters + Shape<NW>::GROUPS - 1) / Shape<NW>::GROUPS;
  const long long blocks = ((long long)a.rows + RPB - 1) / RPB;
  for (long long b = blockIdx.x; b < blocks; b += gridDim.x) {
    const long long r64 = b * RPB + slot;
    const bool live = r64 < a.rows;
    const int rowi = live ? (int)r64 : a.rows - 1;   // (a wave behind the last row repeats it and writes nothing)
    const T* row = reinterpret_cast<const T*>(a.logits) + (long long)rowi * a.ldz + begin;
    const float inf = __builtin_inff();
    float M = -inf, lim = -inf, c = 0.f, s = 0.f, t = 0.f;
    float v[N];
    // one 16-byte piece
    auto take = [&](const float (&v)[N]) __attribute__((always_inline)) {
      const float cm = max_of<N>(v, -inf);
      if (cm > lim) {
        const float cn = finite(cm * kLog2e);
        if (s != 0.f) move_by<ENT>(s, t, c - cn);
        c = cn;
        lim = cm + 0.6875f;   // the reference follows when it is a factor of two behind
      }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float d = fmaf(v[j], kLog2e, -c), e = exp2_fast(d);
        s += e;
        if (ENT) t = fmaf(e, fmaxf(d, -1e30f), t);   // (0 * -inf would be NaN)
      }
      return cm;
    };
    // Four pieces on their way at a time; pieces [from, to) of the thread.
    auto run = [&](int from, int to) __attribute__((always_inline)) {
      constexpr int kAhead = 4;
      float gm = -inf;
      int it = from;
      const int whole = n / N > tid ? (n / N - tid + TPR - 1) / TPR : 0;   // the thread's pieces that lie inside the row
      for (; it + kAhead <= to && it + kAhead <= whole; it += kAhead) {
        typename Wide<T>::type raw[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
          raw[i] = *reinterpret_cast<const typename Wide<T>::unaligned*>(row + ((it + i) * TPR + tid) * N);
        __builtin_amdgcn_sched_barrier(0);   // (or the first one's values would be waited for before the last is sent)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
#pragma unroll
          for (int j = 0; j < N; ++j) v[j] = (float)raw[i][j];
          const float cm = take(v);
          gm = max3(gm, cm, cm);
        }
      }
      for (; it < to; ++it) {
        const int at = (it * TPR + tid) * N;
        if (at >= n) break;
        load_at(row, n, at, v);
        const float cm = take(v);
        gm = max3(gm, cm, cm);
      }
      return gm;
    };
    if constexpr (TOP) {
      for (int g = 0; g * per_group < iters; ++g) {
        const float gm = clean(run(g * per_group, (g + 1) * per_group < iters ? (g + 1) * per_group : iters));
        sh.group_max[slot][g][tid] = gm;
        M = fmaxf(M, gm);
      }
      sh.thread_max[slot][tid] = M;
    } else {
      M = clean(run(0, iters));
    }
    if (s != s) {
      M = -inf;
      for (int it = 0, g = 0, end = per_group; it < iters; end += per_group, ++g) {
        float gm = -inf;
        for (; it < end && it < iters; ++it) {
          const int at = (it * TPR + tid) * N;
          if (at < n) {
            load_at(row, n, at, v);
            gm = clean_max_of<N>(v, gm);
          }
        }
        if constexpr (TOP) sh.group_max[slot][g][tid] = gm;
        M = fmaxf(M, gm);
      }
      if constexpr (TOP) sh.thread_max[slot][tid] = M;
    }
    // the row's maximum, and every thread's sums relative to it
    const float own_max = M;
    M = wave_max_f(M);
    if (NW > 1) {
      if (lane == 0) sh.wave_max[wave] = M;
      __syncthreads();
      for (int i = 0; i < NW; ++i) M = fmaxf(M, sh.wave_max[i]);
    }
    if (fabsf(M) > 0x1p24f && fabsf(M) < inf) {
      // L M is rounded by more than 1, which all of the row's values would carry in their exponents, or out of range (a row masked
      // throughout, whatever the mask's value): once more with z - M first
      s = t = 0.f;
      for (int it = 0; it < iters; ++it) {
        const int at = (it * TPR + tid) * N;
        if (at >= n) break;
        load_at(row, n, at, v);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float d = (v[j] - M) * kLog2e, e = exp2_fast(d);
          s += e;
          if (ENT) t = fmaf(e, fmaxf(d, -1e30f), t);
        }
      }
    } else if (s != 0.f) {
      // c is L times some logit, rounded: the exact product with M's is what the sums refer to from here on
      move_by<ENT>(s, t, own_max == -inf ? 0.f : fmaf(-M, kLog2e, c));
    }
    s = wave_sum_f(s);
    if (ENT) t = wave_sum_f(t);
    if (NW > 1) {
      if (lane == 0) {
        sh.wave_s[wave] = s;
        sh.wave_t[wave] = t;
      }
      __syncthreads();
      s = sh.wave_s[0];
      t = sh.wave_t[0];
      for (int i = 1; i < NW; ++i) {
        s += sh.wave_s[i];
        t += sh.wave_t[i];
      }
    }
    if (w.parts > 1) {
      const long long p = (long long)rowi * w.parts + part;
      if (tid == 0 && live) {
        w.sums[3 * p] = M;
        w.sums[3 * p + 1] = s;
        w.sums[3 * p + 2] = t;
      }
      if constexpr (TOP) {
        const int k = a.top < n ? a.top : n;
        if (tid >= k && tid < a.top && live) w.idx[p * a.top + tid] = -1;
        row_sync<NW>();
        top_values<T, NW>(sh, slot, row, n, iters, per_group, k, tid, [&](int rank, float val, int idx) {
          if (!live) return;
          w.val[p * a.top + rank] = val;
          w.idx[p * a.top + rank] = begin + idx;
        });
      }
    } else {
      if (tid == 0) {
        float log_s = 0.f;
        const RowSums r = {M, s, t};
        if (live) finish_row<T>(a, rowi, r, &log_s);
        sh.log_s[slot] = log_s;
      }
      if constexpr (TOP) {
        row_sync<NW>();
        const float log_s = sh.log_s[slot];
        const bool empty = is_empty(M, s);
        top_values<T, NW>(sh, slot, row, n, iters, per_group, a.top, tid, [&](int rank, float val, int idx) {
          if (!live) return;
          a.top_index[(long long)rowi * a.top + rank] = idx;
          a.top_logp[(long long)rowi * a.top + rank] = log_prob(val, M, log_s, empty);   // (next to a NaN or +inf, log_s is NaN)
        });
      }
    }
    row_sync<NW>();   // the next row uses the same shared memory
  }
}

// Rows of a few values: sixteen lanes a row, which stays in registers; its alternatives are found one after the other.  65536 rows: 10 float32
// values 8.4 us, 200 bf16 values 8.8 us (3.0 TB/s), a launch and one round trip to memory; three alternatives of 200 cost 20 us more, a few
// instructions a value and alternative.
template <typename T, bool ENT, int PIECES>
__global__ __launch_bounds__(kThreads) void logprobs_narrow_kernel(LogprobsArgs a) {
  constexpr int N = Wide<T>::N;
  const int lane = threadIdx.x % 16;
  const float inf = __builtin_inff();
  auto reduce = [](float v, auto f) {
    v = f(v, dpp<kDppXor1>(v));
    v = f(v, dpp<kDppXor2>(v));
    v = f(v, dpp<kDppHalfMirror>(v));
    return f(v, dpp<kDppMirror>(v));
  };
  auto add = [](float x, float y) { return x + y; };
  const long long rows_up = ((long long)a.rows + 15) / 16 * 16;   // (whole workgroups: the lanes of a row stay together)
  for (long long r64 = (long long)blockIdx.x * (kThreads / 16) + threadIdx.x / 16; r64 < rows_up; r64 += (long long)gridDim.x * (kThreads / 16)) {
    const bool live = r64 < a.rows;
    const int rowi = live ? (int)r64 : a.rows - 1;
    const T* row = reinterpret_cast<const T*>(a.logits) + (long long)rowi * a.ldz;
    float v[PIECES][N], M = -inf, s = 0.f, t = 0.f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int at = (16 * p + lane) * N;
      load_at(row, a.vocab, at, v[p]);   // (-inf behind the row's end)
      M = max_of<N>(v[p], M);
    }
    M = reduce(clean(M), [](float x, float y) { return fmaxf(x, y); });
    const float ref = M > -inf ? M : 0.f;   // (a row of nothing but -inf)
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float d = (v[p][j] - ref) * kLog2e, e = exp2_fast(d);
        s += e;
        if (ENT) t = fmaf(e, fmaxf(d, -1e30f), t);
      }
    s = reduce(s, add);
    if (ENT) t = reduce(t, add);
    if (s != s) {   // (the lanes of a row agree)
      M = -inf;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) M = clean_max_of<N>(v[p], M);
      M = reduce(M, [](float x, float y) { return fmaxf(x, y); });
    }
    float log_s = 0.f;
    const RowSums r = {M, s, t};
    if (live && lane == 0) finish_row<T>(a, rowi, r, &log_s);
    if (a.top > 0) {
      if (M == inf) s = __builtin_nanf("");
      const bool empty = is_empty(M, s);
      log_s = __shfl(log_s, threadIdx.x % 64 - lane, 64);
      float last = inf;
      int last_idx = -1;
      for (int k = 0; k < a.top; ++k) {
        float best = -inf;
        int best_idx = 0x7fffffff;   // (behind the row's end are -inf of higher indices than the row's own: top <= vocab, they are not reached)
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const float c = clean(v[p][j]);
            const int idx = (16 * p + lane) * N + j;
            const bool after = c < last || (c == last && idx > last_idx);
            if (after && (c > best || (c == best && idx < best_idx))) {
              best = c;
              best_idx = idx;
            }
          }
        last = reduce(best, [](float x, float y) { return fmaxf(x, y); });
        int idx = best == last ? best_idx : 0x7fffffff;
        idx = min(idx, dpp_int<kDppXor1>(idx));
        idx = min(idx, dpp_int<kDppXor2>(idx));
        idx = min(idx, dpp_int<kDppHalfMirror>(idx));
        last_idx = min(idx, dpp_int<kDppMirror>(idx));
        if (live && lane == 0) {
          a.top_index[(long long)rowi * a.top + k] = last_idx;
          a.top_logp[(long long)rowi * a.top + k] = log_prob(last, M, log_s, empty);
        }
      }
    }
  }
}

// Joins the parts of a row: one workgroup of one wave a row.  What does not depend on each other is read at once.
template <typename T>
__global__ __launch_bounds__(64) void logprobs_join_kernel(LogprobsArgs a, Parts w) {
  __shared__ __align__(16) float cand_val[kMaxParts * 32];
  __shared__ int cand_idx[kMaxParts * 32];
  __shared__ int count;
  const int lane = threadIdx.x;
  const float inf = __builtin_inff();
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int k = a.top, all = w.parts * k;
    const long long p = row * w.parts + lane;
    RowSums r = {-inf, 0.f, 0.f};
    float head = -inf, first_val = 0.f;
    int first_idx = -1;
    if (lane < w.parts) {
      r = {w.sums[3 * p], w.sums[3 * p + 1], w.sums[3 * p + 2]};
      if (k > 0) head = w.val[p * k];   // (every part has a first value)
    }
    if (lane < all) {
      first_val = w.val[row * all + lane];
      first_idx = w.idx[row * all + lane];
    }
    if (lane == 0) count = 0;
    move_to(r, wave_max_f(r.M));
    r.s = wave_sum_f(r.s);
    r.t = wave_sum_f(r.t);
    float log_s = 0.f;
    if (lane == 0) finish_row<T>(a, (int)row, r, &log_s);
    log_s = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(log_s)));
    if (r.M == inf) r.s = __builtin_nanf("");
    if (k > 0) {
      const bool empty = is_empty(r.M, r.s);
      // the k-th largest of the parts' largest values bounds the k-th largest from below
      int larger = 0;
      for (int i = 0; i < w.parts; ++i) larger += __shfl(head, i, 64) > head ? 1 : 0;
      float tau = -inf;
      if (w.parts >= k) tau = -wave_max_f(lane < w.parts && larger < k ? -head : -inf);
      row_sync<1>();
      for (int i = lane; i < all; i += 64) {
        const float val = i < 64 ? first_val : w.val[row * all + i];
        const int idx = i < 64 ? first_idx : w.idx[row * all + i];
        if (idx >= 0 && val >= tau) {
          const int pos = atomicAdd(&count, 1);
          cand_val[pos] = val;
          cand_idx[pos] = idx;
        }
      }
      row_sync<1>();
      const int found = count;
      for (int i = lane; i < found; i += 64) {
        const float c = cand_val[i];
        const int ci = cand_idx[i];
        int better = 0;
        for (int j = 0; j < found; ++j) {
          const float o = cand_val[j];
          better += (o > c || (o == c && cand_idx[j] < ci)) ? 1 : 0;
        }
        if (better < k) {
          a.top_index[row * k + better] = ci;
          a.top_logp[row * k + better] = log_prob(c, r.M, log_s, empty);
        }
      }
      row_sync<1>();
    }
  }
}

// ---- gradient:  dz_j = g [j = y] + sum_k q_k [j = i_k] - p_j (g + sum_k q_k + h (log p_j + H))
// with g, h, q the gradients of logp, H and the alternatives' log probabilities.
// L threads a segment of a row (16, 64 or 256): 256 / L segments a workgroup.  Each logit is read and each gradient written once, with no
// reduction, so short segments and many workgroups keep the memory busy.  8192 x 32768 bf16: 187 us (5.7 TB/s), bound by memory.  (With
// ordinary stores 167 after a forward pass, which then takes 120 us instead of 95.)
template <typename T, bool ENT, bool TOP, int L>
__global__ __launch_bounds__(kThreads) void logprobs_grad_kernel(LogprobsGradArgs a, int segs, int seg_len) {
  constexpr int N = Wide<T>::N, EACH = kThreads / L;
  static_assert(!TOP || L >= 64, "every alternative has a thread");
  __shared__ int all_idx[EACH][32];
  __shared__ float all_g[EACH][32];
  const int slot = threadIdx.x / L, tid = threadIdx.x % L;
  int (&special_idx)[32] = all_idx[slot];
  float (&special_g)[32] = all_g[slot];
  const long long tiles = (long long)a.rows * segs;
  const float inf = __builtin_inff();
  // (whole workgroups go through the loop: a segment behind the last repeats it and writes nothing)
  for (long long first = (long long)blockIdx.x * EACH; first < tiles; first += (long long)gridDim.x * EACH) {
    const bool live = first + slot < tiles;
    const long long tile = live ? first + slot : tiles - 1;
    const long long row = segs == 1 ? tile : tile / segs;
    const int lo = (int)(tile - row * segs) * seg_len;
    const int n = a.vocab - lo < seg_len ? a.vocab - lo : seg_len;
    const T* z = reinterpret_cast<const T*>(a.logits) + row * a.ldz + lo;
    T* out = reinterpret_cast<T*>(a.dlogits) + row * a.ldd + lo;
    float M = a.stats[2 * row], log_s = a.stats[2 * row + 1];
    const bool empty = M == -inf && log_s == 0.f, past = a.large && on_line(out);
    int y = -1;
    float g = 0.f;
    if (a.grad_logp) {
      y = a.labels[row];
      if (y != -1) g = y >= 0 && y < a.vocab ? a.grad_logp[row] : __builtin_nanf("");
      if (y < 0 || y >= a.vocab) y = -1;
    }
    float sum = g;
    if (TOP) {
      if (tid < a.top) {
        const int idx = a.top_index[row * a.top + tid];
        const bool valid = idx >= 0 && idx < a.vocab;
        special_idx[tid] = valid ? idx : -1;
        special_g[tid] = valid ? a.grad_top[row * a.top + tid] : __builtin_nanf("");
      }
      __syncthreads();
      for (int i = 0; i < a.top; ++i) sum += special_g[i];
    }
    const float h = ENT ? a.grad_entropy[row] : 0.f;
    const float base = ENT ? fmaf(h, a.entropy[row], sum) : sum;
    if (empty) {
      M = 0.f;
      log_s = inf;   // every probability is 0
    }
    // (where p is 0, its logarithm is cut off: 0 * -inf would be NaN)
    auto grad = [&](float v) {
      const float lp = (v - M) - log_s, p = exp2_fast(lp * kLog2e);
      return -p * (ENT ? fmaf(h, fmaxf(lp, -256.f), base) : base);
    };
    // the alternatives' columns of this segment, before anything is overwritten (dlogits may be the logits)
    float kept = 0.f;
    int mine = -1;
    if (TOP && tid < a.top) {
      const int idx = special_idx[tid] - lo;
      if (idx >= 0 && idx < n) {
        mine = idx;
        kept = (float)z[idx];
      }
    }
    if (TOP) __syncthreads();
    if (live)
    for (int at = tid * N; at < n; at += L * N) {
      float v[N];
      if (at + N <= n)
        load_wide(z + at, v);
      else
        load_part(z + at, n - at, -inf, v);
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = grad(v[j]);
      const int hit = y - lo - at;
      if (hit >= 0 && hit < N && !empty) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j == hit) v[j] += g;
      }
      if (at + N <= n && past)
        store_wide_past(out + at, v);
      else if (at + N <= n)
        store_wide(out + at, v);
      else
        store_part(out + at, n - at, v);
    }
    if (TOP) {
      __syncthreads();   // the segment is written: its special columns once more, with all that falls on them
      if (mine >= 0 && !empty && live) {
        float d = grad(kept);
        if (mine == y - lo) d += g;
        for (int i = 0; i < a.top; ++i)
          if (special_idx[i] - lo == mine) d += special_g[i];
        out[mine] = (T)d;
      }
      __syncthreads();
    }
  }
}

// Rows of up to 2048 values take one wave; longer ones four, and sixteen where there are too few rows to fill the chip with four
// (bf16, eight alternatives, us with sixteen waves / with four, which share a row of more than 8192 values between them: 1 x 32000
// 12.4 / 17.0, 256 x 32000 14.3 / 19.0, 400 x 50257 29.4 / 29.8).
bool wave_rows(int vocab) { return vocab <= 2048; }
bool few_rows(int rows) { return rows < 512; }

// Workgroups that share a row, at most one for each compute unit in all.  The join costs a launch, which rows of up to 65536 values do
// not bring in again (shared / whole: 1 x 65536 15.8 / 15.7, 1 x 131072 16.1 / 21.7, 64 x 131072 21.1 / 24.0).
int row_parts(int rows, int vocab) {
  if (vocab <= 65536 || rows > 128 || rows < 1) return 1;
  const int parts = 256 / rows, most = vocab / 8192;
  return std::min(std::min(parts, most), kMaxParts);
}

Parts parts_for(int rows, int vocab, int top, void* workspace) {
  Parts w;
  w.parts = row_parts(rows, vocab);
  const long long unit = 1024 * 8;   // whole 16-byte loads in every part, whatever the type
  w.len = (int)(((vocab + w.parts - 1LL) / w.parts + unit - 1) / unit * unit);
  if (w.parts == 1) w.len = vocab;
  w.parts = w.parts == 1 ? 1 : (int)((vocab + (long long)w.len - 1) / w.len);   // (none of them empty)
  const size_t n = (size_t)rows * w.parts;
  unsigned char* base = reinterpret_cast<unsigned char*>(workspace);
  w.sums = reinterpret_cast<float*>(base);
  base += align_up(n * 3 * sizeof(float), 256);
  w.val = reinterpret_cast<float*>(base);
  base += align_up(n * top * sizeof(float), 256);
  w.idx = reinterpret_cast<int*>(base);
  return w;
}

template <typename T, int NW>
void start(const LogprobsArgs& a, const Parts& w, dim3 grid, hipStream_t stream) {
  const dim3 block(Shape<NW>::THREADS);
  const bool ent = a.entropy != nullptr;
  if (a.top > 0 && ent) hipLaunchKernelGGL((logprobs_kernel<T, NW, true, true>), grid, block, 0, stream, a, w);
  else if (a.top > 0) hipLaunchKernelGGL((logprobs_kernel<T, NW, true, false>), grid, block, 0, stream, a, w);
  else if (ent) hipLaunchKernelGGL((logprobs_kernel<T, NW, false, true>), grid, block, 0, stream, a, w);
  else hipLaunchKernelGGL((logprobs_kernel<T, NW, false, false>), grid, block, 0, stream, a, w);
}

template <typename T>
hipError_t launch_type(const LogprobsArgs& a, const Parts& w, hipStream_t stream) {
  if (a.vocab <= kNarrow) {
    const int blocks = ceil_div(a.rows, kThreads / 16);
    const dim3 grid(blocks < 8192 ? blocks : 8192);
    constexpr int MOST = kNarrow / (16 * Wide<T>::N);
    const bool one = a.vocab <= 16 * Wide<T>::N;   // a piece a lane is all of the row (65536 x 16 float32, sixteen alternatives: 132 -> 42 us)
    if (one && a.entropy != nullptr) hipLaunchKernelGGL((logprobs_narrow_kernel<T, true, 1>), grid, dim3(kThreads), 0, stream, a);
    else if (one) hipLaunchKernelGGL((logprobs_narrow_kernel<T, false, 1>), grid, dim3(kThreads), 0, stream, a);
    else if (a.entropy != nullptr) hipLaunchKernelGGL((logprobs_narrow_kernel<T, true, MOST>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((logprobs_narrow_kernel<T, false, MOST>), grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  }
  const int rpb = wave_rows(a.vocab) ? Shape<1>::ROWS : 1;
  const long long blocks = ((long long)a.rows + rpb - 1) / rpb;
  const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)), w.parts);
  if (wave_rows(a.vocab)) start<T, 1>(a, w, grid, stream);
  else if (few_rows(a.rows)) start<T, 16>(a, w, grid, stream);
  else start<T, 4>(a, w, grid, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || w.parts == 1) return e;
  hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3(a.rows), dim3(64), 0, stream, a, w);
  return hipGetLastError();
}

template <typename T, int L>
hipError_t start_grad(const LogprobsGradArgs& a, hipStream_t stream) {
  const int seg_len = L * Wide<T>::N * 4;
  const int segs = ceil_div(a.vocab, seg_len), each = kThreads / L;
  const long long blocks = ((long long)a.rows * segs + each - 1) / each;
  const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), block(kThreads);
  const bool ent = a.grad_entropy != nullptr, top = a.grad_top != nullptr && a.top > 0;
  if constexpr (L >= 64) {
    if (ent && top) hipLaunchKernelGGL((logprobs_grad_kernel<T, true, true, L>), grid, block, 0, stream, a, segs, seg_len);
    else if (top) hipLaunchKernelGGL((logprobs_grad_kernel<T, false, true, L>), grid, block, 0, stream, a, segs, seg_len);
  }
  if (ent && !top) hipLaunchKernelGGL((logprobs_grad_kernel<T, true, false, L>), grid, block, 0, stream, a, segs, seg_len);
  else if (!top) hipLaunchKernelGGL((logprobs_grad_kernel<T, false, false, L>), grid, block, 0, stream, a, segs, seg_len);
  return hipGetLastError();
}

// Short rows share a workgroup.
template <typename T>
hipError_t launch_grad_type(const LogprobsGradArgs& a, hipStream_t stream) {
  if (a.vocab <= kNarrow && a.grad_top == nullptr) return start_grad<T, 16>(a, stream);
  if (a.vocab <= 64 * Wide<T>::N * 4) return start_grad<T, 64>(a, stream);
  return start_grad<T, 256>(a, stream);
}

}  // namespace

size_t logprobs_workspace_bytes(int rows, int vocab, int top) {
  const Parts w = parts_for(rows, vocab, top, nullptr);
  if (w.parts == 1) return 256;
  const size_t n = (size_t)rows * w.parts;
  return align_up(n * 3 * sizeof(float), 256) + 2 * align_up(n * top * sizeof(float), 256);
}

hipError_t launch_logprobs(const LogprobsArgs& a, void* workspace, hipStream_t stream) {
  const Parts w = parts_for(a.rows, a.vocab, a.top, workspace);
  switch (a.dtype) {
    case ZENO_F32: return launch_type<float>(a, w, stream);
    case ZENO_BF16: return launch_type<__bf16>(a, w, stream);
    default: return launch_type<_Float16>(a, w, stream);
  }
}

hipError_t launch_logprobs_backward(const LogprobsGradArgs& a, hipStream_t stream) {
  switch (a.dtype) {
    case ZENO_F32: return launch_grad_type<float>(a, stream);
    case ZENO_BF16: return launch_grad_type<__bf16>(a, stream);
    default: return launch_grad_type<_Float16>(a, stream);
  }
}

}  // namespace zeno
