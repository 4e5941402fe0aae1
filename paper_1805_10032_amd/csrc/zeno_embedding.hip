// Embedding lookup with a scale, out[t] = s E[id_t], and the table's gradient per group of rows (a worker's tokens),
//   dE_g[v] = s sum_{t in g, id_t = v} dy[t].
//
// The lookup is a copy.  The gradient sums rows that stand anywhere in the batch: tokens are sorted by (group, id), ties in their order, the
// sorted list is cut into pieces of equal length whatever ends in them, and a piece's sums that other pieces share go to slots, which a
// second launch joins in the pieces' order.  So no float is added by an atomic, equal calls give equal bits, and a token that
// half of the batch uses costs no more than any other.
#include "zeno_tokens.h"
#include <algorithm>

namespace zeno {
namespace {

template <typename T, int N>
struct Values {
  typedef T type __attribute__((ext_vector_type(N)));
  typedef type unaligned __attribute__((aligned(sizeof(T))));
};
template <typename T, int N>
__device__ inline void load_values(const T* p, float (&v)[N]) {
  const typename Values<T, N>::type raw = *reinterpret_cast<const typename Values<T, N>::unaligned*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (float)raw[i];
}

// ---- lookup: eight values a lane (one where a row has fewer), `lanes` lanes a row and column block, ROWS rows of a lane on their way at once.
// A row's last lane takes the last eight values, some of them its neighbour's too: both write the same.
// Rows of the output that start on memory lines are written row by row, past the caches from kPastBytes on (65536 of 50257 x 2048 float32 as bf16, 268
// MB: 70 us; row by row alone 96, column block by column block 111).  Others column block by column block (50001 x 777 float32: 31 us, row by row 37,
// past the caches 63).
template <typename T, typename O, int N, int ROWS, bool PAST>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, int lanes, unsigned blocks, unsigned groups, bool by_row) {
  const int lane = threadIdx.x % lanes, part = threadIdx.x / lanes, parts = 256 / lanes;
  const unsigned at = blockIdx.y * gridDim.x + blockIdx.x, block = by_row ? at % blocks : at / groups, group = by_row ? at / blocks : at % groups;
  const long long unit = (long long)block * lanes + lane;
  if (unit * N >= a.width) return;
  const long long col = unit * N < a.width - N ? unit * N : a.width - N;
  const long long first = ((long long)group * parts + part) * ROWS;
  int id[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) id[r] = first + r < a.rows ? a.ids[first + r] : -1;
  float v[ROWS][N];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const bool inside = id[r] >= 0 && id[r] < a.vocab;
    load_values<T, N>(reinterpret_cast<const T*>(a.table) + (inside ? id[r] : 0) * a.ldt + col, v[r]);
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const bool inside = id[r] >= 0 && id[r] < a.vocab;
    const float other = id[r] == -1 ? 0.f : __builtin_nanf("");
    typename Values<O, N>::type raw;
#pragma unroll
    for (int i = 0; i < N; ++i) raw[i] = (O)(inside ? v[r][i] * a.scale : other);
    if (first + r >= a.rows) continue;
    auto to = reinterpret_cast<typename Values<O, N>::unaligned*>(reinterpret_cast<O*>(a.out) + (first + r) * a.ldo + col);
    if (PAST) __builtin_nontemporal_store(raw, to);
    else *to = raw;
  }
}

template <typename T, typename O, int N>
hipError_t launch_embed(const EmbedArgs& a, hipStream_t stream) {
  const long long units = (a.width + N - 1LL) / N;
  int lanes = 1;
  while (lanes < 64 && lanes < units) lanes *= 2;
  const bool many = a.rows >= 8192;
  const long long rows_a_block = 256 / lanes * (many ? 4 : 1);
  const unsigned blocks = (unsigned)((units + lanes - 1) / lanes), groups = (unsigned)((a.rows + rows_a_block - 1) / rows_a_block);
  const bool lines = reinterpret_cast<uintptr_t>(a.out) % 128 == 0 && a.ldo * sizeof(O) % 128 == 0;
  const bool past = lines && a.width * sizeof(O) % 128 == 0 && (long long)a.rows * a.width * (long long)sizeof(O) >= kPastBytes;
  // (a dimension of a launch ends at 2^32 threads; workgroups behind the last find no row or no column)
  const long long all = (long long)blocks * groups;
  const unsigned x = (unsigned)std::min(all, 1LL << 22);
  const dim3 grid(x, (unsigned)((all + x - 1) / x));
  if (many && past) embed_kernel<T, O, N, 4, true><<<grid, 256, 0, stream>>>(a, lanes, blocks, groups, lines);
  else if (many) embed_kernel<T, O, N, 4, false><<<grid, 256, 0, stream>>>(a, lanes, blocks, groups, lines);
  else embed_kernel<T, O, N, 1, false><<<grid, 256, 0, stream>>>(a, lanes, blocks, groups, lines);
  return hipGetLastError();
}
template <typename T, typename O>
hipError_t launch_embed(const EmbedArgs& a, hipStream_t stream) {
  return a.width >= 8 ? launch_embed<T, O, 8>(a, stream) : launch_embed<T, O, 1>(a, stream);
}
template <typename T>
hipError_t launch_embed_from(const EmbedArgs& a, hipStream_t stream) {
  if (a.dtype == ZENO_F32) return launch_embed<T, float>(a, stream);
  if (a.dtype == ZENO_BF16) return launch_embed<T, __bf16>(a, stream);
  return launch_embed<T, _Float16>(a, stream);
}

// ---- tokens by (group, id)

constexpr int kSmallSort = 16384;       // tokens that one workgroup sorts in LDS
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSmallBits = 8, kLargeBits = 11;
constexpr int kChunkThreads = 512, kChunkWaves = kChunkThreads / 64;
constexpr int kMaxChunks = 1024;

// Key of a token: group * vocab + id; tokens of no group and ids outside the vocabulary come last.
__device__ inline unsigned token_key(const EmbedGradArgs& a, int t) {
  const unsigned none = (unsigned)a.m * (unsigned)a.vocab;
  const int id = a.ids[t];
  if (id < 0 || id >= a.vocab) return none;
  int g = 0;
  if (a.offsets != nullptr) {
    int lo = 0, hi = a.m;   // the last group that begins at t or before
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.offsets[mid] <= t) lo = mid;
      else hi = mid;
    }
    g = lo;
    if (t < a.offsets[g] || t >= a.offsets[g + 1]) return none;
  }
  return (unsigned)g * (unsigned)a.vocab + (unsigned)id;
}

// Lanes of the wave whose digit is this lane's, among the active ones.
template <int BITS>
__device__ inline unsigned long long same_digit(unsigned digit, bool active) {
  unsigned long long mask = __ballot(active);
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const unsigned long long set = __ballot(active && ((digit >> b) & 1));
    mask &= (digit >> b) & 1 ? set : ~set;
  }
  return mask;
}
__device__ inline void lds_order() {   // a wave's LDS accesses run in order: the compiler has to keep them so
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  __builtin_amdgcn_wave_barrier();
}

// The place of this lane's item: counter[digit], which the lanes before it that have the same digit come in front of.
template <int BITS>
__device__ inline unsigned place_of(unsigned* counter, unsigned digit, bool active, int lane) {
  const unsigned long long same = same_digit<BITS>(digit, active);
  const unsigned before = (unsigned)__popcll(same & ((1ULL << lane) - 1));
  unsigned at = 0;
  if (active) at = counter[digit];
  lds_order();
  if (active && before == 0) counter[digit] = at + (unsigned)__popcll(same);
  lds_order();
  return at + before;
}

// Clears piece `at` of all groups' rows, cut at memory lines.  A workgroup clears one piece, so that those that run lie near each other: 2.6 GB at 6.1
// TB/s beside the sort (pieces dealt to 2048 workgroups 5.1, stores past the caches 5.1 to 5.4).
__device__ inline void clear_part(const EmbedGradArgs& a, long long at) {
  const long long n = (long long)a.vocab * a.width, per = a.fill_pieces;
  const int g = (int)(at / per);
  const long long c = at % per;
  float* p = a.dtable + g * a.ldg;
  const long long off_line = (long long)((reinterpret_cast<unsigned long long>(p) & 127) / 4);
  const long long lo = c == 0 ? 0 : c * a.fill_floats - off_line;
  const long long hi = (c + 1) * a.fill_floats - off_line < n ? (c + 1) * a.fill_floats - off_line : n;
  long long whole = lo;
  if (c == 0) whole = off_line == 0 ? 0 : (32 - off_line < hi ? 32 - off_line : hi);
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const long long quads = hi > whole ? (hi - whole) / 4 : 0;
#pragma unroll 4
  for (long long q = threadIdx.x; q < quads; q += blockDim.x) reinterpret_cast<f32x4*>(p + whole)[q] = zero;
  if (lo + threadIdx.x < whole) p[lo + threadIdx.x] = 0.f;
  if (whole + 4 * quads + threadIdx.x < hi) p[whole + 4 * quads + threadIdx.x] = 0.f;
}

// Up to kSmallSort tokens: one workgroup, eight bits of the key a pass, a wave's consecutive items in registers between the passes; the other
// workgroups clear gradients meanwhile.
constexpr int kItems = kSmallSort / kSortThreads;
__global__ __launch_bounds__(kSortThreads) void embed_sort_small_kernel(EmbedGradArgs a, int passes) {
  if (blockIdx.x > 0) {
    clear_part(a, blockIdx.x - 1);
    return;
  }
  __shared__ unsigned key[kSmallSort];
  __shared__ unsigned short index[kSmallSort];
  __shared__ unsigned counter[kSortWaves][1 << kSmallBits];
  __shared__ unsigned total[1 << kSmallBits];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int per = ((a.rows + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;   // a wave's items are consecutive
  const int lo = wave * per < a.rows ? wave * per : a.rows, hi = lo + per < a.rows ? lo + per : a.rows;
  unsigned k[kItems];
  unsigned short x[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int t = lo + 64 * i + lane;
    k[i] = t < hi ? token_key(a, t) : 0;
    x[i] = (unsigned short)t;
  }
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * kSmallBits;
    unsigned* mine = counter[wave];
    for (int d = lane; d < 1 << kSmallBits; d += 64) mine[d] = 0;
    lds_order();
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if (lo + 64 * i + lane < hi) atomicAdd(&mine[(k[i] >> shift) & 255], 1u);
    __syncthreads();
    if (tid < 1 << kSmallBits) {
      unsigned sum = 0;
      for (int w = 0; w < kSortWaves; ++w) {
        const unsigned c = counter[w][tid];
        counter[w][tid] = sum;
        sum += c;
      }
      total[tid] = sum;
    }
    __syncthreads();
    if (wave == 0) {   // exclusive sums of the totals, four a lane
      unsigned v[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = sum;
        sum += total[4 * lane + i];
      }
      unsigned scan = sum;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const unsigned up = (unsigned)__shfl_up((int)scan, d);
        if (lane >= d) scan += up;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) total[4 * lane + i] = scan - sum + v[i];
    }
    __syncthreads();
    for (int d = lane; d < 1 << kSmallBits; d += 64) mine[d] += total[d];
    lds_order();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      if (lo + 64 * i >= hi) break;
      const bool active = lo + 64 * i + lane < hi;
      const unsigned at = place_of<kSmallBits>(mine, (k[i] >> shift) & 255, active, lane);
      if (active) {
        key[at] = k[i];
        index[at] = x[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int t = lo + 64 * i + lane;
      if (t < hi) {
        k[i] = key[t];
        x[i] = index[t];
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int t = lo + 64 * i + lane;
    if (t < hi) {
      a.key[0][t] = k[i];
      a.index[0][t] = x[i];
    }
  }
}

// More tokens: chunks of them, kLargeBits of the key a pass.  Counts of digit d in chunk c at count[d * chunks + c].
__device__ inline unsigned source_key(const EmbedGradArgs& a, int pass, int t) {
  return pass == 0 ? token_key(a, t) : a.key[(pass - 1) % 2][t];
}
__global__ __launch_bounds__(kChunkThreads) void embed_count_kernel(EmbedGradArgs a, int pass, int bits, int chunks, int chunk) {
  if ((int)blockIdx.x >= chunks) {
    clear_part(a, blockIdx.x - chunks);
    return;
  }
  __shared__ unsigned count[1 << kLargeBits];
  const int digits = 1 << bits;
  for (int d = threadIdx.x; d < digits; d += kChunkThreads) count[d] = 0;
  __syncthreads();
  const long long lo = (long long)blockIdx.x * chunk, hi = lo + chunk < a.rows ? lo + chunk : a.rows;
  for (long long t = lo + threadIdx.x; t < hi; t += kChunkThreads)
    atomicAdd(&count[(source_key(a, pass, (int)t) >> (pass * bits)) & (digits - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kChunkThreads) a.count[(long long)d * chunks + blockIdx.x] = count[d];
}
// One wave a digit: its chunks' counts become what the chunks before hold, and total[d] the digit's.
__global__ __launch_bounds__(256) void embed_scan_kernel(EmbedGradArgs a, int bits, int chunks) {
  const int d = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x % 64;
  if (d >= 1 << bits) return;
  unsigned before = 0;
  for (int c0 = 0; c0 < chunks; c0 += 64) {
    const unsigned n = c0 + lane < chunks ? a.count[(long long)d * chunks + c0 + lane] : 0;
    unsigned scan = n;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const unsigned up = (unsigned)__shfl_up((int)scan, s);
      if (lane >= s) scan += up;
    }
    if (c0 + lane < chunks) a.count[(long long)d * chunks + c0 + lane] = before + scan - n;
    before += (unsigned)__shfl((int)scan, 63);
  }
  if (lane == 0) a.total[d] = before;
}
__global__ __launch_bounds__(kChunkThreads) void embed_scatter_kernel(EmbedGradArgs a, int pass, int bits, int chunks, int chunk) {
  __shared__ unsigned counter[kChunkWaves][1 << kLargeBits];
  __shared__ unsigned base[1 << kLargeBits];
  __shared__ unsigned wave_total[kChunkWaves];
  constexpr int PER = (1 << kLargeBits) / kChunkThreads;   // digits a thread
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, digits = 1 << bits, shift = pass * bits;
  unsigned* mine = counter[wave];
  for (int d = lane; d < digits; d += 64) mine[d] = 0;
  lds_order();
  const long long begin = (long long)blockIdx.x * chunk, end = begin + chunk < a.rows ? begin + chunk : a.rows;
  const int per = chunk / kChunkWaves;   // (a multiple of 64) a wave's items are consecutive
  const long long lo = begin + (long long)wave * per < end ? begin + (long long)wave * per : end, hi = lo + per < end ? lo + per : end;
  for (long long t = lo + lane; t < hi; t += 64) atomicAdd(&mine[(source_key(a, pass, (int)t) >> shift) & (digits - 1)], 1u);
  {   // exclusive sums of the digits' totals
    unsigned v[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      v[i] = sum;
      const int d = tid * PER + i;
      sum += d < digits ? a.total[d] : 0;
    }
    unsigned scan = sum;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const unsigned up = (unsigned)__shfl_up((int)scan, s);
      if (lane >= s) scan += up;
    }
    if (lane == 63) wave_total[wave] = scan;
    __syncthreads();
    unsigned before = 0;
    for (int w = 0; w < wave; ++w) before += wave_total[w];
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (tid * PER + i < digits) base[tid * PER + i] = before + scan - sum + v[i];
  }
  __syncthreads();
  for (int d = tid; d < digits; d += kChunkThreads) {
    unsigned at = base[d] + a.count[(long long)d * chunks + blockIdx.x];
    for (int w = 0; w < kChunkWaves; ++w) {
      const unsigned c = counter[w][d];
      counter[w][d] = at;
      at += c;
    }
  }
  __syncthreads();
  for (long long t0 = lo; t0 < hi; t0 += 64) {
    const long long t = t0 + lane;
    const bool active = t < hi;
    const unsigned k = active ? source_key(a, pass, (int)t) : 0;
    const int i = active ? (pass == 0 ? (int)t : a.index[(pass - 1) % 2][t]) : 0;
    const unsigned at = place_of<kLargeBits>(mine, (k >> shift) & (digits - 1), active, lane);
    if (active) {
      a.key[pass % 2][at] = k;
      a.index[pass % 2][at] = i;
    }
  }
}

__global__ __launch_bounds__(256) void embed_clear_kernel(EmbedGradArgs a) { clear_part(a, blockIdx.x); }

// ---- sums of the sorted rows
// `lanes` lanes take a piece of the sorted tokens, N columns each; a row's last lane takes its last N columns and writes those that no other has.
// Sums that begin and end in the piece are written to the gradients; one that the piece before shares goes to the piece's first slot, one
// that only the next shares to its second.
constexpr int kAhead = 8;   // rows on their way

template <int N>
__device__ inline void add_to_table(const EmbedGradArgs& a, unsigned key, long long col, int skip, const float (&sum)[N]) {
  const unsigned g = key / (unsigned)a.vocab, v = key % (unsigned)a.vocab;
  float* to = a.dtable + g * a.ldg + (long long)v * a.width + col;
  float r[N];
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = sum[i] * a.scale;
  if (a.accumulate) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i >= skip) r[i] += to[i];
  }
  if (skip == 0) {
    typename Values<float, N>::type raw;
#pragma unroll
    for (int i = 0; i < N; ++i) raw[i] = r[i];
    *reinterpret_cast<typename Values<float, N>::unaligned*>(to) = raw;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i >= skip) to[i] = r[i];
  }
}

template <typename T, int N>
__global__ __launch_bounds__(256) void embed_grad_kernel(EmbedGradArgs a, int lanes, unsigned blocks, int source) {
  const int lane = threadIdx.x % lanes;
  const long long piece = (long long)(blockIdx.x / blocks) * (256 / lanes) + threadIdx.x / lanes;
  const long long unit = (long long)(blockIdx.x % blocks) * lanes + lane;
  if (piece >= a.pieces || unit * N >= a.width) return;
  const long long col = unit * N < a.width - N ? unit * N : a.width - N;
  const int skip = (int)(unit * N - col);
  const unsigned none = (unsigned)a.m * (unsigned)a.vocab;
  const unsigned* key = a.key[source];
  const int* index = a.index[source];
  const long long begin = piece * a.per_piece, end = begin + a.per_piece < a.rows ? begin + a.per_piece : a.rows;
  unsigned now = key[begin];
  if (now >= none) return;   // (they come last)
  bool shared = begin > 0 && key[begin - 1] == now;
  float sum[N] = {};
  auto put = [&](int slot) {
    float* to = a.slots + ((2 * piece + slot) * a.width + col);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i >= skip) to[i] = sum[i];
  };
  const T* dy = reinterpret_cast<const T*>(a.dy) + col;
  float v[kAhead][N];
  unsigned k[kAhead], k_next[kAhead];
  int row[kAhead];   // of the next rows: they are known when these have arrived
  auto look = [&](long long t0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const long long t = t0 + i < end ? t0 + i : end - 1;
      k_next[i] = key[t];
      row[i] = index[t];
    }
  };
  look(begin);
  for (long long t0 = begin; t0 < end; t0 += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      k[i] = k_next[i];
      load_values<T, N>(dy + (long long)row[i] * a.lddy, v[i]);
    }
    look(t0 + kAhead);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (t0 + i >= end) break;
      if (k[i] != now) {
        if (shared) put(0);
        else add_to_table<N>(a, now, col, skip, sum);
        shared = false;
        now = k[i];
        if (now >= none) return;
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] = v[i][j];
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += v[i][j];
      }
    }
  }
  if (shared) put(0);
  else if (end < a.rows && key[end] == now) put(1);
  else add_to_table<N>(a, now, col, skip, sum);
}

// Sums that several pieces share, by the workgroup of the piece where one begins: N columns a lane, the waves take consecutive pieces' slots.
constexpr int kJoinWaves = 8;
template <int N>
__global__ __launch_bounds__(64 * kJoinWaves) void embed_join_kernel(EmbedGradArgs a, int source) {
  __shared__ float part[kJoinWaves][64 * N];
  const unsigned* key = a.key[source];
  const unsigned none = (unsigned)a.m * (unsigned)a.vocab;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const long long piece = blockIdx.x, begin = piece * a.per_piece, next = begin + a.per_piece;
  if (next >= a.rows) return;
  const unsigned mine = key[next], last = key[next - 1], first = key[begin], before = begin > 0 ? key[begin - 1] : none;
  if (mine >= none || last != mine) return;
  if (first == mine && before == mine) return;   // began before
  // the first slots of pieces piece + 1 .. piece + count
  long long count = 1;
  for (;;) {
    const long long p = piece + 1 + count + lane;
    const unsigned long long has = __ballot(p < a.pieces && key[p * a.per_piece] == mine);
    const int run = has == ~0ULL ? 64 : __builtin_ctzll(~has);
    count += run;
    if (run < 64) break;
  }
  const long long per = (count + kJoinWaves - 1) / kJoinWaves;
  const long long from = piece + 1 + (wave * per < count ? wave * per : count), end = piece + 1 + count, to = from + per < end ? from + per : end;
  for (long long unit = lane; unit - lane < (a.width + N - 1) / N; unit += 64) {
    const bool live = unit * N < a.width;
    const long long col = unit * N < a.width - N ? unit * N : a.width - N;
    float sum[N] = {};
    if (live) {
      if (wave == 0) load_values<float, N>(a.slots + (2 * piece + 1) * a.width + col, sum);
#pragma unroll 8
      for (long long p = from; p < to; ++p) {
        float v[N];
        load_values<float, N>(a.slots + 2 * p * a.width + col, v);
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += v[i];
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) part[wave][i * 64 + lane] = sum[i];
    __syncthreads();
    if (wave == 0 && live) {
      for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += part[w][i * 64 + lane];
      add_to_table<N>(a, mine, col, (int)(unit * N - col), sum);
    }
    __syncthreads();
  }
}

struct Plan {
  int bits, passes, chunks, chunk;
  long long per_piece, pieces;
  size_t key[2], index[2], count, total, slots, bytes;
};
Plan plan_of(int rows, int vocab, int width, int m) {
  Plan p = {};
  int bits = 1;
  while (bits < 32 && ((unsigned long long)m * vocab >> bits) != 0) ++bits;   // the key of tokens that do not count is m * vocab
  if (rows <= kSmallSort) {
    p.passes = (bits + kSmallBits - 1) / kSmallBits;
    p.bits = kSmallBits;
  } else {
    p.passes = (bits + kLargeBits - 1) / kLargeBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    const long long chunks = std::min<long long>(kMaxChunks, (rows + 2047LL) / 2048);
    p.chunk = (int)((((long long)rows + chunks - 1) / chunks + kChunkThreads - 1) / kChunkThreads * kChunkThreads);
    p.chunks = (int)(((long long)rows + p.chunk - 1) / p.chunk);
  }
  // 32 tokens a piece, and no more than 2048 pieces, whose slots one workgroup may have to sum
  p.per_piece = std::max<long long>(32, (((long long)rows + 2047) / 2048 + 31) / 32 * 32);
  p.pieces = ((long long)rows + p.per_piece - 1) / p.per_piece;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  for (int i = 0; i < 2; ++i) {
    p.key[i] = take(4 * (size_t)rows);
    p.index[i] = take(4 * (size_t)rows);
  }
  p.count = take((size_t)4 * p.chunks << kLargeBits);
  p.total = take((size_t)4 << kLargeBits);
  p.slots = take((size_t)p.pieces * 2 * width * 4);
  p.bytes = at + 256;
  return p;
}

template <typename T, int N>
void launch_sums(const EmbedGradArgs& a, int source, hipStream_t stream) {
  const long long units = (a.width + N - 1LL) / N;
  int lanes = 1;
  while (lanes < 64 && lanes < units) lanes *= 2;
  const unsigned blocks = (unsigned)((units + lanes - 1) / lanes), groups = (unsigned)((a.pieces + 256 / lanes - 1) / (256 / lanes));
  embed_grad_kernel<T, N><<<groups * blocks, 256, 0, stream>>>(a, lanes, blocks, source);
}
template <typename T>
void launch_sums(const EmbedGradArgs& a, int source, hipStream_t stream) {
  if (a.width >= Wide<T>::N) launch_sums<T, Wide<T>::N>(a, source, stream);
  else launch_sums<T, 1>(a, source, stream);
}

}  // namespace

hipError_t launch_embedding(const EmbedArgs& a, hipStream_t stream) {
  if (a.table_dtype == ZENO_F32) return launch_embed_from<float>(a, stream);
  if (a.table_dtype == ZENO_BF16) return launch_embed_from<__bf16>(a, stream);
  return launch_embed_from<_Float16>(a, stream);
}

size_t embedding_workspace_bytes(int rows, int vocab, int width, int m) { return plan_of(rows, vocab, width, m).bytes; }

hipError_t launch_embedding_backward(EmbedGradArgs a, void* workspace, hipStream_t stream) {
  const Plan p = plan_of(a.rows, a.vocab, a.width, a.m);
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  for (int i = 0; i < 2; ++i) {
    a.key[i] = reinterpret_cast<unsigned*>(ws + p.key[i]);
    a.index[i] = reinterpret_cast<int*>(ws + p.index[i]);
  }
  a.count = reinterpret_cast<unsigned*>(ws + p.count);
  a.total = reinterpret_cast<unsigned*>(ws + p.total);
  a.slots = reinterpret_cast<float*>(ws + p.slots);
  a.pieces = p.pieces;
  a.per_piece = p.per_piece;
  const long long n = (long long)a.vocab * a.width;
  a.fill_floats = a.rows == 0 && n * a.m < 1LL << 33 ? 2048 : 32768;   // of workgroups of 256, 512 and 1024 threads
  a.fill_pieces = (n + 31 + a.fill_floats - 1) / a.fill_floats;   // (31: a part's place in its first line)
  const long long fills = a.accumulate ? 0 : a.fill_pieces * a.m;
  if (a.rows == 0) {
    if (fills > 0) embed_clear_kernel<<<(unsigned)fills, 256, 0, stream>>>(a);
    return hipGetLastError();
  }
  int source = 0;
  if (a.rows <= kSmallSort) {
    embed_sort_small_kernel<<<(unsigned)(1 + fills), kSortThreads, 0, stream>>>(a, p.passes);
  } else {
    const int scans = ((1 << p.bits) + 3) / 4;
    for (int pass = 0; pass < p.passes; ++pass) {   // the gradients are cleared beside the first launch
      embed_count_kernel<<<(unsigned)(p.chunks + (pass == 0 ? fills : 0)), kChunkThreads, 0, stream>>>(a, pass, p.bits, p.chunks, p.chunk);
      embed_scan_kernel<<<scans, 256, 0, stream>>>(a, p.bits, p.chunks);
      embed_scatter_kernel<<<p.chunks, kChunkThreads, 0, stream>>>(a, pass, p.bits, p.chunks, p.chunk);
    }
    source = (p.passes - 1) % 2;
  }
  if (a.dtype == ZENO_F32) launch_sums<float>(a, source, stream);
  else if (a.dtype == ZENO_BF16) launch_sums<__bf16>(a, source, stream);
  else launch_sums<_Float16>(a, source, stream);
  if (p.pieces > 1) {
    if (a.width >= 4) embed_join_kernel<4><<<(unsigned)(p.pieces - 1), 64 * kJoinWaves, 0, stream>>>(a, source);
    else embed_join_kernel<1><<<(unsigned)(p.pieces - 1), 64 * kJoinWaves, 0, stream>>>(a, source);
  }
  return hipGetLastError();
}

}  // namespace zeno
