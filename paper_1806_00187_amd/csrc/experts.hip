// Tokens sorted by expert and back: a counting sort of the choices (stable; integer counts alone are atomic), rows copied to their expert's, the weighted
// sum of a token's rows on the way back, and the gradients.  Bound by memory, the rows that are read and written once, and for few tokens by launches: up to
// kWhole choices the dispatch is one launch, in which every work-group counts all choices for itself; beyond that counts of segments and their sums over the segments before
// each are launches of their own (3 us each), and so are the rows.
// 105402 rows of 1024 bf16 to 64 experts and back: 123 us, 5.3 TB/s (a copy of a gigabyte: 5.2); 7168 of 512 fp16 to 16 experts with room for 8960: 11.6 us in the two kernels.
// A choice is an addition in LDS to its expert's count, so one-sided choices meet at one address: nine tenths of 7168 to one of 16 experts 7.9 -> 12.2 us of dispatch, of 16384 11.5 -> 21.9; of 105402,
// whose segments are counted once, 71.6 and 71.1.
#include "rowtypes.h"

#include <algorithm>
#include <type_traits>

namespace {

constexpr int kThreads = 256;
constexpr int kSegment = 1024;      // choices that share a row of counts
constexpr int kChunk = kWave;       // choices of a work-group of the dispatch, or fewer (spread)
constexpr int kWhole = 16384;       // up to so many choices every work-group of the dispatch counts all of them itself
constexpr int kSummed = 4096;       // up to so many counts of segments every work-group adds up itself (32768 choices to 64 experts and back 33.6 -> 31.4 us, 105402: 124 -> 127)
constexpr int kWholeThreads = 1024;
constexpr int kGroups = 256;        // a compute unit each
constexpr int64_t kCopied = 32 << 10;  // bytes that a work-group of kWholeThreads has in flight
constexpr int64_t kStreamFrom = 96 << 20;  // bytes of the experts' rows (large_rows)
// Fewer wavefronts than these leave compute units waiting: the columns of a token's row go to several.  16 tokens of 8 x 8192 bf16 to the experts and back 21.9 -> 9.8 us,
// 8000 of 4 x 4096 123 -> 118; gradients 46 -> 11.8 and 178 -> 164.
constexpr int kFewWaves = 8192;
constexpr int kMaxExperts = 1024, kMaxChoices = 64;
constexpr int64_t kMaxItems = 1 << 29;

typedef int32_t int4_any __attribute__((ext_vector_type(4), aligned(4)));

struct SortArgs {
  const int32_t* expert;
  int n, experts, capacity, segments, bits, chunk;
  Divisor by_experts;
  int32_t *hist, *totals, *slot, *ranges;
};

// f(index, expert) for the choices [begin, end) that have one, four a thread; a work-group.
template <typename F>
__device__ __forceinline__ void each_choice(const SortArgs& a, int begin, int end, F f) {
  for (int i = begin + 4 * threadIdx.x; i < end; i += 4 * blockDim.x) {
    int32_t id[4];
    if (i + 4 <= end) {
      const int4_any v = *reinterpret_cast<const int4_any*>(a.expert + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) id[e] = v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) id[e] = i + e < end ? a.expert[i + e] : -1;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if ((uint32_t)id[e] < (uint32_t)a.experts) f(i + e, id[e]);
  }
}

// Counts of the experts in every segment.  (Integer sums in LDS: their order does not show.)
__global__ void __launch_bounds__(kThreads) expert_count_kernel(const SortArgs a) {
  extern __shared__ int32_t counts[];
  for (int e = threadIdx.x; e < a.experts; e += kThreads) counts[e] = 0;
  __syncthreads();
  const int begin = blockIdx.x * kSegment;
  each_choice(a, begin, min(begin + kSegment, a.n), [&](int, int e) { atomicAdd(&counts[e], 1); });
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += kThreads) a.hist[(int64_t)blockIdx.x * a.experts + e] = counts[e];
}

// Counts of every segment -> counts of all segments before it, and the totals.  64 experts a work-group, a run of segments a wavefront.
constexpr int kScanWaves = 16;
__global__ void __launch_bounds__(kScanWaves* kWave) expert_scan_kernel(const SortArgs a) {
  __shared__ int32_t part[kScanWaves][kWave];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, e = blockIdx.x * kWave + lane;
  const int run = (a.segments + kScanWaves - 1) / kScanWaves, begin = min(wave * run, a.segments), end = min(begin + run, a.segments);
  int32_t* column = a.hist + min(e, a.experts - 1);
  int32_t s = 0;
  constexpr int AHEAD = 8;
  for (int r = begin; r < end; r += AHEAD) {
    int32_t v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) v[u] = column[(int64_t)min(r + u, end - 1) * a.experts];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) s += r + u < end ? v[u] : 0;
  }
  part[wave][lane] = s;
  __syncthreads();
  s = 0;
  for (int w = 0; w < wave; ++w) s += part[w][lane];
  if (e >= a.experts) return;
  if (wave == kScanWaves - 1) a.totals[e] = s + part[wave][lane];
  for (int r = begin; r < end; r += AHEAD) {
    int32_t v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) v[u] = column[(int64_t)min(r + u, end - 1) * a.experts];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (r + u < end) {
        column[(int64_t)(r + u) * a.experts] = s;
        s += v[u];
      }
  }
}

struct RowsArgs {
  const void *x, *rows, *add;
  void* out;
  int64_t ld_x, ld_rows, ld_add, ld_out;
  const int32_t *slot, *ranges;
  const float* weights;
  float* dweights;
  int tokens, k, d, n_rows, capacity, experts, lanes_log, parts_log;  // 2^lanes_log lanes take a row; of a combine, 2^parts_log wavefronts
  // A row's columns [0, vectors) go in vectors of 16 bytes, the last of which ends with them: where `vectors` is no multiple of a vector it has elements in common with the one
  // before, which come out the same.  The columns from `vectors` on go one by one: of rows shorter than a vector, and of sums formed in place, where nothing may be read twice.
  int vectors;
  int64_t token_groups;                                             // work-groups of tokens; those behind clear rows without a token
  Divisor by_k, by_capacity;
};

template <typename T>
__device__ __forceinline__ void clear_row(T* row, int lane, int lanes, const RowsArgs& a) {
  for (int c = lane * Row<T>::kVec; c < a.vectors; c += Row<T>::kVec * lanes) st_vec(row + min(c, a.vectors - Row<T>::kVec), typename Row<T>::vec{});
  for (int c = a.vectors + lane; c < a.d; c += lanes) row[c] = T(0);
}

// Where the counts before a chunk and the totals come from: WHOLE: every choice is counted here; SUMMED: counts of segments, added up here; SCANNED: by the scan.
enum Counts { WHOLE, SUMMED, SCANNED };

// The slots of a chunk of choices and, T being any type of the rows' size and not void, the rows that go there.
template <typename T, Counts COUNTS, int THREADS>
__global__ void __launch_bounds__(THREADS) expert_dispatch_kernel(const SortArgs s, const RowsArgs a) {
  touch(s);
  touch(a);
  extern __shared__ int32_t lds[];  // three of `experts` each
  __shared__ int32_t slots[kChunk], waves[THREADS / kWave];
  int32_t *before = lds, *total = lds + s.experts, *first = total + s.experts;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int begin = (int)min((int64_t)blockIdx.x * s.chunk, (int64_t)s.n), end = min(begin + s.chunk, s.n);  // (nothing behind the last chunk: only rows to clear)
  const int segment = begin / kSegment;
  for (int e = threadIdx.x; e < s.experts; e += THREADS) {
    before[e] = COUNTS == SCANNED ? s.hist[(int64_t)segment * s.experts + e] : 0;
    total[e] = COUNTS == SCANNED ? s.totals[e] : 0;
  }
  const int mine = begin + lane < end ? s.expert[begin + lane] : -1;  // (wavefront 0's to place)
  __syncthreads();
  if (COUNTS == WHOLE) {
    each_choice(s, 0, s.n, [&](int i, int e) { atomicAdd(i < begin ? &before[e] : &total[e], 1); });
  } else {
    if (COUNTS == SUMMED) {
      const int entries = s.segments * s.experts, mine_from = segment * s.experts;
      constexpr int AHEAD = 8;
      for (int i = threadIdx.x; i < entries; i += AHEAD * THREADS) {
        int32_t v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) v[u] = s.hist[min(i + u * THREADS, entries - 1)];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          const int at = i + u * THREADS;
          uint32_t e;
          div_mod((uint32_t)at, s.by_experts, e);
          if (at < entries && v[u]) atomicAdd(at < mine_from ? &before[e] : &total[e], v[u]);
        }
      }
    }
    __syncthreads();
    if (COUNTS == SUMMED)
      for (int e = threadIdx.x; e < s.experts; e += THREADS) total[e] += before[e];
    __syncthreads();
    each_choice(s, segment * kSegment, begin, [&](int, int e) { atomicAdd(&before[e], 1); });
  }
  __syncthreads();
  if (COUNTS == WHOLE) {
    for (int e = threadIdx.x; e < s.experts; e += THREADS) total[e] += before[e];
    __syncthreads();
  }
  // the experts' first rows
  if (s.capacity) {
    for (int e = threadIdx.x; e < s.experts; e += THREADS) first[e] = e * s.capacity;
  } else {
    int32_t carry = 0;
    for (int e0 = 0; e0 < s.experts; e0 += THREADS) {
      const int e = e0 + threadIdx.x;
      const int32_t own = e < s.experts ? total[e] : 0;
      int32_t sum = own;
#pragma unroll
      for (int step = 1; step < kWave; step *= 2) {
        const int32_t up = __shfl_up(sum, step);
        sum += lane >= step ? up : 0;
      }
      if (lane == kWave - 1) waves[wave] = sum;
      __syncthreads();
      int32_t all = 0;
#pragma unroll
      for (int w = 0; w < THREADS / kWave; ++w) {
        sum += w < wave ? waves[w] : 0;
        all += waves[w];
      }
      if (e < s.experts) first[e] = carry + sum - own;
      carry += all;
      __syncthreads();
    }
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int e = threadIdx.x; e < s.experts; e += THREADS) {
      s.ranges[2 * e] = first[e];
      s.ranges[2 * e + 1] = s.capacity ? min(total[e], s.capacity) : total[e];
    }
  if (wave == 0) {
    // the lanes before this one with the same expert
    const bool valid = (uint32_t)mine < (uint32_t)s.experts;
    uint64_t same = __ballot(valid);
    for (int b = 0; b < s.bits; ++b) {
      const uint64_t set = __ballot((mine >> b) & 1);
      same &= (mine >> b) & 1 ? set : ~set;
    }
    int32_t slot = -1;
    if (valid) {
      const int32_t rank = before[mine] + __popcll(same & ((1ull << lane) - 1));
      if (s.capacity == 0 || rank < s.capacity) slot = first[mine] + rank;
    }
    slots[lane] = slot;
    if (begin + lane < end) s.slot[begin + lane] = slot;
  }
  if constexpr (!std::is_same_v<T, void>) {
    __syncthreads();
    constexpr int N = Row<T>::kVec, AHEAD = 4;
    const T* x = static_cast<const T*>(a.x);
    T* rows = static_cast<T*>(a.out);
    const int part = threadIdx.x & ((1 << a.lanes_log) - 1), at_once = THREADS >> a.lanes_log;
    for (int i0 = threadIdx.x >> a.lanes_log; i0 < end - begin; i0 += AHEAD * at_once) {
      const T* from[AHEAD];
      T* to[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = i0 + u * at_once, slot = i < end - begin ? slots[i] : -1;
        uint32_t rest;
        from[u] = x + (int64_t)div_mod((uint32_t)(begin + min(i, end - begin - 1)), a.by_k, rest) * a.ld_x;
        to[u] = slot < 0 ? nullptr : rows + (int64_t)slot * a.ld_out;
      }
      for (int c0 = part * N; c0 < a.vectors; c0 += N << a.lanes_log) {
        const int c = min(c0, a.vectors - N);
        typename Row<T>::vec v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) v[u] = ld_vec(from[u] + c);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
          if (to[u]) st_vec(to[u] + c, v[u]);
      }
      for (int c = a.vectors + part; c < a.d; c += 1 << a.lanes_log)
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
          if (to[u]) to[u][c] = from[u][c];
    }
    // rows of fixed room that no token took
    const uint32_t room = (uint32_t)s.experts * (uint32_t)s.capacity;
    for (uint32_t r = blockIdx.x * (uint32_t)at_once + (threadIdx.x >> a.lanes_log); r < room; r += gridDim.x * (uint32_t)at_once) {
      uint32_t rank;
      const uint32_t e = div_mod(r, a.by_capacity, rank);
      if ((int)rank >= total[e]) clear_row(rows + (int64_t)r * a.ld_out, part, 1 << a.lanes_log, a);
    }
  }
}

// Work-groups in two dimensions: one has less than 2^32 threads.
__device__ __forceinline__ int64_t group_of() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// Rows of fixed room that no token took become zero.
template <typename T>
__device__ __forceinline__ void clear_rows(const RowsArgs& a, void* rows, int64_t ld, int64_t group) {
  const int per = kThreads >> a.lanes_log;
  const int64_t s = group * per + (threadIdx.x >> a.lanes_log);
  if (s >= (int64_t)a.experts * a.capacity) return;
  uint32_t rank;
  const uint32_t e = div_mod((uint32_t)s, a.by_capacity, rank);
  if ((int)rank < a.ranges[2 * e + 1]) return;
  clear_row(static_cast<T*>(rows) + s * ld, threadIdx.x & ((1 << a.lanes_log) - 1), 1 << a.lanes_log, a);
}

// rows[slot[t, j]] = x[t]; T is any type of the rows' size.
template <typename T, bool STREAM>
__global__ void __launch_bounds__(kThreads) expert_scatter_kernel(const RowsArgs a) {
  constexpr int N = Row<T>::kVec;
  touch(a);
  if (group_of() >= a.token_groups) {
    clear_rows<T>(a, a.out, a.ld_out, group_of() - a.token_groups);
    return;
  }
  const int64_t t = group_of() * (kThreads >> a.lanes_log) + (threadIdx.x >> a.lanes_log);
  if (t >= a.tokens) return;
  const T* x = static_cast<const T*>(a.x) + t * a.ld_x;
  T* rows = static_cast<T*>(a.out);
  const int lane = threadIdx.x & ((1 << a.lanes_log) - 1);
  for (int c0 = lane * N; c0 < a.vectors; c0 += N << a.lanes_log) {
    const int c = min(c0, a.vectors - N);
    const typename Row<T>::vec v = ld_vec(x + c);
    for (int j = 0; j < a.k; ++j) {
      const int32_t s = a.slot[t * a.k + j];
      if (s >= 0) st_vec<STREAM>(rows + (int64_t)s * a.ld_out + c, v);
    }
  }
  for (int c = a.vectors + lane; c < a.d; c += 1 << a.lanes_log) {
    const T v = x[c];
    for (int j = 0; j < a.k; ++j) {
      const int32_t s = a.slot[t * a.k + j];
      if (s >= 0) rows[(int64_t)s * a.ld_out + c] = v;
    }
  }
}

// The rows and weights of AHEAD choices of a token from the j0-th on, all asked for before the first is waited for.  A choice that is none takes row 0, if there is
// one, and `there` says so; nothing hangs on a branch.
template <int AHEAD>
struct Choices {
  int64_t row[AHEAD];
  float w[AHEAD];
  bool there[AHEAD];
  __device__ __forceinline__ void load(const RowsArgs& a, int64_t first, int j0) {  // first: the token's first choice
    const float* weights = a.weights ? a.weights : reinterpret_cast<const float*>(a.slot);  // (read in either case, and not used without weights)
    int32_t at[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      at[u] = a.slot[first + min(j0 + u, a.k - 1)];
      w[u] = weights[first + min(j0 + u, a.k - 1)];
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      there[u] = j0 + u < a.k && (uint32_t)at[u] < (uint32_t)a.n_rows;
      row[u] = there[u] ? at[u] : 0;
      w[u] = a.weights ? w[u] : 1.f;
    }
  }
};
// A single element, rounded as those of a vector are: to fp32 and then to T.  (One instruction would do both and round once, so that results in place, where rows end in
// single elements, would differ from others now and then.)
template <typename T>
__device__ __forceinline__ T rounded(float v) {
  asm volatile("" : "+v"(v));
  return (T)v;
}

// The token of LANES lanes; of a whole wavefront a number the scalar unit holds, and with it its slots and weights.
template <int LANES>
__device__ __forceinline__ int64_t token_of() {
  const uint32_t mine = threadIdx.x / LANES;
  return group_of() * (kThreads / LANES) + (LANES >= 64 ? __builtin_amdgcn_readfirstlane(mine) : mine);
}

// out[t] = add[t] + sum over j of weights[t, j] rows[slot[t, j]], in the order of j.  LANES lanes per token; AHEAD rows, two vectors a lane of each, are asked for together.
template <typename T, int LANES, int AHEAD, bool STREAM>
__global__ void __launch_bounds__(kThreads) expert_combine_kernel(const RowsArgs a) {
  constexpr int N = Row<T>::kVec, VECS = LANES == 64 ? 2 : 1;
  touch(a);
  const int lane = threadIdx.x % LANES;
  const int64_t mine = token_of<LANES>(), t = LANES == 64 ? mine >> a.parts_log : mine;
  const int part = LANES == 64 ? (int)mine & ((1 << a.parts_log) - 1) : 0;
  const int step = (VECS * N * LANES) << (LANES == 64 ? a.parts_log : 0);
  if (t >= a.tokens) return;
  const T* add = static_cast<const T*>(a.add) + t * a.ld_add;
  const T* rows = static_cast<const T*>(a.rows);
  T* out = static_cast<T*>(a.out) + t * a.ld_out;
  Choices<AHEAD> at;
  at.load(a, t * a.k, 0);
  for (int c = (part * VECS * LANES + lane) * N; c < a.vectors; c += step) {
    const int col[2] = {min(c, a.vectors - N), min(c + N * LANES, a.vectors - N)};  // (the last vector twice where there is no second)
    float s[VECS][N];
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      typename Row<T>::vec v = {};
      if (a.add) v = ld_vec(add + col[i]);
#pragma unroll
      for (int e = 0; e < N; ++e) s[i][e] = (float)v[e];
    }
    for (int j0 = 0; j0 < a.k && a.n_rows > 0; j0 += AHEAD) {
      if (a.k > AHEAD) at.load(a, t * a.k, j0);
      typename Row<T>::vec v[AHEAD][VECS];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int i = 0; i < VECS; ++i) v[u][i] = ld_vec<STREAM>(rows + at.row[u] * a.ld_rows + col[i]);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int i = 0; i < VECS; ++i)
#pragma unroll
          for (int e = 0; e < N; ++e) s[i][e] = at.there[u] ? s[i][e] + at.w[u] * (float)v[u][i][e] : s[i][e];
    }
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      typename Row<T>::vec o;
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] = (T)s[i][e];
      st_vec<STREAM>(out + col[i], o);
    }
  }
  if (const int c = a.vectors + lane; c < a.d && part == 0) {
    float s = a.add ? (float)add[c] : 0.f;
    for (int j0 = 0; j0 < a.k && a.n_rows > 0; j0 += AHEAD) {
      if (a.k > AHEAD) at.load(a, t * a.k, j0);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const float v = (float)rows[at.row[u] * a.ld_rows + c];
        s = at.there[u] ? s + at.w[u] * v : s;
      }
    }
    out[c] = rounded<T>(s);
  }
}

// out[slot[t, j]] = weights[t, j] x[t] and dweights[t, j] = <x[t], rows[slot[t, j]]>; LANES lanes per token, AHEAD rows asked for together.
template <typename T, int LANES, int AHEAD, bool STREAM>
__global__ void __launch_bounds__(kThreads) expert_combine_bwd_kernel(const RowsArgs a) {
  constexpr int N = Row<T>::kVec;
  __shared__ float part[LANES / kWave + 1][AHEAD];
  touch(a);
  if (group_of() >= a.token_groups) {
    clear_rows<T>(a, a.out, a.ld_out, group_of() - a.token_groups);
    return;
  }
  const int lane = threadIdx.x % LANES;
  const int64_t t = token_of<LANES>();
  if (t >= a.tokens) return;
  const T* x = static_cast<const T*>(a.x) + t * a.ld_x;
  const T* rows = static_cast<const T*>(a.rows);
  T* out = static_cast<T*>(a.out);
  const bool read = a.dweights && a.n_rows > 0;
  for (int j0 = 0; j0 < a.k; j0 += AHEAD) {
    Choices<AHEAD> at;
    at.load(a, t * a.k, j0);
    float dot[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) dot[u] = 0.f;
    for (int c0 = lane * N; c0 < a.vectors; c0 += N * LANES) {
      const int c = min(c0, a.vectors - N);
      const typename Row<T>::vec g = ld_vec(x + c);
      typename Row<T>::vec v[AHEAD] = {};
      if (read) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) v[u] = ld_vec<STREAM>(rows + at.row[u] * a.ld_rows + c);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        typename Row<T>::vec o;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          dot[u] += e >= c0 - c ? (float)g[e] * (float)v[u][e] : 0.f;
          o[e] = (T)((float)g[e] * at.w[u]);
        }
        if (at.there[u]) st_vec<STREAM>(out + at.row[u] * a.ld_out + c, o);
      }
    }
    if (const int c = a.vectors + lane; c < a.d) {
      const float g = (float)x[c];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (!at.there[u]) continue;
        if (read) dot[u] += g * (float)rows[at.row[u] * a.ld_rows + c];
        out[at.row[u] * a.ld_out + c] = rounded<T>(g * at.w[u]);
      }
    }
    if (a.dweights) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        dot[u] = lanes_sum<LANES < kWave ? LANES : kWave>(dot[u]);
        if (LANES > kWave && lane % kWave == 0) part[lane / kWave][u] = dot[u];
      }
      if (LANES > kWave) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          dot[u] = 0.f;
#pragma unroll
          for (int w = 0; w < LANES / kWave; ++w) dot[u] += part[w][u];
        }
        __syncthreads();
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (lane == 0 && j0 + u < a.k) a.dweights[t * a.k + j0 + u] = at.there[u] ? dot[u] : 0.f;
    }
  }
}

int lanes_log_of(int d, int type) {
  const int vecs = ceil_div(d, 16 / row_type_bytes(type));
  int l = 0;
  while ((1 << l) < vecs && l < 8) ++l;
  return l;
}

int vector_columns(int d, int type) { return d >= 16 / row_type_bytes(type) ? d : 0; }

// Rows that the last-level cache would not hold until they are read again go past it: 105402 x 1024 bf16 (216 MB) to the experts and back 142 -> 123 us, the gradients of
// 52012 x 1024 fp16 (107 MB) 80 -> 68.  With two products each way in between there is nothing in it (216 MB: 1105 and 1107 us, 131 MB: 661 and 669), and smaller rows lose
// (41 MB: 255 -> 262 us, 7 MB: 58 -> 60).
bool large_rows(int64_t rows, int d, size_t size) { return rows * d * (int64_t)size >= kStreamFrom; }

int segments_of(int64_t n) { return (int)((n + kSegment - 1) / kSegment); }

dim3 grid_of(int64_t groups) {
  const int64_t x = std::min<int64_t>(groups, 1 << 20);
  return dim3((uint32_t)x, x ? (uint32_t)((groups + x - 1) / x) : 1);
}

// A dispatch of one launch: chunks of fewer choices where these work-groups are few and have much to copy each (16 tokens of 8 x 8192 bf16 and back 37.8 -> 21.9 us), and
// work-groups beyond the chunks' to clear rows (64 experts' 512 rows of 512 fp16 for 128 choices 213 -> 12 us).
void spread(int64_t n, int64_t row_bytes, int64_t room, int* chunk, int* groups) {
  while (*chunk > 1 && *groups < kGroups && *chunk * row_bytes > kCopied) *chunk /= 2, *groups = ceil_div(n, *chunk);
  *groups = std::max<int64_t>(*groups, std::min<int64_t>(kGroups, room * row_bytes / kCopied));
}

int64_t scratch_of(int tokens, int k, int experts) { return tokens ? (int64_t)(segments_of((int64_t)tokens * k) + 1) * experts : 0; }

int check_lists(const char* who, int tokens, int k, int experts, int capacity) {
  NMT_REQUIRE(tokens >= 0 && k >= 1 && k <= kMaxChoices && (int64_t)tokens * k <= kMaxItems, "%s: %d tokens of %d choices", who, tokens, k);
  NMT_REQUIRE(experts >= 1 && experts <= kMaxExperts, "%s: %d experts outside [1, %d]", who, experts, kMaxExperts);
  NMT_REQUIRE(capacity >= 0 && (int64_t)experts * capacity <= kMaxItems, "%s: a capacity of %d rows", who, capacity);
  return NMT_OK;
}
int check_rows(const char* who, int d, int type) {
  NMT_REQUIRE(d >= 1 && d <= (1 << 20), "%s: d = %d", who, d);
  NMT_REQUIRE(row_type_ok(type), "%s: unknown type %d", who, type);
  return NMT_OK;
}
#define EXPERT_ROWS(ptr, n, ld, what) NMT_REQUIRE(!(ptr) || (n) <= 1 || (ld) >= d, "%s: rows of " what " overlap", who)

}  // namespace

extern "C" int64_t nmt_op_expert_dispatch_scratch(int32_t tokens, int32_t k, int32_t experts) {
  if (check_lists("nmt_op_expert_dispatch_scratch", tokens, k, experts, 0) != NMT_OK) return NMT_EINVAL;
  return scratch_of(tokens, k, experts);
}

extern "C" int nmt_op_expert_dispatch(const int32_t* d_expert, int32_t tokens, int32_t k, int32_t experts, int32_t capacity, const void* d_x,
                                      int64_t ld_x, int32_t d, int32_t type, void* d_rows, int64_t ld_rows, int32_t* d_slot,
                                      int32_t* d_ranges, int32_t* d_scratch, int64_t scratch_ints, void* stream_) {
  const char* who = "nmt_op_expert_dispatch";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (const int rc = check_lists(who, tokens, k, experts, capacity); rc != NMT_OK) return rc;
  NMT_REQUIRE(!d_x == !d_rows || tokens == 0, "%s: tokens and the experts' rows belong together", who);
  const int64_t n = (int64_t)tokens * k;
  if (d_rows) {
    if (const int rc = check_rows(who, d, type); rc != NMT_OK) return rc;
    EXPERT_ROWS(d_x, tokens, ld_x, "x");
    EXPERT_ROWS(d_rows, capacity ? (int64_t)experts * capacity : n, ld_rows, "the experts");
  }
  NMT_REQUIRE(d_ranges && (tokens == 0 || (d_expert && d_slot)), "%s: null pointer", who);
  if (const int64_t need = scratch_of(tokens, k, experts); need > (d_scratch ? scratch_ints : 0)) {
    nmt_set_error("%s: scratch of %lld elements, %lld needed", who, (long long)(d_scratch ? scratch_ints : 0), (long long)need);
    return NMT_ENOMEM;
  }
  NMT_REQUIRE(tokens == 0 || d_expert != d_slot, "%s: slots in place of the choices, which every work-group reads", who);
  SortArgs s = {};
  s.expert = d_expert, s.n = (int)n, s.experts = experts, s.capacity = capacity, s.segments = segments_of(n);
  s.hist = d_scratch, s.totals = d_scratch + (int64_t)s.segments * experts, s.slot = d_slot, s.ranges = d_ranges;
  while ((1 << s.bits) < experts) ++s.bits;
  RowsArgs a = {};
  a.slot = d_slot, a.ranges = d_ranges;
  a.tokens = tokens, a.k = k, a.capacity = capacity, a.experts = experts, a.by_k = divisor(k), a.by_capacity = divisor(std::max(capacity, 1));
  if (d_rows) {
    a.x = d_x, a.ld_x = ld_x, a.out = d_rows, a.ld_out = ld_rows;
    a.d = d, a.vectors = vector_columns(d, type), a.lanes_log = lanes_log_of(d, type);
  }
  s.by_experts = divisor(experts);
  const bool whole = n <= kWhole, scan = (int64_t)s.segments * experts > kSummed;
  if (!whole) {
    hipLaunchKernelGGL(expert_count_kernel, dim3(s.segments), dim3(kThreads), sizeof(int32_t) * experts, stream, s);
    NMT_LAUNCH_CHECK();
    if (scan) hipLaunchKernelGGL(expert_scan_kernel, dim3(ceil_div(experts, kWave)), dim3(kScanWaves * kWave), 0, stream, s);
    NMT_LAUNCH_CHECK();
  }
  s.chunk = kChunk;
  int groups = ceil_div(n, kChunk);
  if (whole && d_rows) spread(n, (int64_t)d * row_type_bytes(type), (int64_t)experts * capacity, &s.chunk, &groups);
  const dim3 grid(std::max(1, groups));
  const size_t lds = sizeof(int32_t) * experts * 3;
  if (whole) {
    if (!d_rows) hipLaunchKernelGGL((expert_dispatch_kernel<void, WHOLE, kWholeThreads>), grid, dim3(kWholeThreads), lds, stream, s, a);
    else if (type == NMT_F32) hipLaunchKernelGGL((expert_dispatch_kernel<uint32_t, WHOLE, kWholeThreads>), grid, dim3(kWholeThreads), lds, stream, s, a);
    else hipLaunchKernelGGL((expert_dispatch_kernel<uint16_t, WHOLE, kWholeThreads>), grid, dim3(kWholeThreads), lds, stream, s, a);
    NMT_LAUNCH_CHECK();
    return NMT_OK;
  }
  if (scan) hipLaunchKernelGGL((expert_dispatch_kernel<void, SCANNED, kThreads>), grid, dim3(kThreads), lds, stream, s, a);
  else hipLaunchKernelGGL((expert_dispatch_kernel<void, SUMMED, kThreads>), grid, dim3(kThreads), lds, stream, s, a);
  NMT_LAUNCH_CHECK();
  if (!d_rows) return NMT_OK;
  const int per = kThreads >> a.lanes_log;
  a.token_groups = ceil_div(tokens, per);
  const dim3 rows_grid = grid_of(a.token_groups + ceil_div((int64_t)experts * capacity, per));
  const bool large = large_rows(n, d, row_type_bytes(type));
  if (type == NMT_F32) hipLaunchKernelGGL((large ? expert_scatter_kernel<uint32_t, true> : expert_scatter_kernel<uint32_t, false>), rows_grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((large ? expert_scatter_kernel<uint16_t, true> : expert_scatter_kernel<uint16_t, false>), rows_grid, dim3(kThreads), 0, stream, a);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}

template <typename T, int LANES, bool STREAM>
static void launch_combine(const RowsArgs& a, hipStream_t stream) {
  const dim3 grid = grid_of(ceil_div((int64_t)a.tokens << a.parts_log, kThreads / LANES));
  if (a.k == 1) hipLaunchKernelGGL((expert_combine_kernel<T, LANES, 1, STREAM>), grid, dim3(kThreads), 0, stream, a);
  else if (a.k == 2) hipLaunchKernelGGL((expert_combine_kernel<T, LANES, 2, STREAM>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((expert_combine_kernel<T, LANES, 4, STREAM>), grid, dim3(kThreads), 0, stream, a);
}
template <typename T>
static void launch_combine(RowsArgs a, hipStream_t stream) {
  if (a.lanes_log > 5)
    while (((int64_t)a.tokens << a.parts_log) < kFewWaves && (2 * 64 * Row<T>::kVec) << a.parts_log < a.d) ++a.parts_log;
  if (a.lanes_log <= 4) launch_combine<T, 16, false>(a, stream);
  else if (a.lanes_log == 5) launch_combine<T, 32, false>(a, stream);
  else if (large_rows((int64_t)a.tokens * a.k, a.d, sizeof(T))) launch_combine<T, 64, true>(a, stream);
  else launch_combine<T, 64, false>(a, stream);
}
template <typename T, int LANES, bool STREAM>
static void launch_combine_bwd(RowsArgs a, hipStream_t stream) {
  a.token_groups = ceil_div(a.tokens, kThreads / LANES);
  const dim3 grid = grid_of(a.token_groups + ceil_div((int64_t)a.experts * a.capacity, kThreads >> a.lanes_log));
  if (grid.x == 0) return;
  if (a.k == 1) hipLaunchKernelGGL((expert_combine_bwd_kernel<T, LANES, 1, STREAM>), grid, dim3(kThreads), 0, stream, a);
  else if (a.k == 2) hipLaunchKernelGGL((expert_combine_bwd_kernel<T, LANES, 2, STREAM>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((expert_combine_bwd_kernel<T, LANES, 4, STREAM>), grid, dim3(kThreads), 0, stream, a);
}
template <typename T>
static void launch_combine_bwd(RowsArgs a, hipStream_t stream) {
  const bool large = large_rows((int64_t)a.tokens * a.k, a.d, sizeof(T));
  if (a.lanes_log > 7 && a.tokens < kFewWaves) {
    if (a.rows == a.out) a.vectors = a.d / Row<T>::kVec * Row<T>::kVec;  // (no wavefront reads what another has written)
    return large ? launch_combine_bwd<T, 256, true>(a, stream) : launch_combine_bwd<T, 256, false>(a, stream);
  }
  if (a.lanes_log <= 4) launch_combine_bwd<T, 16, false>(a, stream);
  else if (a.lanes_log == 5) launch_combine_bwd<T, 32, false>(a, stream);
  else if (large) launch_combine_bwd<T, 64, true>(a, stream);
  else launch_combine_bwd<T, 64, false>(a, stream);
}

extern "C" int nmt_op_expert_combine(const void* d_rows, int64_t ld_rows, int32_t n_rows, const int32_t* d_slot, const float* d_weights,
                                     const void* d_add, int64_t ld_add, void* d_out, int64_t ld_out, int32_t tokens, int32_t k, int32_t d,
                                     int32_t type, void* stream_) {
  const char* who = "nmt_op_expert_combine";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (const int rc = check_lists(who, tokens, k, 1, 0); rc != NMT_OK) return rc;
  if (const int rc = check_rows(who, d, type); rc != NMT_OK) return rc;
  NMT_REQUIRE(n_rows >= 0, "%s: %d rows", who, n_rows);
  if (tokens == 0) return NMT_OK;
  NMT_REQUIRE((d_rows || n_rows == 0) && d_slot && d_out, "%s: null pointer", who);
  EXPERT_ROWS(d_rows, n_rows, ld_rows, "the experts");
  EXPERT_ROWS(d_add, tokens, ld_add, "add");
  EXPERT_ROWS(d_out, tokens, ld_out, "out");
  RowsArgs a = {};
  a.rows = d_rows, a.ld_rows = ld_rows, a.n_rows = n_rows, a.slot = d_slot, a.weights = d_weights, a.add = d_add, a.ld_add = ld_add;
  a.out = d_out, a.ld_out = ld_out, a.tokens = tokens, a.k = k, a.d = d, a.lanes_log = lanes_log_of(d, type);
  const int vec = 16 / row_type_bytes(type);
  a.vectors = d_add && d_add == d_out ? d / vec * vec : vector_columns(d, type);
  if (type == NMT_F16) launch_combine<half_t>(a, stream);
  else if (type == NMT_BF16) launch_combine<bf16_t>(a, stream);
  else launch_combine<float>(a, stream);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}

extern "C" int nmt_op_expert_combine_bwd(const void* d_dout, int64_t ld_dout, const void* d_rows, int64_t ld_rows, int32_t n_rows,
                                         const int32_t* d_slot, const float* d_weights, void* d_drows, int64_t ld_drows, float* d_dweights,
                                         const int32_t* d_ranges, int32_t experts, int32_t capacity, int32_t tokens, int32_t k, int32_t d,
                                         int32_t type, void* stream_) {
  const char* who = "nmt_op_expert_combine_bwd";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (const int rc = check_lists(who, tokens, k, experts, capacity); rc != NMT_OK) return rc;
  if (const int rc = check_rows(who, d, type); rc != NMT_OK) return rc;
  NMT_REQUIRE(n_rows >= 0, "%s: %d rows", who, n_rows);
  NMT_REQUIRE(capacity == 0 || (int64_t)experts * capacity == n_rows, "%s: %d experts of %d rows are not the %d rows there are", who, experts, capacity, n_rows);
  NMT_REQUIRE(!d_rows == !d_dweights || n_rows == 0 || tokens == 0, "%s: the experts' rows are read for the weights' gradient and for nothing else", who);
  if (tokens == 0 && capacity == 0) return NMT_OK;
  NMT_REQUIRE((tokens == 0 || (d_dout && d_slot)) && (d_drows || n_rows == 0) && (d_ranges || capacity == 0), "%s: null pointer", who);
  EXPERT_ROWS(d_dout, tokens, ld_dout, "dout");
  EXPERT_ROWS(d_rows, n_rows, ld_rows, "the experts");
  EXPERT_ROWS(d_drows, n_rows, ld_drows, "the experts' gradient");
  RowsArgs a = {};
  a.x = d_dout, a.ld_x = ld_dout, a.rows = d_rows, a.ld_rows = ld_rows, a.n_rows = n_rows, a.slot = d_slot, a.ranges = d_ranges;
  a.weights = d_weights, a.dweights = d_dweights, a.out = d_drows, a.ld_out = ld_drows;
  a.tokens = tokens, a.k = k, a.d = d, a.vectors = vector_columns(d, type), a.capacity = capacity, a.experts = experts, a.lanes_log = lanes_log_of(d, type);
  a.by_capacity = divisor(std::max(capacity, 1));
  if (type == NMT_F16) launch_combine_bwd<half_t>(a, stream);
  else if (type == NMT_BF16) launch_combine_bwd<bf16_t>(a, stream);
  else launch_combine_bwd<float>(a, stream);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}
