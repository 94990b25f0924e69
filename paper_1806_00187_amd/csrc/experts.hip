// Tokens sorted by expert and back.  A counting sort of the choices (stable, no atomics), rows copied to their expert's, the weighted
// sum of a token's rows on the way back, and the gradients.  Bound by memory: the rows that are read and written once.
#include "rowtypes.h"

#include <algorithm>

namespace {

constexpr int kThreads = 256;
constexpr int kSegment = 1024;      // choices of a work-group of the sort
constexpr int kMaxExperts = 1024, kMaxChoices = 64;
constexpr int64_t kMaxItems = 1 << 30;
constexpr int kWaves = kThreads / kWave, kPerWave = kSegment / kWaves;

// The lanes whose key equals this lane's, among those with a valid one (0 for the others).
__device__ __forceinline__ uint64_t same_key(uint32_t key, bool valid, int bits) {
  uint64_t m = __ballot(valid);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((key >> b) & 1);
    m &= (key >> b) & 1 ? set : ~set;
  }
  return valid ? m : 0;
}

struct SortArgs {
  const int32_t* expert;
  int n, experts, capacity, segments, bits;
  int32_t *hist, *slot, *ranges;
};

// Counts of the experts among a wavefront's choices, in LDS: one lane of those with the same expert adds for all of them.
__device__ __forceinline__ void count_wave(const SortArgs& a, int64_t first, int32_t* counts) {
  const int lane = threadIdx.x & 63;
  for (int r = 0; r < kPerWave; r += kWave) {
    const int64_t i = first + r + lane;
    const uint32_t key = i < a.n ? (uint32_t)a.expert[i] : 0xFFFFFFFFu;
    const uint64_t same = same_key(key, key < (uint32_t)a.experts, a.bits);
    if (same && (same & ((1ull << lane) - 1)) == 0) counts[key] += __popcll(same);
    wave_sync();
  }
}

__global__ void __launch_bounds__(kThreads) expert_count_kernel(const SortArgs a) {
  extern __shared__ int32_t lds[];  // kWaves * experts
  for (int e = threadIdx.x; e < kWaves * a.experts; e += kThreads) lds[e] = 0;
  __syncthreads();
  const int wave = threadIdx.x >> 6;
  count_wave(a, (int64_t)blockIdx.x * kSegment + wave * kPerWave, lds + wave * a.experts);
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    int32_t s = 0;
    for (int w = 0; w < kWaves; ++w) s += lds[w * a.experts + e];
    a.hist[(int64_t)blockIdx.x * a.experts + e] = s;
  }
}

__global__ void __launch_bounds__(kThreads) expert_rank_kernel(const SortArgs a) {
  extern __shared__ int32_t lds[];  // kWaves * experts counts, then experts first rows and experts counts of earlier segments
  int32_t* first = lds + kWaves * a.experts;
  int32_t* earlier = first + a.experts;
  for (int e = threadIdx.x; e < kWaves * a.experts; e += kThreads) lds[e] = 0;
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    int32_t before = 0, all = 0;
    for (int s = 0; s < a.segments; ++s) {
      const int32_t h = a.hist[(int64_t)s * a.experts + e];
      before += s < (int)blockIdx.x ? h : 0;
      all += h;
    }
    first[e] = all;
    earlier[e] = before;
  }
  __syncthreads();
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t begin = (int64_t)blockIdx.x * kSegment + wave * kPerWave;
  count_wave(a, begin, lds + wave * a.experts);
  if (threadIdx.x == 0) {  // the experts' first rows
    int32_t s = 0;
    for (int e = 0; e < a.experts; ++e) {
      const int32_t all = first[e];
      first[e] = a.capacity ? e * a.capacity : s;
      if (blockIdx.x == 0) {
        a.ranges[2 * e] = first[e];
        a.ranges[2 * e + 1] = a.capacity ? min(all, a.capacity) : all;
      }
      s += all;
    }
  }
  __syncthreads();
  // a wavefront's rank among the choices of an expert: those of earlier segments and of earlier wavefronts
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    int32_t s = earlier[e];
    for (int w = 0; w < kWaves; ++w) {
      const int32_t c = lds[w * a.experts + e];
      lds[w * a.experts + e] = s;
      s += c;
    }
  }
  __syncthreads();
  for (int r = 0; r < kPerWave; r += kWave) {
    const int64_t i = begin + r + lane;
    const uint32_t key = i < a.n ? (uint32_t)a.expert[i] : 0xFFFFFFFFu;
    const bool valid = key < (uint32_t)a.experts;
    const uint64_t same = same_key(key, valid, a.bits);
    const uint64_t before = same & ((1ull << lane) - 1);
    int32_t* next = lds + wave * a.experts;
    const int32_t rank = valid ? next[key] + __popcll(before) : 0;
    wave_sync();
    if (valid && before == 0) next[key] += __popcll(same);
    wave_sync();
    if (i < a.n) a.slot[i] = valid && (a.capacity == 0 || rank < a.capacity) ? first[key] + rank : -1;
  }
}

// The rows of a work-group's tokens: 2^lanes_log lanes for a row, 16 bytes each.
struct RowsArgs {
  const void *x, *rows, *add;
  void* out;
  int64_t ld_x, ld_rows, ld_add, ld_out;
  const int32_t *slot, *ranges;
  const float* weights;
  float* dweights;
  int tokens, k, d, vectors, n_rows, capacity, experts, lanes_log;  // vectors: columns in whole vectors of 16 bytes
  int64_t token_groups;  // work-groups of tokens; those behind clear rows without a token
};

// Rows of fixed room that no token took become zero.
template <typename T>
__device__ __forceinline__ void clear_rows(const RowsArgs& a, void* rows, int64_t ld, int64_t group) {
  constexpr int N = Row<T>::kVec;
  const int per = kThreads >> a.lanes_log;
  const int64_t s = group * per + (threadIdx.x >> a.lanes_log);
  if (s >= (int64_t)a.experts * a.capacity) return;
  const int e = (int)(s / a.capacity);
  if ((int)(s - (int64_t)e * a.capacity) < a.ranges[2 * e + 1]) return;
  T* row = static_cast<T*>(rows) + s * ld;
  const int lane = threadIdx.x & ((1 << a.lanes_log) - 1);
  for (int c = lane * N; c < a.vectors; c += N << a.lanes_log) st_vec(row + c, typename Row<T>::vec{});
  for (int c = a.vectors + lane; c < a.d; c += 1 << a.lanes_log) row[c] = T(0);
}

// rows[slot[t, j]] = x[t]; T is any type of the rows' size.
template <typename T>
__global__ void __launch_bounds__(kThreads) expert_scatter_kernel(const RowsArgs a) {
  constexpr int N = Row<T>::kVec;
  if (blockIdx.x >= a.token_groups) {
    clear_rows<T>(a, a.out, a.ld_out, blockIdx.x - a.token_groups);
    return;
  }
  const int64_t t = (int64_t)blockIdx.x * (kThreads >> a.lanes_log) + (threadIdx.x >> a.lanes_log);
  if (t >= a.tokens) return;
  const T* x = static_cast<const T*>(a.x) + t * a.ld_x;
  T* rows = static_cast<T*>(a.out);
  const int lane = threadIdx.x & ((1 << a.lanes_log) - 1);
  for (int c = lane * N; c < a.vectors; c += N << a.lanes_log) {
    const typename Row<T>::vec v = ld_vec(x + c);
    for (int j = 0; j < a.k; ++j) {
      const int32_t s = a.slot[t * a.k + j];
      if (s >= 0) st_vec(rows + (int64_t)s * a.ld_out + c, v);
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

// out[t] = add[t] + sum over j of weights[t, j] rows[slot[t, j]]
template <typename T>
__global__ void __launch_bounds__(kThreads) expert_combine_kernel(const RowsArgs a) {
  constexpr int N = Row<T>::kVec;
  const int64_t t = (int64_t)blockIdx.x * (kThreads >> a.lanes_log) + (threadIdx.x >> a.lanes_log);
  if (t >= a.tokens) return;
  const T* add = static_cast<const T*>(a.add) + t * a.ld_add;
  T* out = static_cast<T*>(a.out) + t * a.ld_out;
  const int lane = threadIdx.x & ((1 << a.lanes_log) - 1);
  for (int c = lane * N; c < a.vectors; c += N << a.lanes_log) {
    float s[N];
    typename Row<T>::vec v = {};
    if (a.add) v = ld_vec(add + c);
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] = (float)v[e];
    for (int j = 0; j < a.k; ++j) {
      const int32_t at = a.slot[t * a.k + j];
      if ((uint32_t)at >= (uint32_t)a.n_rows) continue;
      const float w = a.weights ? a.weights[t * a.k + j] : 1.f;
      v = ld_vec(static_cast<const T*>(a.rows) + (int64_t)at * a.ld_rows + c);
#pragma unroll
      for (int e = 0; e < N; ++e) s[e] += w * (float)v[e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (T)s[e];
    st_vec(out + c, v);
  }
  for (int c = a.vectors + lane; c < a.d; c += 1 << a.lanes_log) {
    float s = a.add ? (float)add[c] : 0.f;
    for (int j = 0; j < a.k; ++j) {
      const int32_t at = a.slot[t * a.k + j];
      if ((uint32_t)at >= (uint32_t)a.n_rows) continue;
      s += (a.weights ? a.weights[t * a.k + j] : 1.f) * (float)static_cast<const T*>(a.rows)[(int64_t)at * a.ld_rows + c];
    }
    out[c] = (T)s;
  }
}

// out[slot[t, j]] = weights[t, j] x[t] and dweights[t, j] = <x[t], rows[slot[t, j]]>; a wavefront per token.
template <typename T>
__global__ void __launch_bounds__(kThreads) expert_combine_bwd_kernel(const RowsArgs a) {
  constexpr int N = Row<T>::kVec;
  if (blockIdx.x >= a.token_groups) {
    clear_rows<T>(a, a.out, a.ld_out, blockIdx.x - a.token_groups);
    return;
  }
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (t >= a.tokens) return;
  const T* x = static_cast<const T*>(a.x) + t * a.ld_x;
  for (int j = 0; j < a.k; ++j) {
    const int32_t at = a.slot[t * a.k + j];
    float dot = 0.f;
    if ((uint32_t)at < (uint32_t)a.n_rows) {
      const float w = a.weights ? a.weights[t * a.k + j] : 1.f;
      const T* row = static_cast<const T*>(a.rows) + (int64_t)at * a.ld_rows;
      T* out = static_cast<T*>(a.out) + (int64_t)at * a.ld_out;
      for (int c = lane * N; c < a.vectors; c += N * kWave) {
        typename Row<T>::vec g = ld_vec(x + c);
        if (a.dweights) {
          const typename Row<T>::vec v = ld_vec(row + c);
#pragma unroll
          for (int e = 0; e < N; ++e) dot += (float)g[e] * (float)v[e];
        }
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = (T)((float)g[e] * w);
        st_vec(out + c, g);
      }
      if (const int c = a.vectors + lane; c < a.d) {
        const float g = (float)x[c];
        if (a.dweights) dot += g * (float)row[c];
        out[c] = (T)(g * w);
      }
    }
    if (a.dweights) {
      dot = wave_sum(dot);
      if (lane == 0) a.dweights[t * a.k + j] = dot;
    }
  }
}

int lanes_log_of(int d, int type) {
  const int vecs = ceil_div(d, 16 / row_type_bytes(type));
  int l = 0;
  while ((1 << l) < vecs && l < 8) ++l;
  return l;
}

int whole_vectors(int d, int type) { return d / (16 / row_type_bytes(type)) * (16 / row_type_bytes(type)); }

int segments_of(int64_t n) { return (int)((n + kSegment - 1) / kSegment); }

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
  return (int64_t)segments_of((int64_t)tokens * k) * experts;
}

extern "C" int nmt_op_expert_dispatch(const int32_t* d_expert, int32_t tokens, int32_t k, int32_t experts, int32_t capacity, const void* d_x,
                                      int64_t ld_x, int32_t d, int32_t type, void* d_rows, int64_t ld_rows, int32_t* d_slot,
                                      int32_t* d_ranges, int32_t* d_scratch, void* stream_) {
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
  NMT_REQUIRE(d_ranges && (tokens == 0 || (d_expert && d_slot && d_scratch)), "%s: null pointer", who);
  SortArgs s = {d_expert, (int)n, experts, capacity, segments_of(n), 0, d_scratch, d_slot, d_ranges};
  while ((1 << s.bits) < experts) ++s.bits;
  if (tokens) {
    hipLaunchKernelGGL(expert_count_kernel, dim3(s.segments), dim3(kThreads), sizeof(int32_t) * kWaves * experts, stream, s);
    NMT_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL(expert_rank_kernel, dim3(std::max(s.segments, 1)), dim3(kThreads), sizeof(int32_t) * (kWaves + 2) * experts, stream, s);
  NMT_LAUNCH_CHECK();
  if (!d_rows) return NMT_OK;
  RowsArgs a = {};
  a.x = d_x, a.ld_x = ld_x, a.out = d_rows, a.ld_out = ld_rows, a.slot = d_slot, a.ranges = d_ranges;
  a.tokens = tokens, a.k = k, a.d = d, a.vectors = whole_vectors(d, type), a.capacity = capacity, a.experts = experts, a.lanes_log = lanes_log_of(d, type);
  const int per = kThreads >> a.lanes_log;
  a.token_groups = ceil_div(tokens, per);
  const dim3 grid((uint32_t)(a.token_groups + ceil_div((int64_t)experts * capacity, per)));
  if (grid.x == 0) return NMT_OK;
  if (type == NMT_F32) hipLaunchKernelGGL(expert_scatter_kernel<uint32_t>, grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(expert_scatter_kernel<uint16_t>, grid, dim3(kThreads), 0, stream, a);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
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
  a.out = d_out, a.ld_out = ld_out, a.tokens = tokens, a.k = k, a.d = d, a.vectors = whole_vectors(d, type), a.lanes_log = lanes_log_of(d, type);
  const dim3 grid(ceil_div(tokens, kThreads >> a.lanes_log));
  if (type == NMT_F16) hipLaunchKernelGGL(expert_combine_kernel<half_t>, grid, dim3(kThreads), 0, stream, a);
  else if (type == NMT_BF16) hipLaunchKernelGGL(expert_combine_kernel<bf16_t>, grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(expert_combine_kernel<float>, grid, dim3(kThreads), 0, stream, a);
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
  a.tokens = tokens, a.k = k, a.d = d, a.vectors = whole_vectors(d, type), a.capacity = capacity, a.experts = experts, a.lanes_log = lanes_log_of(d, type);
  a.token_groups = ceil_div(tokens, kWaves);
  const dim3 grid((uint32_t)(a.token_groups + ceil_div((int64_t)experts * capacity, kThreads >> a.lanes_log)));
  if (grid.x == 0) return NMT_OK;
  if (type == NMT_F16) hipLaunchKernelGGL(expert_combine_bwd_kernel<half_t>, grid, dim3(kThreads), 0, stream, a);
  else if (type == NMT_BF16) hipLaunchKernelGGL(expert_combine_bwd_kernel<bf16_t>, grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(expert_combine_bwd_kernel<float>, grid, dim3(kThreads), 0, stream, a);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}
