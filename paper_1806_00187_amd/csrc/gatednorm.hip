// The norms around a gated residual block, one pass over the rows each way:
//   h = a x + gate post(y), n = pre(h);  post, pre: LayerNorm or RMS norm with gain and shift.
// Bound by memory: forward reads x, y and writes h, n (n needs h's statistics, which are there while h is still in registers), backward
// reads y, h and the gradients at h and n and writes those at x and y.  A row is held in registers by 8 to 64 lanes (up to 64, 128, 256, 512 columns) or by
// several wavefronts, each lane's share of it 16 bytes at a time; the next row is in flight while one is worked on.
// Forward 52701 x 1024 bf16: 72 us, 6.0 TB/s (a copy of a gigabyte: 5.2).  Backward 26001 x 1024 fp16 with one gate: 73 us for 320 MB, 4.7 TB/s in the main kernel, 5 us of sums over work-groups;
// a wavefront per SIMD has its registers full of column sums and two rows.  Backward, fp32 rows of 4097 to 8192 columns do without the second row (3001 x 5000: 100 us for 360 MB), and so
// do rows of more than 8192, whose shifts' sums are in LDS (2001 x 9000 bf16: 85 us for 216 MB, 1101 x 16384 bf16: 103, fp32, which spill: 209 for 433).
#include "rowtypes.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace {

constexpr int kMaxRows = 0x7FFFFFFF - 65536, kMaxCols = 16384;

struct NormArgs {
  int rows, d, kind, rows_per_gate, chunk, gates;  // chunk: rows of a worker, the lanes that hold a row
  int stream;                                      // results are written past the caches
  Divisor per_gate;
  float eps, resid_scale;
  int64_t ld_x, ld_y, ld_h, ld_n;
  const void *x, *y, *post_gain, *post_shift, *gate, *pre_gain, *pre_shift;
  void *h, *n;
  float* stats;
  // backward
  int64_t ld_dh, ld_dn, ld_dx, ld_dy;
  const void *dh, *dn;
  void *dx, *dy, *dpost_gain, *dpost_shift, *dgate, *dpre_gain, *dpre_shift;
  float *partial, *gate_partial;
  int groups, pitch, sums;  // work-groups of the backward pass, floats of a row of partial sums, such rows of a work-group
};

typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));

// Sum over the LANES lanes (of WAVES wavefronts) that hold a row; every lane gets it.  red: WAVES floats of LDS that the call before the last
// one before this may have used, but not the last.
template <int LANES, int WAVES>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = lanes_sum<LANES>(v);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += red[w];
  }
  return v;
}

// Of a work-group whose rows are held by `waves` wavefronts each.
constexpr int threads_of(int waves) { return waves > 4 ? 64 * waves : waves == 2 ? 128 : 256; }

// LANES lanes of each of WAVES wavefronts hold a row: every LANES * WAVES-th of its vectors of 16 bytes, VECS a lane (or none, and an element each, of rows
// shorter than that).  RAGGED: d is no multiple of a vector; the last one then ends with the row and has elements in common with the one before.  A lane to
// which nothing is left takes the last vector once more.  What lanes have in common they compute and store alike, bit for bit, and one of them adds it to
// the sums over the row.  So no access hangs on a branch, and the compiler can tell which of the accesses in flight a wait is for.
template <typename T, int VECS, int LANES, int WAVES, bool RAGGED_>
struct Shape {
  typedef T type;
  static constexpr bool RAGGED = RAGGED_;
  static constexpr int kVec = VECS ? Row<T>::kVec : 1, kN = VECS ? VECS : 1, kStep = LANES * WAVES * kVec, kE = kN * kVec;  // kE: elements of a lane
  static constexpr int kLanes = LANES, kWaves = WAVES, kCover = kN * kStep;
  static constexpr int kThreads = threads_of(WAVES);
  static constexpr int kRows = kThreads / (LANES * WAVES);  // workers of a work-group
  typedef T vec __attribute__((ext_vector_type(kVec), aligned(sizeof(T))));
  static __device__ __forceinline__ int worker() { return WAVES > 1 ? 0 : threadIdx.x / LANES; }
  static __device__ __forceinline__ int lane() { return WAVES > 1 ? threadIdx.x : threadIdx.x % LANES; }
};
template <typename S>
struct Columns {
  int at[S::kN];    // the first column of every vector
  int skip[S::kN];  // and how many of its elements, from its first, another lane adds up
  __device__ __forceinline__ explicit Columns(int d) {
#pragma unroll
    for (int i = 0; i < S::kN; ++i) {
      const int c = S::lane() * S::kVec + i * S::kStep;
      at[i] = min(c, d - S::kVec);
      skip[i] = min(c - at[i], S::kVec);
    }
  }
};

// A lane's share of a row, as it lies in memory; converted where it is used.
template <typename S>
struct Share {
  typedef typename S::type T;
  typedef typename S::vec vec;
  vec v[S::kN];
  __device__ __forceinline__ float operator()(int e) const { return (float)v[e / S::kVec][e % S::kVec]; }
  __device__ __forceinline__ void load(const void* base, int64_t at, const Columns<S>& c) {
#pragma unroll
    for (int i = 0; i < S::kN; ++i) v[i] = *reinterpret_cast<const vec*>(static_cast<const T*>(base) + at + c.at[i]);
  }
  __device__ __forceinline__ void store(void* base, int64_t at, const Columns<S>& c) const {
#pragma unroll
    for (int i = 0; i < S::kN; ++i) *reinterpret_cast<vec*>(static_cast<T*>(base) + at + c.at[i]) = v[i];
  }
  // Past the caches.  (The empty asm keeps the compiler from merging these stores with ordinary ones on the other side of a branch, as which both would end up.)
  __device__ __forceinline__ void store_nt(void* base, int64_t at, const Columns<S>& c) const {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < S::kN; ++i) __builtin_nontemporal_store(v[i], reinterpret_cast<vec*>(static_cast<T*>(base) + at + c.at[i]));
    asm volatile("" ::: "memory");
  }
  __device__ __forceinline__ void set(const float (&x)[S::kE]) {
#pragma unroll
    for (int e = 0; e < S::kE; ++e) v[e / S::kVec][e % S::kVec] = (T)x[e];
  }
  __device__ __forceinline__ void fill(float x) {
#pragma unroll
    for (int e = 0; e < S::kE; ++e) v[e / S::kVec][e % S::kVec] = (T)x;
  }
  // What was loaded has arrived.  Asked for ahead of a row's stores, which the next wait for a load would otherwise wait for too (both count down one counter, in order).
  __device__ __forceinline__ void arrive() {
#pragma unroll
    for (int i = 0; i < S::kN; ++i) {
      if constexpr (S::kVec > 1) {
        asm volatile("" : "+v"(v[i]));
      } else {
        T t = v[i][0];
        if constexpr (sizeof(T) == 4) {
          asm volatile("" : "+v"(t));
        } else {
          uint16_t bits = __builtin_bit_cast(uint16_t, t);
          asm volatile("" : "+v"(bits));
          t = __builtin_bit_cast(T, bits);
        }
        v[i][0] = t;
      }
    }
  }
};
// Sum over a lane's own elements of f(element).
template <typename S, typename F>
__device__ __forceinline__ float own_sum(const Columns<S>& c, F f) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < S::kN; ++i) {
    float p = 0.f;
#pragma unroll
    for (int e = 0; e < S::kVec; ++e) {
      const float x = f(i * S::kVec + e);
      p += !S::RAGGED || e >= c.skip[i] ? x : 0.f;
    }
    s += S::RAGGED || c.skip[i] == 0 ? p : 0.f;
  }
  return s;
}
// Sums in fp32.
template <typename S>
__device__ __forceinline__ void st_sums(float* row, const Columns<S>& c, const float (&x)[S::kE]) {
  typedef float any4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int i = 0; i < S::kN; ++i) {
    if constexpr (S::kVec == 1) {
      row[c.at[i]] = x[i];
    } else {
#pragma unroll
      for (int e = 0; e < S::kVec; e += 4)
        *reinterpret_cast<any4*>(row + c.at[i] + e) = any4{x[i * S::kVec + e], x[i * S::kVec + e + 1], x[i * S::kVec + e + 2], x[i * S::kVec + e + 3]};
    }
  }
}
template <int E>
__device__ __forceinline__ void fill(float (&v)[E], float x) {
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = x;
}

// Which gate a worker's rows take: one for all rows or none (GROUPED = false), or row after row the one of row / rows_per_gate.
struct GateRows {
  int64_t row = -1, end = 0;  // the gate at hand, and the row behind its last
  __device__ __forceinline__ bool next(int64_t r, int rows_per_gate) {  // whether row r, the one behind the last asked for, takes another one
    if (r < end) return false;
    row = row < 0 ? (int64_t)((uint32_t)r / (uint32_t)rows_per_gate) : row + 1;
    end = (row + 1) * rows_per_gate;
    return true;
  }
};

// Forward.  Gains, shifts and a gate for all rows stay in registers, and a worker's next row is asked for before the one at hand is worked on.
template <typename S, bool GROUPED>
__global__ void __launch_bounds__(S::kThreads) gated_norm_fwd_kernel(const NormArgs a) {
  constexpr int E = S::kE, LANES = S::kLanes, WAVES = S::kWaves;
  using V = Share<S>;
  __shared__ float red[2][WAVES];
  touch(a);
  const int d = a.d;
  const Columns<S> c(d);
  const float inv_d = 1.f / (float)d;
  const int64_t worker = (int64_t)blockIdx.x * S::kRows + S::worker();
  const int64_t begin = min(worker * a.chunk, (int64_t)a.rows), end = min(begin + a.chunk, (int64_t)a.rows);
  V post_gain, post_shift, pre_gain, pre_shift, gate, next_gate, next_x, next_y;
  auto vectors = [&] {
    if (a.post_gain) post_gain.load(a.post_gain, 0, c);
    if (a.post_shift) post_shift.load(a.post_shift, 0, c);
    if (!GROUPED && a.gate) gate.load(a.gate, 0, c);
    if (a.n) pre_gain.load(a.pre_gain, 0, c);
    if (a.pre_shift) pre_shift.load(a.pre_shift, 0, c);
  };
  constexpr bool AHEAD = WAVES <= 8 || E <= 8;  // (16 wavefronts of 16 columns a lane: 128 registers, which do not hold two rows and the gains)
  if (AHEAD) vectors();
  auto ask = [&](int64_t row) {
    next_x.load(a.x, row * a.ld_x, c);
    if (a.y) next_y.load(a.y, row * a.ld_y, c);
    if (GROUPED) {
      uint32_t rest;
      next_gate.load(a.gate, (int64_t)div_mod((uint32_t)row, a.per_gate, rest) * d, c);
    }
  };
  // v -> (v - mean) / sqrt(mean((v - mean)^2) + eps), two passes over the registers
  auto normalise = [&](float (&v)[E], float& mean, float& rstd) {
    mean = 0.f;
    if (a.kind == NMT_NORM_LAYER) {
      mean = row_sum<LANES, WAVES>(own_sum<S>(c, [&](int e) { return v[e]; }), red[0]) * inv_d;
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] -= mean;
    }
    rstd = 1.f / sqrtf(row_sum<LANES, WAVES>(own_sum<S>(c, [&](int e) { return v[e] * v[e]; }), red[1]) * inv_d + a.eps);
    if (WAVES > 1 && a.kind != NMT_NORM_LAYER) __syncthreads();  // (red[1] may be next)
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= rstd;
  };
  if (AHEAD && begin < end) ask(begin);
  for (int64_t row = begin; row < end; ++row) {
    if (!AHEAD) {
      ask(row);
      vectors();
    }
    const V x = next_x, y = next_y;
    if (GROUPED) gate = next_gate;
    if (AHEAD && row + 1 < end) ask(row + 1);
    if (AHEAD) __builtin_amdgcn_sched_barrier(0);
    float h[E], mean_y = 0.f, rstd_y = 1.f, mean_h = 0.f, rstd_h = 1.f;
    V out_h, out_n;
#pragma unroll
    for (int e = 0; e < E; ++e) h[e] = x(e);
    if (a.y) {
      float z[E];
#pragma unroll
      for (int e = 0; e < E; ++e) z[e] = y(e);
      if (a.post_gain) {
        normalise(z, mean_y, rstd_y);
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] *= post_gain(e);
        if (a.post_shift)
#pragma unroll
          for (int e = 0; e < E; ++e) z[e] += post_shift(e);
      }
      if (a.gate)
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] *= gate(e);
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] = a.resid_scale * h[e] + z[e];
      out_h.set(h);
    }
    if (a.n) {
      normalise(h, mean_h, rstd_h);
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] *= pre_gain(e);
      if (a.pre_shift)
#pragma unroll
        for (int e = 0; e < E; ++e) h[e] += pre_shift(e);
      out_n.set(h);
    }
    if (WAVES > 1 && !a.post_gain && !a.n) {  // (h may lie where x does, and lanes of two wavefronts may have loaded the same of it: no sum over the row has held the first up)
      out_h.arrive();
      __syncthreads();
    }
    if (AHEAD) {
      next_x.arrive();
      if (a.y) next_y.arrive();
      if (GROUPED) next_gate.arrive();
    }
    if (a.stream) {
      if (a.y) out_h.store_nt(a.h, row * a.ld_h, c);
      if (a.n) out_n.store_nt(a.n, row * a.ld_n, c);
    } else {
      if (a.y) out_h.store(a.h, row * a.ld_h, c);
      if (a.n) out_n.store(a.n, row * a.ld_n, c);
    }
    if (a.stats && S::lane() == 0) *reinterpret_cast<float4_any*>(a.stats + 4 * row) = float4_any{mean_y, rstd_y, mean_h, rstd_h};
  }
}

// Backward.  A worker takes `chunk` rows in a row and keeps column sums in registers, of dn hhat (0) for the gain before the next block, of D yhat (1)
// for the gain after this one, D = dh, and, if there are SHIFTS, of dn (2) and D (3) for the shifts.  One gate for all rows (or none): the gradients of gain,
// shift and gate all follow from the totals over dh.  GROUPED: D = gate dh, and the gate's gradient is a sum of its own, over its rows; where the gate's
// rows end it is written if all of them were this worker's, and else left as a partial sum, of which a worker has two at most (of the gate it
// begins in, if that began before it, and of the one it ends in).
template <typename S, bool GROUPED, bool SHIFTS>
__global__ void __launch_bounds__(S::kThreads, S::kWaves > 12 ? 4 : S::kWaves > 8 ? 3 : S::kE < 16 || S::kWaves == 8 ? 2 : 1) gated_norm_bwd_kernel(const NormArgs a) {
  constexpr int E = S::kE, LANES = S::kLanes, WAVES = S::kWaves, SUMS = SHIFTS ? 4 : 2;
  using V = Share<S>;
  __shared__ float red[4][WAVES];
  __shared__ __attribute__((aligned(16))) float sums[S::kRows > 1 ? SUMS : 1][S::kRows > 1 ? S::kRows * S::kCover : 1];
  // Twelve wavefronts have 168 registers a lane, sixteen 128: the shifts' sums, which are added up without a product, are in LDS (with all sums in the registers of eight
  // 2001 x 9000 bf16 took 316 us instead of 85, 1101 x 16384 233 instead of 103; sixteen wavefronts for the former 113).
  constexpr bool WIDE = WAVES > 8;
  constexpr int HELD = WIDE ? 2 : SUMS;
  __shared__ float4 outside[WIDE && SHIFTS ? 2 * E / 4 : 1][WIDE && SHIFTS ? S::kThreads : 1];
  touch(a);
  const int d = a.d;
  const Columns<S> c(d);
  const float inv_d = 1.f / (float)d;
  const int64_t worker = (int64_t)blockIdx.x * S::kRows + S::worker();
  const int64_t begin = min(worker * a.chunk, (int64_t)a.rows), end = min(begin + a.chunk, (int64_t)a.rows);
  V gain, shift, pre, gate, next_gate, next_dh, next_dn, next_h, next_y;
  float4_any next_st;
  gain.fill(1.f), shift.fill(0.f), gate.fill(1.f), next_dh.fill(0.f);  // (where there is none)
  auto vectors_after = [&] {
    if (a.post_gain) gain.load(a.post_gain, 0, c);
    if (GROUPED && SHIFTS && a.post_shift) shift.load(a.post_shift, 0, c);
    if (!GROUPED && a.gate) gate.load(a.gate, 0, c);
  };
  auto vectors_before = [&] {
    if (a.dn) pre.load(a.pre_gain, 0, c);
  };
  // Where the column sums and a row fill the registers by themselves gains are fetched where they are used, row after row.
  constexpr bool LATE = WIDE && sizeof(typename S::type) == 4;  // y is not asked for before it is needed, and dx written before (1101 x 16384 275 -> 209 us)
  constexpr bool AHEAD = !WIDE && E * sizeof(typename S::type) <= 32;
  if (AHEAD) vectors_after(), vectors_before();
  float sum[HELD][E], gate_sum[GROUPED ? E : 1];
#pragma unroll
  for (int q = 0; q < HELD; ++q) fill(sum[q], 0.f);
  if constexpr (WIDE && SHIFTS)
#pragma unroll
    for (int i = 0; i < 2 * E / 4; ++i) outside[i][threadIdx.x] = float4{0.f, 0.f, 0.f, 0.f};
  auto add_outside = [&](int q, auto f) {  // (a lane's own)
    if constexpr (WIDE && SHIFTS)
#pragma unroll
      for (int i = 0; i < E / 4; ++i) {
        float4 t = outside[q * (E / 4) + i][threadIdx.x];
        t.x += f(4 * i), t.y += f(4 * i + 1), t.z += f(4 * i + 2), t.w += f(4 * i + 3);
        outside[q * (E / 4) + i][threadIdx.x] = t;
      }
  };
  GateRows gates;
  int64_t gate_row = -1;  // of the rows at hand
  bool other_gate = false;
  auto ask = [&](int64_t row) {
    next_st = *reinterpret_cast<const float4_any*>(a.stats + 4 * row);
    if (a.dn) {
      next_h.load(a.h, row * a.ld_h, c);
      next_dn.load(a.dn, row * a.ld_dn, c);
    }
    if (a.dh) next_dh.load(a.dh, row * a.ld_dh, c);
    if (a.y && !LATE) next_y.load(a.y, row * a.ld_y, c);
    if (GROUPED) {
      other_gate = gates.next(row, a.rows_per_gate);
      if (other_gate) next_gate.load(a.gate, gates.row * d, c);
    }
  };
  auto close_gate = [&](int64_t row) {  // row: the one behind its last of this worker
    if constexpr (GROUPED) {
      if (gate_row >= 0 && a.dgate) {
        const int64_t first = gate_row * a.rows_per_gate, last = min(first + a.rows_per_gate, (int64_t)a.rows);
        if (first >= begin && last <= row) {
          V out;
          out.set(gate_sum);
          out.store(a.dgate, gate_row * d, c);
        }
        else st_sums<S>(a.gate_partial + (2 * worker + (first >= begin)) * a.pitch, c, gate_sum);
      }
      fill(gate_sum, 0.f);
    }
  };
  if (AHEAD && begin < end) ask(begin);
  for (int64_t row = begin; row < end; ++row) {
    if (!AHEAD) {
      next_dh.fill(0.f), next_dn.fill(0.f), next_h.fill(0.f), next_y.fill(0.f);  // (nothing of a row is kept for the next one, there or not)
      pre.fill(1.f), gain.fill(1.f), shift.fill(0.f);
      if (!GROUPED) gate.fill(1.f);
      ask(row);
      vectors_before();
    }
    V dh = next_dh, dn = next_dn, h = next_h, y = next_y;
    // Where registers are short nothing formed from these is kept from one use to the next: it is formed again (3001 x 5000 fp32 119 -> 100 us).
    auto anew = [&](auto&... v) {
      if constexpr (!AHEAD) (v.arrive(), ...);
    };
    const float4_any st = next_st;
    if (GROUPED && other_gate) {
      close_gate(row);
      gate = next_gate;
      gate_row = gates.row;
    }
    if (AHEAD && row + 1 < end) ask(row + 1);
    if (AHEAD) __builtin_amdgcn_sched_barrier(0);
    float g[E];  // the gradient at h
#pragma unroll
    for (int e = 0; e < E; ++e) g[e] = dh(e);
    if (a.dn) {
      const float rstd = st[3], off = -st[2] * st[3];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        sum[0][e] += dn(e) * (h(e) * rstd + off);
        if (SHIFTS && !WIDE) sum[HELD - 2][e] += dn(e);
      }
      add_outside(0, [&](int e) { return dn(e); });
      anew(dn, h);
      const float m1 = a.kind == NMT_NORM_LAYER ? row_sum<LANES, WAVES>(own_sum<S>(c, [&](int e) { return dn(e) * pre(e); }), red[0]) * inv_d : 0.f;
      anew(dn, pre);
      const float m2 = row_sum<LANES, WAVES>(own_sum<S>(c, [&](int e) { return dn(e) * pre(e) * (h(e) * rstd + off); }), red[1]) * inv_d;
      anew(dn, h, pre);
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] += rstd * (dn(e) * pre(e) - m1 - (h(e) * rstd + off) * m2);
    }
    V out_x, out_y;
    {
      float out[E];
#pragma unroll
      for (int e = 0; e < E; ++e) out[e] = a.resid_scale * g[e];
      out_x.set(out);
    }
    if (LATE) {  // (a wait as the one below: dx may lie where dh does)
      out_x.arrive();
      __syncthreads();
      out_x.store(a.dx, row * a.ld_dx, c);
      if (a.y) y.load(a.y, row * a.ld_y, c);
    }
    if (!AHEAD) vectors_after();
    if (a.y) {
      const float rstd = st[1], off = -st[0] * st[1];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float yhat = y(e) * rstd + off;
        if constexpr (GROUPED) gate_sum[e] += g[e] * (SHIFTS ? yhat * gain(e) + shift(e) : yhat * gain(e));
        const float dz = gate(e) * g[e], at = GROUPED ? dz : g[e];
        sum[1][e] += at * yhat;
        if (SHIFTS && !WIDE) sum[HELD - 1][e] += at;
        if (!WIDE) g[e] = dz * gain(e);
      }
      if constexpr (WIDE) {
        add_outside(1, [&](int e) { return GROUPED ? gate(e) * g[e] : g[e]; });
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = gate(e) * g[e] * gain(e);
      }
      if (a.post_gain) {
        anew(y);
        const float m3 = a.kind == NMT_NORM_LAYER ? row_sum<LANES, WAVES>(own_sum<S>(c, [&](int e) { return g[e]; }), red[2]) * inv_d : 0.f;
        const float m4 = row_sum<LANES, WAVES>(own_sum<S>(c, [&](int e) { return g[e] * (y(e) * rstd + off); }), red[3]) * inv_d;
        anew(y);
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = rstd * (g[e] - m3 - (y(e) * rstd + off) * m4);
      }
      out_y.set(g);
    }
    if (AHEAD) {
      if (a.dn) next_h.arrive(), next_dn.arrive();
      if (a.dh) next_dh.arrive();
      if (a.y) next_y.arrive();
      asm volatile("" : "+v"(next_st));
    }
    if (WAVES > 1) {  // the sums' places are used again; and dx may lie where dh does, dy where dn, of which lanes of two wavefronts may have loaded the same
      if (!LATE) out_x.arrive();
      if (a.y) out_y.arrive();
      __syncthreads();
    }
    if (!LATE) out_x.store(a.dx, row * a.ld_dx, c);
    if (a.y) out_y.store(a.dy, row * a.ld_dy, c);
  }
  close_gate(end);
  // the work-group's column sums: its workers' in increasing order
  float* out = a.partial + (int64_t)blockIdx.x * SUMS * a.pitch;
  if constexpr (S::kRows == 1) {
#pragma unroll
    for (int q = 0; q < HELD; ++q) st_sums<S>(out + (int64_t)q * a.pitch, c, sum[q]);
    if constexpr (HELD < SUMS)
#pragma unroll
      for (int q = 0; q < SUMS - HELD; ++q) {
#pragma unroll
        for (int i = 0; i < E / 4; ++i) {
          const float4 t = outside[q * (E / 4) + i][threadIdx.x];
          sum[0][4 * i] = t.x, sum[0][4 * i + 1] = t.y, sum[0][4 * i + 2] = t.z, sum[0][4 * i + 3] = t.w;
        }
        st_sums<S>(out + (int64_t)(HELD + q) * a.pitch, c, sum[0]);
      }
  } else {
#pragma unroll
    for (int q = 0; q < SUMS; ++q) st_sums<S>(sums[q] + S::worker() * S::kCover, c, sum[q]);
    __syncthreads();
    for (int i = threadIdx.x; i < d; i += S::kThreads)
#pragma unroll
      for (int q = 0; q < SUMS; ++q) {
        float t = sums[q][i];
#pragma unroll
        for (int w = 1; w < S::kRows; ++w) t += sums[q][w * S::kCover + i];
        out[(int64_t)q * a.pitch + i] = t;
      }
  }
}

constexpr int kSumCols = 32, kSumLanes = 32, kSumAhead = 8;  // of a work-group of the last kernel

// Totals over the work-groups' partial sums, in a fixed order, and the gradients that follow from them; behind those work-groups
// the gates whose rows several workers had.
template <typename T, bool GROUPED>
__global__ void __launch_bounds__(kSumCols* kSumLanes) gated_norm_sums_kernel(const NormArgs a) {
  touch(a);
  const int cblocks = (a.d + kSumCols - 1) / kSumCols;
  const int cx = threadIdx.x % kSumCols, ry = threadIdx.x / kSumCols;
  if (GROUPED && (int)blockIdx.x >= 2 * cblocks) {
    // a row of gates per row of threads: the partial sums of its workers in increasing order
    const int block = blockIdx.x - 2 * cblocks;
    const int64_t g = (int64_t)(block / cblocks) * kSumLanes + ry;
    const int c = (block % cblocks) * kSumCols + cx;
    if (g >= a.gates || c >= a.d) return;
    const int64_t first = g * a.rows_per_gate, last = min(first + a.rows_per_gate, (int64_t)a.rows) - 1;
    const int64_t w0 = first / a.chunk, w1 = last / a.chunk;
    if (w0 == w1) return;  // (written already)
    float s = 0.f;
    for (int64_t w = w0; w <= w1; ++w) s += a.gate_partial[(2 * w + (first >= w * a.chunk)) * a.pitch + c];
    static_cast<T*>(a.dgate)[g * a.d + c] = (T)s;
    return;
  }
  __shared__ float red[2][kSumLanes][kSumCols + 1];
  const int which = blockIdx.x / cblocks, c = (blockIdx.x % cblocks) * kSumCols + cx;  // 0: before the next block, 1: after this one
  float s = 0.f, t = 0.f;
  if (c < a.d) {
    auto total = [&](int q) {
      const float* p = a.partial + (int64_t)q * a.pitch + c;
      const int64_t step = (int64_t)a.sums * a.pitch;
      float sum = 0.f;
      for (int b = ry; b < a.groups; b += kSumLanes * kSumAhead) {
        float v[kSumAhead];
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) v[u] = p[min(b + u * kSumLanes, a.groups - 1) * step];
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) sum += b + u * kSumLanes < a.groups ? v[u] : 0.f;
      }
      return sum;
    };
    s = total(which);
    if (a.sums > 2) t = total(which + 2);
  }
  red[0][ry][cx] = s;
  red[1][ry][cx] = t;
  __syncthreads();
  // half a wavefront for a column
  static_assert(kSumLanes == 32, "");
  const int lane = threadIdx.x % 32, mine = threadIdx.x / 32, col = c - cx + mine;
  s = lanes_sum<32>(red[0][lane][mine]);
  t = lanes_sum<32>(red[1][lane][mine]);
  if (lane || col >= a.d) return;
  auto at = [&](const void* p, float none) { return p ? (float)static_cast<const T*>(p)[col] : none; };
  auto put = [&](void* p, float v) {
    if (p) static_cast<T*>(p)[col] = (T)v;
  };
  if (which == 0) {
    put(a.dpre_gain, s);
    put(a.dpre_shift, t);
  } else {
    const float gate = GROUPED ? 1.f : at(a.gate, 1.f);
    put(a.dpost_gain, gate * s);
    put(a.dpost_shift, gate * t);
    if (!GROUPED) put(a.dgate, at(a.post_gain, 1.f) * s + (a.post_shift ? at(a.post_shift, 0.f) * t : 0.f));
  }
}

// What a row of d columns is held by: -1: 16 lanes of one column (of less than a vector), 0 to 3: 8, 16, 32, 64 lanes of 8, 4 to 7: 2 to 16 wavefronts of 8 columns a lane, or, backward and
// 16-bit, 1 to 8 of 16 (fp32: 8 of 16 instead of 16 of 8), 8: 16 of 16, backward 12;
// 9, more than 12288 columns: 16 of 16.
enum { kForward, kBackward, kBackwardWide };
int shape_of(int d, int type) {
  if (d < 16 / row_type_bytes(type)) return -1;
  int s = 0;
  for (int most = 64; s < 8 && d > most; ++s) most *= 2;
  return d > 12288 ? 9 : s;
}
int waves_of_row(int shape, int form) { return shape <= 3 ? 1 : shape == 9 ? 16 : shape == 8 ? (form == kForward ? 16 : 12) : form == kForward ? std::min(16, 2 << (shape - 4)) : std::min(8, (form == kBackward ? 1 : 2) << (shape - 4)); }
int workers_of(int shape, int form) { return shape < 0 ? 16 : shape <= 3 ? 32 >> shape : waves_of_row(shape, form) == 1 ? 4 : 1; }  // of a work-group
int backward_form(int type) { return type == NMT_F32 ? kBackwardWide : kBackward; }

// Forward: two rows a worker, so that the second's loads are under way while the first is worked on and gains are fetched half as often, if that still makes
// kFwdWaves wavefronts, and one otherwise (26001 x 1024 fp16, one row, two, three: 48, 43, 45 us; 2001 x 8000 fp32, one, two: 68, 61).
// Backward: every work-group leaves a row of column sums, so no more of them than run side by side (kBwdWaves: a wavefront per SIMD with its
// registers full; 1280 and 2048 cost 26001 x 1024 fp16 90 and 75 us instead of 74, and 3584 x 512 15 and 14 instead of 13).
constexpr int kFwdWaves = 4096, kBwdWaves = 1024;
int bwd_groups(int waves) { return std::max(kBwdWaves / waves, device_info().cus); }  // (of wavefronts for a row: one work-group to a compute unit)
constexpr int64_t kStreamFrom = 64 << 20;  // bytes of a result
constexpr int kMostGroups = (1 << 22) - 1;  // a grid has less than 2^32 threads, of which a work-group has 1024 at most

struct Split {
  int chunk, groups, workers, pitch;
};
Split split_rows(int rows, int d, int type, int form, int rows_per_gate) {
  const int shape = shape_of(d, type), at_once = workers_of(shape, form), waves = std::max(at_once > 1 ? 4 : 1, waves_of_row(shape, form));
  Split p;
  if (form == kForward) {
    p.chunk = (int64_t)rows * waves >= (int64_t)2 * kFwdWaves * at_once ? std::max(2, ceil_div(rows, (int64_t)at_once * kMostGroups)) : 1;
  } else {
    p.chunk = ceil_div(rows, bwd_groups(waves) * at_once);
    // Whole gates, so that no gate's rows are two workers' and none leaves a partial sum, if a gate has at most two runs' rows.  26001 x 1024 fp16, a run being 26 rows, with 27, 30, 40, 52 rows a gate:
    // 72, 73, 75, 83 us, and 78, 78, 77, 75 without; 2001 x 8192 with 16: 56 and 58.  Where a run nearly doubles the work-groups halve, and that costs more than it saves: the 52 above, and of
    // smaller calls 3584 x 512 with 8: 14.7 and 12.7, 52000 x 64 with 13: 17.4 and 15.8.
    if (rows_per_gate < rows && rows_per_gate <= 2 * (int64_t)p.chunk) p.chunk = ceil_div(p.chunk, rows_per_gate) * rows_per_gate;
  }
  p.groups = ceil_div(rows, p.chunk * at_once);
  p.workers = p.groups * at_once;
  p.pitch = (d + 7) / 8 * 8;
  return p;
}
// Of a pass of up to `rows` rows, of any type.
int64_t scratch_floats(int rows, int d, int rows_per_gate) {
  int64_t most = 0;
  for (int type : {NMT_F16, NMT_F32}) {
    const int shape = shape_of(d, type), form = backward_form(type), at_once = workers_of(shape, form), waves = std::max(at_once > 1 ? 4 : 1, waves_of_row(shape, form));
    const int64_t groups = std::min(ceil_div(rows, at_once), bwd_groups(waves)), pitch = (d + 7) / 8 * 8;
    most = std::max(most, groups * 4 * pitch + (rows_per_gate < rows ? groups * at_once * 2 * pitch : 0));
  }
  return most;
}

#define NORM_LAUNCH(KERNEL, T, VECS, LANES, WAVES, ...)                                                                  \
  if ((VECS) && a.d % Row<T>::kVec) {                                                                                    \
    using S = Shape<T, VECS, LANES, WAVES, true>;                                                                        \
    hipLaunchKernelGGL((KERNEL<S, __VA_ARGS__>), grid, dim3(S::kThreads), 0, stream, a);                                 \
  } else {                                                                                                               \
    using S = Shape<T, VECS, LANES, WAVES, false>;                                                                       \
    hipLaunchKernelGGL((KERNEL<S, __VA_ARGS__>), grid, dim3(S::kThreads), 0, stream, a);                                 \
  }
// FORM: see shape_of.
#define NORM_SHAPES(KERNEL, T, FORM, ...)                                                                                \
  constexpr int v8 = 8 / Row<T>::kVec, v = (FORM) == kBackward ? 2 * v8 : v8, w = (FORM) == kBackward ? 1 : 2;           \
  constexpr bool f = (FORM) == kForward;                                                                                 \
  switch (shape) {                                                                                                       \
    case -1: NORM_LAUNCH(KERNEL, T, 0, 16, 1, __VA_ARGS__) break;                                                        \
    case 0: NORM_LAUNCH(KERNEL, T, v8, 8, 1, __VA_ARGS__) break;                                                         \
    case 1: NORM_LAUNCH(KERNEL, T, v8, 16, 1, __VA_ARGS__) break;                                                        \
    case 2: NORM_LAUNCH(KERNEL, T, v8, 32, 1, __VA_ARGS__) break;                                                        \
    case 3: NORM_LAUNCH(KERNEL, T, v8, 64, 1, __VA_ARGS__) break;                                                        \
    case 4: NORM_LAUNCH(KERNEL, T, v, 64, w, __VA_ARGS__) break;                                                         \
    case 5: NORM_LAUNCH(KERNEL, T, v, 64, 2 * w, __VA_ARGS__) break;                                                     \
    case 6: NORM_LAUNCH(KERNEL, T, v, 64, 4 * w, __VA_ARGS__) break;                                                     \
    case 7: NORM_LAUNCH(KERNEL, T, f ? v8 : 2 * v8, 64, f ? 16 : 8, __VA_ARGS__) break;                                  \
    case 8: NORM_LAUNCH(KERNEL, T, 2 * v8, 64, f ? 16 : 12, __VA_ARGS__) break;                                          \
    default: NORM_LAUNCH(KERNEL, T, 2 * v8, 64, 16, __VA_ARGS__)                                                           \
  }

template <typename T>
void launch_fwd(const NormArgs& a, dim3 grid, int shape, bool grouped, hipStream_t stream) {
  if (grouped) { NORM_SHAPES(gated_norm_fwd_kernel, T, kForward, true) }
  else { NORM_SHAPES(gated_norm_fwd_kernel, T, kForward, false) }
}
template <typename T>
void launch_bwd(const NormArgs& a, dim3 grid, int shape, bool grouped, hipStream_t stream) {
  constexpr int form = sizeof(T) == 4 ? kBackwardWide : kBackward;  // (backward_form)
  const bool shifts = a.sums > 2;
  if (grouped && shifts) { NORM_SHAPES(gated_norm_bwd_kernel, T, form, true, true) }
  else if (grouped) { NORM_SHAPES(gated_norm_bwd_kernel, T, form, true, false) }
  else if (shifts) { NORM_SHAPES(gated_norm_bwd_kernel, T, form, false, true) }
  else { NORM_SHAPES(gated_norm_bwd_kernel, T, form, false, false) }
}
template <typename T>
void launch_sums(const NormArgs& a, bool grouped, hipStream_t stream) {
  const int cblocks = ceil_div(a.d, kSumCols);
  if (grouped) {
    const int64_t gates = a.dgate && a.chunk % a.rows_per_gate != 0 ? ceil_div(a.gates, kSumLanes) : 0;  // (otherwise no gate's rows are two workers')
    hipLaunchKernelGGL((gated_norm_sums_kernel<T, true>), dim3((uint32_t)(cblocks * (2 + gates))), dim3(kSumCols * kSumLanes), 0, stream, a);
  } else {
    hipLaunchKernelGGL((gated_norm_sums_kernel<T, false>), dim3(2 * cblocks), dim3(kSumCols * kSumLanes), 0, stream, a);
  }
}

int launch_sums(const NormArgs& a, int type, bool grouped, hipStream_t stream) {
  if (type == NMT_F16) launch_sums<half_t>(a, grouped, stream);
  else if (type == NMT_BF16) launch_sums<bf16_t>(a, grouped, stream);
  else launch_sums<float>(a, grouped, stream);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}

int check_common(const nmt_gated_norm* a, const char* who) {
  NMT_REQUIRE(a, "%s: null argument", who);
  NMT_REQUIRE(a->rows >= 0 && a->rows <= kMaxRows, "%s: %d rows", who, a->rows);
  NMT_REQUIRE(a->d >= 1 && a->d <= kMaxCols, "%s: d = %d outside [1, %d]", who, a->d, kMaxCols);
  NMT_REQUIRE(row_type_ok(a->type), "%s: unknown type %d", who, a->type);
  NMT_REQUIRE(a->kind == NMT_NORM_LAYER || a->kind == NMT_NORM_RMS, "%s: unknown kind of norm %d", who, a->kind);
  NMT_REQUIRE(std::isfinite(a->resid_scale), "%s: resid_scale is not finite", who);
  NMT_REQUIRE(!a->d_gate || a->rows_per_gate >= 1, "%s: rows_per_gate must be at least 1", who);
  return NMT_OK;
}
int check_block(const nmt_gated_norm* a, const char* who) {
  NMT_REQUIRE(!a->d_post_shift || a->d_post_gain, "%s: a shift after the block needs a gain", who);
  NMT_REQUIRE(a->d_y || (!a->d_post_gain && !a->d_gate), "%s: a gain or gate after the block needs the block's output", who);
  return NMT_OK;
}
#define NORM_ROWS(ptr, ld, what) NMT_REQUIRE(!(ptr) || a->rows <= 1 || (ld) >= a->d, "%s: rows of " what " overlap", who)

NormArgs common_args(const nmt_gated_norm* a) {
  NormArgs k = {};
  k.rows = a->rows, k.d = a->d, k.kind = a->kind;
  k.rows_per_gate = a->d_gate ? a->rows_per_gate : a->rows;
  k.gates = ceil_div(a->rows, k.rows_per_gate);
  k.per_gate = divisor((uint32_t)k.rows_per_gate);
  k.stream = (int64_t)a->rows * a->d * row_type_bytes(a->type) >= kStreamFrom;
  k.eps = a->eps, k.resid_scale = a->resid_scale;
  k.ld_x = a->ld_x, k.ld_y = a->ld_y, k.ld_h = a->ld_h, k.ld_n = a->ld_n;
  k.x = a->d_x, k.y = a->d_y, k.h = a->d_h, k.n = a->d_n, k.stats = a->d_stats;
  k.post_gain = a->d_post_gain, k.post_shift = a->d_post_shift, k.gate = a->d_gate, k.pre_gain = a->d_pre_gain, k.pre_shift = a->d_pre_shift;
  return k;
}

}  // namespace

extern "C" int nmt_op_gated_norm_fwd(const nmt_gated_norm* a, void* stream_) {
  const char* who = "nmt_op_gated_norm_fwd";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (const int rc = check_common(a, who); rc != NMT_OK) return rc;
  NMT_REQUIRE(a->eps > 0.f && std::isfinite(a->eps), "%s: eps must be positive", who);
  if (a->rows == 0) return NMT_OK;
  if (const int rc = check_block(a, who); rc != NMT_OK) return rc;
  NMT_REQUIRE(!a->d_pre_shift || a->d_pre_gain, "%s: a shift before the next block needs a gain", who);
  NMT_REQUIRE(!a->d_n == !a->d_pre_gain, "%s: the next block's input and its gain belong together", who);
  NMT_REQUIRE(a->d_y ? a->d_h != nullptr : !a->d_h && a->d_n, "%s: with a block's output the sum is written, without one the norm alone", who);
  NMT_REQUIRE(a->d_y || a->resid_scale == 1.f, "%s: without a block's output nothing is scaled: resid_scale is 1", who);
  NMT_REQUIRE(a->d_x, "%s: null pointer", who);
  NORM_ROWS(a->d_x, a->ld_x, "x");
  NORM_ROWS(a->d_y, a->ld_y, "y");
  NORM_ROWS(a->d_h, a->ld_h, "h");
  NORM_ROWS(a->d_n, a->ld_n, "n");
  NormArgs k = common_args(a);
  const Split p = split_rows(a->rows, a->d, a->type, kForward, a->rows);
  k.chunk = p.chunk;
  const bool grouped = a->d_gate && a->rows_per_gate < a->rows;
  const int shape = shape_of(a->d, a->type);
  if (a->type == NMT_F16) launch_fwd<half_t>(k, dim3(p.groups), shape, grouped, stream);
  else if (a->type == NMT_BF16) launch_fwd<bf16_t>(k, dim3(p.groups), shape, grouped, stream);
  else launch_fwd<float>(k, dim3(p.groups), shape, grouped, stream);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}

extern "C" int nmt_debug_gated_norm_grid(int32_t rows, int32_t d, int32_t type, int64_t* groups, int32_t* threads) {
  const char* who = "nmt_debug_gated_norm_grid";
  NMT_REQUIRE(rows >= 1 && rows <= kMaxRows && d >= 1 && d <= kMaxCols && row_type_ok(type) && groups && threads, "%s: bad argument", who);
  *groups = split_rows(rows, d, type, kForward, rows).groups;
  *threads = threads_of(waves_of_row(shape_of(d, type), kForward));
  return NMT_OK;
}

extern "C" int64_t nmt_op_gated_norm_bwd_scratch(int32_t rows, int32_t d, int32_t rows_per_gate) {
  if (rows < 0 || rows > kMaxRows || d < 1 || d > kMaxCols || rows_per_gate < 1) return NMT_EINVAL;
  return rows ? scratch_floats(rows, d, rows_per_gate) : 0;
}

extern "C" int nmt_op_gated_norm_bwd(const nmt_gated_norm* a, const nmt_gated_norm_grad* g, void* stream_) {
  const char* who = "nmt_op_gated_norm_bwd";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  if (const int rc = check_common(a, who); rc != NMT_OK) return rc;
  NMT_REQUIRE(g, "%s: null argument", who);
  if (a->rows == 0) {  // (sums over no rows; of gates there are none then but the one that all rows share)
    NormArgs k = {};
    k.d = a->d, k.sums = 4;
    k.dpost_gain = g->d_dpost_gain, k.dpost_shift = g->d_dpost_shift;
    k.dgate = a->d_gate && a->rows_per_gate == NMT_ONE_GATE ? g->d_dgate : nullptr;
    k.dpre_gain = g->d_dpre_gain, k.dpre_shift = g->d_dpre_shift;
    if (!k.dpost_gain && !k.dpost_shift && !k.dgate && !k.dpre_gain && !k.dpre_shift) return NMT_OK;
    return launch_sums(k, a->type, false, stream);
  }
  if (const int rc = check_block(a, who); rc != NMT_OK) return rc;
  NMT_REQUIRE(g->d_dh || g->d_dn, "%s: a gradient has to arrive at h or at n", who);
  NMT_REQUIRE(!g->d_dn || a->d_pre_gain, "%s: a gradient at n needs the gain before the next block", who);
  NMT_REQUIRE(g->d_dn || (!g->d_dpre_gain && !g->d_dpre_shift), "%s: no gradient arrives at n: those of its gain and shift are not formed", who);
  NMT_REQUIRE(!a->d_y == !g->d_dy, "%s: the block's output and its gradient belong together", who);
  NMT_REQUIRE(a->d_post_gain || (!g->d_dpost_gain && !g->d_dpost_shift), "%s: there is no gain after the block whose gradient could be formed", who);
  NMT_REQUIRE(a->d_gate || !g->d_dgate, "%s: there is no gate whose gradient could be formed", who);
  NMT_REQUIRE(a->d_stats && g->d_dx && (!g->d_dn || a->d_h), "%s: null pointer", who);
  NORM_ROWS(a->d_y, a->ld_y, "y");
  NORM_ROWS(a->d_h, a->ld_h, "h");
  NORM_ROWS(g->d_dh, g->ld_dh, "dh");
  NORM_ROWS(g->d_dn, g->ld_dn, "dn");
  NORM_ROWS(g->d_dx, g->ld_dx, "dx");
  NORM_ROWS(g->d_dy, g->ld_dy, "dy");
  NormArgs k = common_args(a);
  const bool grouped = a->d_gate && a->rows_per_gate < a->rows;
  const int64_t need = scratch_floats(a->rows, a->d, k.rows_per_gate);
  if (!g->d_scratch || g->scratch_floats < need) {
    nmt_set_error("%s: scratch of %lld floats, %lld needed", who, (long long)(g->d_scratch ? g->scratch_floats : 0), (long long)need);
    return NMT_ENOMEM;
  }
  NMT_REQUIRE(aligned16(g->d_scratch), "%s: the scratch buffer must be 16-byte aligned", who);
  const Split p = split_rows(a->rows, a->d, a->type, backward_form(a->type), k.rows_per_gate);
  k.chunk = p.chunk, k.groups = p.groups, k.pitch = p.pitch;
  k.sums = a->d_post_shift || g->d_dpost_shift || g->d_dpre_shift ? 4 : 2;
  k.partial = g->d_scratch, k.gate_partial = g->d_scratch + (int64_t)p.groups * 4 * p.pitch;
  k.ld_dh = g->ld_dh, k.ld_dn = g->ld_dn, k.ld_dx = g->ld_dx, k.ld_dy = g->ld_dy;
  k.dh = g->d_dh, k.dn = g->d_dn, k.dx = g->d_dx, k.dy = g->d_dy;
  k.dpost_gain = g->d_dpost_gain, k.dpost_shift = g->d_dpost_shift, k.dgate = g->d_dgate;
  k.dpre_gain = g->d_dpre_gain, k.dpre_shift = g->d_dpre_shift;
  const int shape = shape_of(a->d, a->type);
  const dim3 grid(p.groups);
  if (a->type == NMT_F16) launch_bwd<half_t>(k, grid, shape, grouped, stream);
  else if (a->type == NMT_BF16) launch_bwd<bf16_t>(k, grid, shape, grouped, stream);
  else launch_bwd<float>(k, grid, shape, grouped, stream);
  NMT_LAUNCH_CHECK();
  const bool sums = g->d_dpost_gain || g->d_dpost_shift || g->d_dgate || g->d_dpre_gain || g->d_dpre_shift;
  return sums ? launch_sums(k, a->type, grouped, stream) : NMT_OK;
}
