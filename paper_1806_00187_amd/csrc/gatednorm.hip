// The norms around a gated residual block, one pass over the rows each way:
//   h = a x + gate post(y), n = pre(h);  post, pre: LayerNorm or RMS norm with gain and shift.
// Bound by memory: forward reads x, y and writes h, n (n needs h's statistics, which are there while h is still in registers), backward
// reads y, h and the gradients at h and n and writes those at x and y.  A row is held in registers by 16 lanes (up to 128 columns), by a
// wavefront (up to 1024) or by up to 16 wavefronts.
#include "rowtypes.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace {

constexpr int kMaxRows = 0x7FFFFFFF - 65536, kMaxCols = 16384;

struct NormArgs {
  int rows, d, kind, rows_per_gate, chunk, gates;  // chunk: rows of a worker of the backward pass
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
  int groups, pitch;  // work-groups of the backward pass; floats of a row of partial sums
};

typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));

// Sum over the LANES lanes (of WAVES wavefronts) that hold a row; every lane gets it.  red: WAVES floats of LDS that the call before the last
// one before this may have used, but not the last.
template <int LANES, int WAVES>
__device__ __forceinline__ float row_sum(float v, float* red) {
  if constexpr (LANES == 16) {
    auto rot = [](float x, auto ctrl) {
      return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    v = rot(v, std::integral_constant<int, 0x128>{});  // row_ror:8
    v = rot(v, std::integral_constant<int, 0x124>{});  // row_ror:4
    v = rot(v, std::integral_constant<int, 0x4E>{});   // quad_perm:[2,3,0,1]
    return rot(v, std::integral_constant<int, 0xB1>{});  // quad_perm:[1,0,3,2]
  } else {
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
      __syncthreads();
      v = red[0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) v += red[w];
    }
    return v;
  }
}

// LANES lanes of each of WAVES wavefronts hold a row, E elements a lane, in vectors of 16 bytes LANES * WAVES vectors apart.
template <typename T, int E, int LANES, int WAVES>
struct Shape {
  static constexpr int kVec = Row<T>::kVec, kN = E / kVec, kStep = LANES * WAVES * kVec;
  static constexpr int kThreads = WAVES > 4 ? 64 * WAVES : WAVES == 2 ? 128 : 256;
  static constexpr int kRows = kThreads / (LANES * WAVES);  // rows a work-group holds at a time
  static __device__ __forceinline__ int worker() { return WAVES > 1 ? 0 : threadIdx.x / LANES; }
  static __device__ __forceinline__ int column() { return (WAVES > 1 ? threadIdx.x : threadIdx.x % LANES) * kVec; }
};
#define NORM_SHAPE(T, E, LANES, WAVES)              \
  using S = Shape<T, E, LANES, WAVES>;              \
  constexpr int VEC = S::kVec, NV = S::kN, STEP = S::kStep

template <bool RAGGED, typename S, typename T, int E>
__device__ __forceinline__ void ld_all(const T* row, int c0, int d, float (&v)[E]) {
#pragma unroll
  for (int i = 0; i < S::kN; ++i) ld_row<RAGGED>(row, c0 + i * S::kStep, d, v + i * S::kVec);
}
template <bool RAGGED, typename S, typename T, int E>
__device__ __forceinline__ void st_all(T* row, int c0, int d, const float (&v)[E]) {
#pragma unroll
  for (int i = 0; i < S::kN; ++i) st_row<RAGGED>(row, c0 + i * S::kStep, d, v + i * S::kVec);
}

// Sums in fp32: whole vectors, up to the pitch of their rows, a multiple of eight.
template <typename S, int E>
__device__ __forceinline__ void st_sums(float* row, int c0, int d, const float (&v)[E]) {
#pragma unroll
  for (int i = 0; i < S::kN; ++i)
    if (const int c = c0 + i * S::kStep; c < d)
#pragma unroll
      for (int e = 0; e < S::kVec; e += 4) *reinterpret_cast<floatx4*>(row + c + e) = floatx4{v[i * S::kVec + e], v[i * S::kVec + e + 1], v[i * S::kVec + e + 2], v[i * S::kVec + e + 3]};
}

template <typename T, int E, int LANES, int WAVES, bool RAGGED>
__global__ void __launch_bounds__((Shape<T, E, LANES, WAVES>::kThreads)) gated_norm_fwd_kernel(const NormArgs a) {
  NORM_SHAPE(T, E, LANES, WAVES);
  __shared__ float red[2][WAVES];
  const int c0 = S::column(), d = a.d;
  const float inv_d = 1.f / (float)d;
  // v -> (v - mean) / sqrt(mean((v - mean)^2) + eps), two passes over the registers
  auto normalise = [&](float (&v)[E], float& mean, float& rstd) {
    mean = 0.f;
    if (a.kind == NMT_NORM_LAYER) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) s += v[e];
      mean = row_sum<LANES, WAVES>(s, red[0]) * inv_d;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float& x = v[i * VEC + e];
        const int c = c0 + i * STEP;
        x = (RAGGED ? c + e < d : c < d) ? x - mean : 0.f;
        q += x * x;
      }
    rstd = 1.f / sqrtf(row_sum<LANES, WAVES>(q, red[1]) * inv_d + a.eps);
    if (WAVES > 1 && a.kind != NMT_NORM_LAYER) __syncthreads();  // (red[1] may be next)
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= rstd;
  };
  auto affine = [&](float (&v)[E], const void* gain, const void* shift) {
    float g[E];
    ld_all<RAGGED, S>(static_cast<const T*>(gain), c0, d, g);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= g[e];
    if (shift) {
      ld_all<RAGGED, S>(static_cast<const T*>(shift), c0, d, g);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += g[e];
    }
  };
  const int64_t stride = (int64_t)gridDim.x * S::kRows;
  for (int64_t row = (int64_t)blockIdx.x * S::kRows + S::worker(); row < a.rows; row += stride) {
    float h[E], mean_y = 0.f, rstd_y = 1.f, mean_h = 0.f, rstd_h = 1.f;
    ld_all<RAGGED, S>(static_cast<const T*>(a.x) + row * a.ld_x, c0, d, h);
    if (a.y) {
      float y[E];
      ld_all<RAGGED, S>(static_cast<const T*>(a.y) + row * a.ld_y, c0, d, y);
      if (a.post_gain) {
        normalise(y, mean_y, rstd_y);
        affine(y, a.post_gain, a.post_shift);
      }
      if (a.gate) {
        float g[E];
        ld_all<RAGGED, S>(static_cast<const T*>(a.gate) + (int64_t)((uint32_t)row / (uint32_t)a.rows_per_gate) * d, c0, d, g);
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] *= g[e];
      }
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] = a.resid_scale * h[e] + y[e];
      st_all<RAGGED, S>(static_cast<T*>(a.h) + row * a.ld_h, c0, d, h);
    }
    if (a.n) {
      normalise(h, mean_h, rstd_h);
      affine(h, a.pre_gain, a.pre_shift);
      st_all<RAGGED, S>(static_cast<T*>(a.n) + row * a.ld_n, c0, d, h);
    }
    if (a.stats && c0 == 0) *reinterpret_cast<float4_any*>(a.stats + 4 * row) = float4_any{mean_y, rstd_y, mean_h, rstd_h};
  }
}

// Backward.  A worker (the lanes that hold a row) takes `chunk` rows in a row and keeps four column sums in registers: of dh yhat and dh, from which
// the gradients of post's gain and shift (times the gate) and of the gate (gain, shift times the two) follow, and of dn hhat and dn.
// One gate for all (GROUPED = false): the factors are applied to the totals.  Otherwise whenever a gate's rows end: its gradient is written if
// all its rows were this worker's, and else left as a partial sum, of which a worker has two at most (the gate it begins in, begun before it, and the one it ends in).
template <typename T, int E, int LANES, int WAVES, bool RAGGED, bool GROUPED>
__global__ void __launch_bounds__((Shape<T, E, LANES, WAVES>::kThreads)) gated_norm_bwd_kernel(const NormArgs a) {
  NORM_SHAPE(T, E, LANES, WAVES);
  __shared__ float red[4][WAVES];
  __shared__ float sums[S::kRows > 1 ? S::kRows * LANES * E : 1];
  const int c0 = S::column(), d = a.d;
  const float inv_d = 1.f / (float)d;
  const int64_t worker = (int64_t)blockIdx.x * S::kRows + S::worker();
  const int64_t begin = min(worker * a.chunk, (int64_t)a.rows), end = min(begin + a.chunk, (int64_t)a.rows);
  auto fill = [](float (&v)[E], float x) {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = x;
  };
  float gain[E], shift[E], gate[E], pre[E];  // 1, 0, 1, - where there is none
  fill(gain, 1.f), fill(shift, 0.f), fill(gate, 1.f), fill(pre, 0.f);
  if (a.post_gain) ld_all<RAGGED, S>(static_cast<const T*>(a.post_gain), c0, d, gain);
  if (GROUPED && a.post_shift) ld_all<RAGGED, S>(static_cast<const T*>(a.post_shift), c0, d, shift);
  if (!GROUPED && a.gate) ld_all<RAGGED, S>(static_cast<const T*>(a.gate), c0, d, gate);
  if (a.dn) ld_all<RAGGED, S>(static_cast<const T*>(a.pre_gain), c0, d, pre);
  float sum_a[E], sum_b[E], sum_p[E], sum_q[E], gate_a[E], gate_b[E];
  fill(sum_a, 0.f), fill(sum_b, 0.f), fill(sum_p, 0.f), fill(sum_q, 0.f);
  int64_t gate_row = -1, gate_end = begin;  // the gate at hand and the row behind its last here
  auto close_gate = [&](int64_t row) {      // (row: the one behind its last of this worker)
    if (gate_row < 0) return;
    float g[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      sum_a[e] += gate[e] * gate_a[e];
      sum_b[e] += gate[e] * gate_b[e];
      g[e] = gain[e] * gate_a[e] + shift[e] * gate_b[e];
    }
    if (!a.dgate) return;
    const int64_t first = gate_row * a.rows_per_gate, last = min(first + a.rows_per_gate, (int64_t)a.rows);
    if (first >= begin && last <= row) {
      st_all<RAGGED, S>(static_cast<T*>(a.dgate) + gate_row * d, c0, d, g);
    } else {
      st_sums<S>(a.gate_partial + (2 * worker + (first >= begin)) * a.pitch, c0, d, g);
    }
  };
  for (int64_t row = begin; row < end; ++row) {
    if (GROUPED && row == gate_end) {
      close_gate(row);
      gate_row = (uint32_t)row / (uint32_t)a.rows_per_gate;
      gate_end = min((gate_row + 1) * a.rows_per_gate, end);
      ld_all<RAGGED, S>(static_cast<const T*>(a.gate) + gate_row * d, c0, d, gate);
      fill(gate_a, 0.f), fill(gate_b, 0.f);
    }
    const float4_any st = *reinterpret_cast<const float4_any*>(a.stats + 4 * row);
    float dh[E];
    fill(dh, 0.f);
    if (a.dh) ld_all<RAGGED, S>(static_cast<const T*>(a.dh) + row * a.ld_dh, c0, d, dh);
    if (a.dn) {
      float h[E], dn[E];
      ld_all<RAGGED, S>(static_cast<const T*>(a.h) + row * a.ld_h, c0, d, h);
      ld_all<RAGGED, S>(static_cast<const T*>(a.dn) + row * a.ld_dn, c0, d, dn);
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        h[e] = (h[e] - st[2]) * st[3];
        sum_p[e] += dn[e] * h[e];
        sum_q[e] += dn[e];
        dn[e] *= pre[e];
        s1 += dn[e];
        s2 += dn[e] * h[e];
      }
      const float m1 = a.kind == NMT_NORM_LAYER ? row_sum<LANES, WAVES>(s1, red[0]) * inv_d : 0.f;
      const float m2 = row_sum<LANES, WAVES>(s2, red[1]) * inv_d;
#pragma unroll
      for (int e = 0; e < E; ++e) dh[e] += st[3] * (dn[e] - m1 - h[e] * m2);
    }
    float out[E];
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = a.resid_scale * dh[e];
    st_all<RAGGED, S>(static_cast<T*>(a.dx) + row * a.ld_dx, c0, d, out);
    if (a.y) {
      float y[E];
      ld_all<RAGGED, S>(static_cast<const T*>(a.y) + row * a.ld_y, c0, d, y);
      float s3 = 0.f, s4 = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        y[e] = (y[e] - st[0]) * st[1];
        float& ga = GROUPED ? gate_a[e] : sum_a[e];
        float& gb = GROUPED ? gate_b[e] : sum_b[e];
        ga += dh[e] * y[e];
        gb += dh[e];
        out[e] = gate[e] * dh[e] * gain[e];
        s3 += out[e];
        s4 += out[e] * y[e];
      }
      if (a.post_gain) {
        const float m3 = a.kind == NMT_NORM_LAYER ? row_sum<LANES, WAVES>(s3, red[2]) * inv_d : 0.f;
        const float m4 = row_sum<LANES, WAVES>(s4, red[3]) * inv_d;
#pragma unroll
        for (int e = 0; e < E; ++e) out[e] = st[1] * (out[e] - m3 - y[e] * m4);
      }
      st_all<RAGGED, S>(static_cast<T*>(a.dy) + row * a.ld_dy, c0, d, out);
    }
    if (WAVES > 1) __syncthreads();  // (the sums' places are used again)
  }
  if (GROUPED) close_gate(end);
  // the work-group's column sums: its workers' in increasing order
  auto leave = [&](float (&v)[E], int which) {
    float* out = a.partial + ((int64_t)blockIdx.x * 4 + which) * a.pitch;
    if constexpr (S::kRows == 1) {
      st_sums<S>(out, c0, d, v);
    } else {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sums[(size_t)S::worker() * LANES * E + c0 + i * STEP + e] = v[i * VEC + e];
      __syncthreads();
      for (int c = threadIdx.x; c < d; c += S::kThreads) {
        float t = sums[c];
#pragma unroll
        for (int w = 1; w < S::kRows; ++w) t += sums[w * LANES * E + c];
        out[c] = t;
      }
    }
  };
  leave(sum_a, 0);
  leave(sum_b, 1);
  leave(sum_p, 2);
  leave(sum_q, 3);
}

constexpr int kSumCols = 32, kSumLanes = 32;  // of a work-group of the last kernel

// Totals over the work-groups' partial sums, in a fixed order, and the gradients that follow from them; behind those work-groups
// the gates whose rows several workers had.
template <typename T, bool GROUPED>
__global__ void __launch_bounds__(kSumCols* kSumLanes) gated_norm_sums_kernel(const NormArgs a) {
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
  const int pair = blockIdx.x / cblocks, c = (blockIdx.x % cblocks) * kSumCols + cx;
  float s = 0.f, t = 0.f;
  if (c < a.d)
    for (int b = ry; b < a.groups; b += kSumLanes) {
      const float* p = a.partial + ((int64_t)b * 4 + 2 * pair) * a.pitch + c;
      s += p[0];
      t += p[a.pitch];
    }
  red[0][ry][cx] = s;
  red[1][ry][cx] = t;
  __syncthreads();
  if (ry || c >= a.d) return;
  for (int r = 1; r < kSumLanes; ++r) {
    s += red[0][r][cx];
    t += red[1][r][cx];
  }
  auto at = [&](const void* p, float none) { return p ? (float)static_cast<const T*>(p)[c] : none; };
  auto put = [&](void* p, float v) {
    if (p) static_cast<T*>(p)[c] = (T)v;
  };
  if (pair) {
    put(a.dpre_gain, s);
    put(a.dpre_shift, t);
  } else {
    const float gate = GROUPED ? 1.f : at(a.gate, 1.f);
    put(a.dpost_gain, gate * s);
    put(a.dpost_shift, gate * t);
    if (!GROUPED) put(a.dgate, at(a.post_gain, 1.f) * s + at(a.post_shift, 0.f) * t);
  }
}

// What a row of d columns is held by: 0: 16 lanes of 8 columns, 1: 64 of 8, 2: 64 of 16, 3 to 6: 2, 4, 8, 16 wavefronts of 16 columns a lane.
int shape_of(int d) {
  int s = 0;
  for (int most = 128; s < 6 && d > most; ++s) most = s == 0 ? 512 : most * 2;
  return s;
}
int rows_at_a_time(int shape) { return shape == 0 ? 16 : shape <= 2 ? 4 : 1; }
int threads_of(int shape) { return shape <= 2 ? 256 : 64 << (shape - 2); }

constexpr int kFwdGroups = 2048, kBwdWaves = 2048;

struct BwdPlan {
  int chunk, groups, workers, pitch;
};
BwdPlan bwd_plan(int rows, int d) {
  const int shape = shape_of(d), at_once = rows_at_a_time(shape);
  const int most = kBwdWaves / (threads_of(shape) / 64);
  BwdPlan p;
  p.chunk = std::max<int64_t>(1, ((int64_t)rows + (int64_t)most * at_once - 1) / ((int64_t)most * at_once));
  p.groups = (int)(((int64_t)rows + (int64_t)p.chunk * at_once - 1) / ((int64_t)p.chunk * at_once));
  p.workers = p.groups * at_once;
  p.pitch = (d + 7) / 8 * 8;
  return p;
}
int64_t scratch_floats(int rows, int d, int rows_per_gate) {
  const BwdPlan p = bwd_plan(rows, d);
  return (int64_t)p.groups * 4 * p.pitch + (rows_per_gate < rows ? (int64_t)p.workers * 2 * p.pitch : 0);
}

#define NORM_LAUNCH(KERNEL, T, E, LANES, WAVES, ...)                                                                              \
  if (ragged)                                                                                                                     \
    hipLaunchKernelGGL((KERNEL<T, E, LANES, WAVES, true, ##__VA_ARGS__>), grid, dim3(Shape<T, E, LANES, WAVES>::kThreads), 0, stream, a); \
  else                                                                                                                            \
    hipLaunchKernelGGL((KERNEL<T, E, LANES, WAVES, false, ##__VA_ARGS__>), grid, dim3(Shape<T, E, LANES, WAVES>::kThreads), 0, stream, a)
#define NORM_SHAPES(KERNEL, T, ...)                                   \
  switch (shape) {                                                    \
    case 0: NORM_LAUNCH(KERNEL, T, 8, 16, 1, ##__VA_ARGS__); break;   \
    case 1: NORM_LAUNCH(KERNEL, T, 8, 64, 1, ##__VA_ARGS__); break;   \
    case 2: NORM_LAUNCH(KERNEL, T, 16, 64, 1, ##__VA_ARGS__); break;  \
    case 3: NORM_LAUNCH(KERNEL, T, 16, 64, 2, ##__VA_ARGS__); break;  \
    case 4: NORM_LAUNCH(KERNEL, T, 16, 64, 4, ##__VA_ARGS__); break;  \
    case 5: NORM_LAUNCH(KERNEL, T, 16, 64, 8, ##__VA_ARGS__); break;  \
    default: NORM_LAUNCH(KERNEL, T, 16, 64, 16, ##__VA_ARGS__);       \
  }

template <typename T>
void launch_fwd(const NormArgs& a, dim3 grid, int shape, hipStream_t stream) {
  const bool ragged = a.d % Row<T>::kVec != 0;
  NORM_SHAPES(gated_norm_fwd_kernel, T);
}
template <typename T>
void launch_bwd(const NormArgs& a, dim3 grid, int shape, bool grouped, hipStream_t stream) {
  const bool ragged = a.d % Row<T>::kVec != 0;
  if (grouped) { NORM_SHAPES(gated_norm_bwd_kernel, T, true); }
  else { NORM_SHAPES(gated_norm_bwd_kernel, T, false); }
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
  NMT_REQUIRE(a->d_x, "%s: null pointer", who);
  NORM_ROWS(a->d_x, a->ld_x, "x");
  NORM_ROWS(a->d_y, a->ld_y, "y");
  NORM_ROWS(a->d_h, a->ld_h, "h");
  NORM_ROWS(a->d_n, a->ld_n, "n");
  const NormArgs k = common_args(a);
  const int shape = shape_of(a->d);
  const dim3 grid(std::min(ceil_div(a->rows, rows_at_a_time(shape)), kFwdGroups));
  if (a->type == NMT_F16) launch_fwd<half_t>(k, grid, shape, stream);
  else if (a->type == NMT_BF16) launch_fwd<bf16_t>(k, grid, shape, stream);
  else launch_fwd<float>(k, grid, shape, stream);
  NMT_LAUNCH_CHECK();
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
  const bool sums = g->d_dpost_gain || g->d_dpost_shift || g->d_dgate || g->d_dpre_gain || g->d_dpre_shift;
  if (a->rows == 0) {  // (sums over no rows)
    if (!sums) return NMT_OK;
    NormArgs k = {};
    k.d = a->d;
    k.dpost_gain = g->d_dpost_gain, k.dpost_shift = g->d_dpost_shift, k.dgate = g->d_dgate;
    k.dpre_gain = g->d_dpre_gain, k.dpre_shift = g->d_dpre_shift;
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
  const BwdPlan p = bwd_plan(a->rows, a->d);
  k.chunk = p.chunk, k.groups = p.groups, k.pitch = p.pitch;
  k.partial = g->d_scratch, k.gate_partial = g->d_scratch + (int64_t)p.groups * 4 * p.pitch;
  k.ld_dh = g->ld_dh, k.ld_dn = g->ld_dn, k.ld_dx = g->ld_dx, k.ld_dy = g->ld_dy;
  k.dh = g->d_dh, k.dn = g->d_dn, k.dx = g->d_dx, k.dy = g->d_dy;
  k.dpost_gain = g->d_dpost_gain, k.dpost_shift = g->d_dpost_shift, k.dgate = g->d_dgate;
  k.dpre_gain = g->d_dpre_gain, k.dpre_shift = g->d_dpre_shift;
  const int shape = shape_of(a->d);
  const dim3 grid(p.groups);
  if (a->type == NMT_F16) launch_bwd<half_t>(k, grid, shape, grouped, stream);
  else if (a->type == NMT_BF16) launch_bwd<bf16_t>(k, grid, shape, grouped, stream);
  else launch_bwd<float>(k, grid, shape, grouped, stream);
  NMT_LAUNCH_CHECK();
  return sums ? launch_sums(k, a->type, grouped, stream) : NMT_OK;
}
