// Rows into 8 bits: a matrix as it is, and the norm that leaves its result so.  Bound by memory: what is read is read once, whatever forms of it are written.
#include "block8.h"

#include <algorithm>
#include <cmath>

namespace {

constexpr int kMaxRows = 0x7FFFFFFF - 65536, kMaxCols = 16384;
constexpr int kThreads = 512;
constexpr int kGridX = 1 << 22;  // work-groups in a row of the grid: one has less than 2^32 threads

// ---- a matrix into 8 bits --------------------------------------------------------------------------
struct QuantArgs {
  const void* x;
  int64_t ld_x, ld_codes, ld_codes_t, ld_scales, ld_scales_t;
  int rows, d, square;
  uint8_t *codes, *codes_t;
  float *scales, *scales_t;
  int64_t tiles;
  Divisor col_tiles;
};

// A work-group takes 128 x 128 elements, a thread 4 rows of 8 columns of them: 16 lanes hold 128 of a row, which share a scale, and a column's 128 are spread over 32
// groups of lanes.  (8 rows to a thread: three work-groups of half as many wavefronts to a compute unit, 26001 x 1024 24 us instead of 22.)  Codes of columns turn round in LDS, 4 rows of one column to a word; words of a column are
// swapped about by fours, by the column, so that the 16 lanes of a row write to different banks and a column's 16 codes lie side by side.
// Measured: 52701 x 1024 bf16 as it lies 25.4 us, 6.4 TB/s, its transpose 28, 5.8; 26001 x 1024 fp16 both 21.9, 4.9; 26001 x 4096 91; 4096 x 1024 fp32, squares, both 6.0.  Columns wait for all rows of a tile and twice for LDS.
// COLS: all 128 columns are there.
template <typename T, bool COLS>
__device__ __forceinline__ void quantize_tile(const QuantArgs& a, int64_t r0, int64_t c0, uint32_t (&turn)[128][32], uint32_t (&tops)[8][128], float (&backs)[128]) {
  const int lane16 = threadIdx.x & 15, group = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int64_t r = r0 + 4 * group, c = c0 + 8 * lane16;
  const int rows = (int)min((int64_t)a.rows - r, (int64_t)4), cols = (int)max(min((int64_t)a.d - c, (int64_t)8), (int64_t)0);  // of this thread's (rows may be negative)
  const T* x = static_cast<const T*>(a.x);
  // (kept as they came, and made numbers where they are used: 64 registers less for rows of 16 bits)
  Eight<T, !COLS> t[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i].load(x + min(r + i, (int64_t)a.rows - 1) * a.ld_x, (int)c, a.d);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    t[i].v = t[i].settled((int)c, a.d);
    if (i >= rows) t[i].v = typename Eight<T, !COLS>::vec{};
  }
  auto row_of = [&](int i, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)t[i].v[e];
  };
  auto column_of = [&](int e, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)t[i].v[e];
  };
  auto apart = [&] {  // (what was made of them is not kept)
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(t[i].v));
  };
  Scale8 whole = {0.f, 0.f};
  if (a.square) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[8];
      row_of(i, v);
      top = max(top, magnitude8(v));
    }
    apart();
    top = lanes16_max(top);
    if (lane16 == 0) tops[0][group] = top;
    __syncthreads();
    top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, tops[0][i]);
    whole = scale8(top);
    if (threadIdx.x == 0) {
      if (a.codes) a.scales[(c0 >> 7) * a.ld_scales + (r0 >> 7)] = whole.scale;
      if (a.codes_t) a.scales_t[(r0 >> 7) * a.ld_scales_t + (c0 >> 7)] = whole.scale;
    }
  }
  if (a.codes) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      Scale8 s = whole;
      float v[8];
      row_of(i, v);
      if (!a.square) {
        s = scale8(lanes16_max(magnitude8(v)));
        if (lane16 == 0 && i < rows) a.scales[(c0 >> 7) * a.ld_scales + r + i] = s.scale;
      }
      if (i < rows)
        store8<!COLS>(a.codes + (r + i) * a.ld_codes + c, codes8(v[0], v[1], v[2], v[3], s.back), codes8(v[4], v[5], v[6], v[7], s.back), cols);
    }
    apart();
  }
  if (a.codes_t) {
    if (!a.square) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v[4];
        column_of(e, v);
        uint32_t top = magnitude8(v);
        const auto rows16 = __builtin_amdgcn_permlane16_swap(top, top, false, false);
        top = max(rows16[0], rows16[1]);
        const auto halves = __builtin_amdgcn_permlane32_swap(top, top, false, false);
        top = max(halves[0], halves[1]);
        if ((threadIdx.x & 63) < 16) tops[wave][8 * lane16 + e] = top;
      }
      apart();
      __syncthreads();
      // a column's scale is formed once, by one thread
      const int col = threadIdx.x;
      if (col < kBlock8) {
        uint32_t top = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) top = max(top, tops[w][col]);
        const Scale8 s = scale8(top);
        if (c0 + col < a.d) a.scales_t[(r0 >> 7) * a.ld_scales_t + c0 + col] = s.scale;
        backs[col] = s.back;
      }
      __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v[4];
      column_of(e, v);
      turn[8 * lane16 + e][group ^ (lane16 & 7) << 2] = codes8(v[0], v[1], v[2], v[3], a.square ? whole.back : backs[8 * lane16 + e]);
    }
    __syncthreads();
    // a column's 128 codes lie with 8 lanes, 16 each
    const int at = threadIdx.x & 7;
    const int64_t row = r0 + 16 * at;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int col = (threadIdx.x >> 3) + 64 * i;
      const code4_t w = *reinterpret_cast<const code4_t*>(&turn[col][4 * (at ^ (col >> 3 & 7))]);
      if (c0 + col >= a.d) continue;
      uint8_t* to = a.codes_t + (c0 + col) * a.ld_codes_t + row;
      if (row + 16 <= a.rows) {
        *reinterpret_cast<code4_any*>(to) = (code4_any)w;
      } else {
        for (int e = 0; row + e < a.rows; ++e) to[e] = (uint8_t)((e < 8 ? e < 4 ? w[0] : w[1] : e < 12 ? w[2] : w[3]) >> 8 * (e & 3));
      }
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) quantize8_kernel(const QuantArgs a) {
  __shared__ __attribute__((aligned(16))) uint32_t turn[128][32];
  __shared__ uint32_t tops[8][128];
  __shared__ __attribute__((aligned(16))) float backs[128];
  const int64_t tile = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (tile >= a.tiles) return;
  uint32_t col;
  const uint32_t row = div_mod((uint32_t)tile, a.col_tiles, col);
  const int64_t r0 = (int64_t)row * kBlock8, c0 = (int64_t)col * kBlock8;
  if (c0 + kBlock8 <= a.d) quantize_tile<T, true>(a, r0, c0, turn, tops, backs);
  else quantize_tile<T, false>(a, r0, c0, turn, tops, backs);
}

// ---- the norm ----------------------------------------------------------------------------------------
struct Norm8Args {
  int rows, d, kind, chunk;  // chunk: rows of a worker, the lanes that hold a row
  float eps, resid_scale;
  int64_t ld_x, ld_y, ld_h, ld_n, ld_codes, ld_scales;
  const void *x, *y, *gain, *shift;
  void *h, *n;
  uint8_t* codes;
  float *scales, *stats;
};
typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));

// A row is read once into registers, and everything is formed there.  Measured: 52701 x 1024 bf16 with a sum 67 us, 5.6 TB/s; 13000 x 2048 fp16 30, 6.3; 6000 x 4096 fp32 55 to 59, 5.4 to 5.8; 2000 x 16384 bf16 39, 5.8; 20000 x 1001 fp16 25, 5.6; 1531 x
// 777 fp32 6.9; 5 x 512 fp16 2.2.
// LANES lanes of each of WAVES wavefronts hold a row, VECS times eight elements each: 16 lanes hold the 128 that share a scale.
template <typename T, int LANES, int VECS, int WAVES, bool RAGGED>
__global__ void __launch_bounds__(WAVES > 4 ? 64 * WAVES : 256) norm8_kernel(const Norm8Args a) {
  constexpr int THREADS = WAVES > 4 ? 64 * WAVES : 256, HOLD = LANES * WAVES, WORKERS = THREADS / HOLD;
  using V = Eight<T, RAGGED>;
  __shared__ float red[2][THREADS / 64];
  touch(a);
  const int d = a.d, lane = threadIdx.x % HOLD, worker = threadIdx.x / HOLD, first_wave = worker * WAVES;
  const float inv_d = 1.f / (float)d;
  const int64_t begin = min(((int64_t)blockIdx.x * WORKERS + worker) * a.chunk, (int64_t)a.rows), end = min(begin + a.chunk, (int64_t)a.rows);
  int at[VECS], there[VECS];  // the first column of every eight, and how many of them there are
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    at[i] = (lane + i * HOLD) * 8;
    there[i] = min(max(d - at[i], 0), 8);
  }
  // (columns past the row's end: its last are loaded, and count as zero)
  const int most = RAGGED ? 0x7FFFFFFF : d - 8;
  const T *x = static_cast<const T*>(a.x), *y = static_cast<const T*>(a.y);
  V gain[VECS], shift[VECS], next_x[VECS], next_y[VECS];
  auto ask = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < VECS; ++i) next_x[i].load(x + row * a.ld_x, min(at[i], most), d);
    if (a.y)
#pragma unroll
      for (int i = 0; i < VECS; ++i) next_y[i].load(y + row * a.ld_y, min(at[i], most), d);
  };
  auto sum = [&](float v, float* lds) {
    v = lanes_sum<LANES>(v);
    if constexpr (WAVES > 1) {
      if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
      __syncthreads();
      v = lds[first_wave];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) v += lds[first_wave + w];
    }
    return v;
  };
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    gain[i].load(static_cast<const T*>(a.gain), min(at[i], most), d);
    if (a.shift) shift[i].load(static_cast<const T*>(a.shift), min(at[i], most), d);
  }
  if (begin < end) ask(begin);
  // (rows that several wavefronts hold: every worker of a work-group goes round as often, for the barriers)
  for (int64_t row = begin, last = WAVES > 1 ? begin + a.chunk : end; row < last; ++row) {
    const bool mine = row < end;
    float h[VECS][8];
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      float t[8];
      next_x[i].get(h[i], at[i], d);
      if (a.y) {
        next_y[i].get(t, at[i], d);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] = a.resid_scale * h[i][e] + t[e];
      }
      if (!RAGGED && at[i] > most)
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] = 0.f;
    }
    V keep[VECS];
    if (a.h)
#pragma unroll
      for (int i = 0; i < VECS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) keep[i].v[e] = (T)h[i][e];
    if (row + 1 < end) ask(row + 1);
    float mean = 0.f, s = 0.f;
    if (a.kind == NMT_NORM_LAYER) {
#pragma unroll
      for (int i = 0; i < VECS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += h[i][e];
      mean = sum(s, red[0]) * inv_d;
      s = 0.f;
#pragma unroll
      for (int i = 0; i < VECS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] = (RAGGED ? e < there[i] : at[i] <= most) ? h[i][e] - mean : 0.f;
    }
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += h[i][e] * h[i][e];
    const float rstd = 1.f / sqrtf(sum(s, red[1]) * inv_d + a.eps);
    if (WAVES > 1 && a.kind != NMT_NORM_LAYER) __syncthreads();  // (red[1] is next)
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      float g[8], b[8];
      gain[i].get(g, at[i], d);
      if (a.shift) shift[i].get(b, at[i], d);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[i][e] = h[i][e] * rstd * g[e];
        if (a.shift) h[i][e] += b[e];
      }
      const Scale8 sc = scale8(lanes16_max(RAGGED || at[i] <= most ? magnitude8(h[i]) : 0u));
      if (!mine || there[i] == 0) continue;
      if ((lane & 15) == 0) a.scales[(int64_t)(at[i] >> 7) * a.ld_scales + row] = sc.scale;
      store8<RAGGED>(a.codes + row * a.ld_codes + at[i], codes8(h[i][0], h[i][1], h[i][2], h[i][3], sc.back), codes8(h[i][4], h[i][5], h[i][6], h[i][7], sc.back), there[i]);
      if (a.h) V::store(static_cast<T*>(a.h) + row * a.ld_h + at[i], keep[i].v, there[i]);
      if (a.n) {
        typename V::vec t;
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = (T)h[i][e];
        V::store(static_cast<T*>(a.n) + row * a.ld_n + at[i], t, there[i]);
      }
    }
    if (a.stats && mine && lane == 0) *reinterpret_cast<float4_any*>(a.stats + 4 * row) = float4_any{0.f, 1.f, mean, rstd};
  }
}

template <typename T, int LANES, int VECS, int WAVES>
int launch_norm8(Norm8Args a, hipStream_t stream) {
  constexpr int THREADS = WAVES > 4 ? 64 * WAVES : 256, WORKERS = THREADS / (LANES * WAVES);
  // A row each (52701 x 1024 bf16 66.7 us; seven rows to each of as many workers as there is room for 78.5), but few rows of the widest ones in turn (2000 x 16384 39.2 us, 44.6).
  const int64_t workers = (int64_t)device_info().cus * (VECS > 2 ? 16 : 256) / WAVES * (64 / LANES);
  a.chunk = (int)std::max<int64_t>(1, (a.rows + workers - 1) / workers);
  const int groups = ceil_div(ceil_div(a.rows, a.chunk), WORKERS);
  if (a.d % 8) hipLaunchKernelGGL((norm8_kernel<T, LANES, VECS, WAVES, true>), dim3(groups), dim3(THREADS), 0, stream, a);
  else hipLaunchKernelGGL((norm8_kernel<T, LANES, VECS, WAVES, false>), dim3(groups), dim3(THREADS), 0, stream, a);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}
template <typename T>
int launch_norm8_of(const Norm8Args& a, hipStream_t stream) {
  if (a.d <= 128) return launch_norm8<T, 16, 1, 1>(a, stream);
  if (a.d <= 256) return launch_norm8<T, 32, 1, 1>(a, stream);
  if (a.d <= 512) return launch_norm8<T, 64, 1, 1>(a, stream);
  if (a.d <= 1024) return launch_norm8<T, 64, 2, 1>(a, stream);
  if (a.d <= 2048) return launch_norm8<T, 64, 2, 2>(a, stream);
  if (a.d <= 4096) return launch_norm8<T, 64, 2, 4>(a, stream);
  if (a.d <= 8192) return launch_norm8<T, 64, 2, 8>(a, stream);
  return launch_norm8<T, 64, 4, 8>(a, stream);
}

}  // namespace

#define ROWS8_LD(ptr, n, ld, least, what) NMT_REQUIRE(!(ptr) || (n) <= 1 || (ld) >= (least), "%s: rows of " what " overlap", who)

extern "C" int nmt_op_quantize8(const void* d_x, int64_t ld_x, int32_t rows, int32_t d, int32_t type, int32_t square, void* d_codes, int64_t ld_codes,
                                float* d_scales, int64_t ld_scales, void* d_codes_t, int64_t ld_codes_t, float* d_scales_t, int64_t ld_scales_t,
                                void* stream_) {
  const char* who = "nmt_op_quantize8";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  NMT_REQUIRE(rows >= 0 && rows <= kMaxRows, "%s: %d rows", who, rows);
  NMT_REQUIRE(d >= 1 && d <= kMaxRows, "%s: d = %d", who, d);
  NMT_REQUIRE(row_type_ok(type), "%s: unknown type %d", who, type);
  const int64_t col_tiles = ceil_div(d, kBlock8), row_tiles = ceil_div(rows, kBlock8), tiles = col_tiles * row_tiles;
  NMT_REQUIRE(tiles < (1ll << 31), "%s: %d x %d elements are too many", who, rows, d);
  NMT_REQUIRE(!d_codes == !d_scales && !d_codes_t == !d_scales_t, "%s: codes and their scales belong together", who);
  if (rows == 0) return NMT_OK;
  NMT_REQUIRE(d_codes || d_codes_t, "%s: there is nothing to write", who);
  NMT_REQUIRE(d_x, "%s: null pointer", who);
  ROWS8_LD(d_x, rows, ld_x, d, "x");
  ROWS8_LD(d_codes, rows, ld_codes, d, "codes");
  ROWS8_LD(d_codes_t, d, ld_codes_t, rows, "codes_t");
  ROWS8_LD(d_scales, col_tiles, ld_scales, square ? row_tiles : rows, "scales");
  ROWS8_LD(d_scales_t, row_tiles, ld_scales_t, square ? col_tiles : d, "scales_t");
  QuantArgs a = {};
  a.x = d_x, a.ld_x = ld_x, a.rows = rows, a.d = d, a.square = square != 0;
  a.codes = static_cast<uint8_t*>(d_codes), a.ld_codes = ld_codes, a.scales = d_scales, a.ld_scales = ld_scales;
  a.codes_t = static_cast<uint8_t*>(d_codes_t), a.ld_codes_t = ld_codes_t, a.scales_t = d_scales_t, a.ld_scales_t = ld_scales_t;
  a.tiles = tiles, a.col_tiles = divisor((uint32_t)col_tiles);
  const dim3 grid((uint32_t)std::min<int64_t>(tiles, kGridX), (uint32_t)((tiles + kGridX - 1) / kGridX));
  if (type == NMT_F16) hipLaunchKernelGGL(quantize8_kernel<half_t>, grid, dim3(kThreads), 0, stream, a);
  else if (type == NMT_BF16) hipLaunchKernelGGL(quantize8_kernel<bf16_t>, grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(quantize8_kernel<float>, grid, dim3(kThreads), 0, stream, a);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}

extern "C" int nmt_op_norm8(const nmt_norm8* p, void* stream_) {
  const char* who = "nmt_op_norm8";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  NMT_REQUIRE(p, "%s: null argument", who);
  NMT_REQUIRE(p->rows >= 0 && p->rows <= kMaxRows, "%s: %d rows", who, p->rows);
  NMT_REQUIRE(p->d >= 1 && p->d <= kMaxCols, "%s: d = %d outside [1, %d]", who, p->d, kMaxCols);
  NMT_REQUIRE(row_type_ok(p->type), "%s: unknown type %d", who, p->type);
  NMT_REQUIRE(p->kind == NMT_NORM_LAYER || p->kind == NMT_NORM_RMS, "%s: unknown kind of norm %d", who, p->kind);
  NMT_REQUIRE(p->eps > 0.f && std::isfinite(p->eps), "%s: eps must be positive", who);
  NMT_REQUIRE(std::isfinite(p->resid_scale), "%s: resid_scale is not finite", who);
  NMT_REQUIRE(p->d_y || (!p->d_h && p->resid_scale == 1.f), "%s: without a block's output there is no sum to write, and nothing is scaled", who);
  if (p->rows == 0) return NMT_OK;
  NMT_REQUIRE(p->d_x && p->d_gain && p->d_codes && p->d_scales, "%s: null pointer", who);
  ROWS8_LD(p->d_x, p->rows, p->ld_x, p->d, "x");
  ROWS8_LD(p->d_y, p->rows, p->ld_y, p->d, "y");
  ROWS8_LD(p->d_h, p->rows, p->ld_h, p->d, "h");
  ROWS8_LD(p->d_n, p->rows, p->ld_n, p->d, "n");
  ROWS8_LD(p->d_codes, p->rows, p->ld_codes, p->d, "codes");
  ROWS8_LD(p->d_scales, ceil_div(p->d, kBlock8), p->ld_scales, p->rows, "scales");
  NMT_REQUIRE(p->rows <= 1 || ((!p->d_h || p->d_h != p->d_x || p->ld_h == p->ld_x) && (!p->d_n || p->d_n != p->d_y || p->ld_n == p->ld_y)),
              "%s: what is written in place has the distance of what was read", who);
  Norm8Args a = {};
  a.rows = p->rows, a.d = p->d, a.kind = p->kind, a.eps = p->eps, a.resid_scale = p->resid_scale;
  a.ld_x = p->ld_x, a.ld_y = p->ld_y, a.ld_h = p->ld_h, a.ld_n = p->ld_n, a.ld_codes = p->ld_codes, a.ld_scales = p->ld_scales;
  a.x = p->d_x, a.y = p->d_y, a.gain = p->d_gain, a.shift = p->d_shift, a.h = p->d_h, a.n = p->d_n;
  a.codes = static_cast<uint8_t*>(p->d_codes), a.scales = p->d_scales, a.stats = p->d_stats;
  if (p->type == NMT_F16) return launch_norm8_of<half_t>(a, stream);
  if (p->type == NMT_BF16) return launch_norm8_of<bf16_t>(a, stream);
  return launch_norm8_of<float>(a, stream);
}
