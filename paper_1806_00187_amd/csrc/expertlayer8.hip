// A sparse layer over few tokens, its experts' weights held in 8 bits with a scale for each 128 x 128:
//   hidden[t, j] = act(up[e(t, j)] x[t]),  out[t] = add[t] + sum over j of weights[t, j] down[e(t, j)] hidden[t, j].
// Bound by the weights of the experts that have a token, which are read once for each 32 choices of an expert (16, where a work-group has 16 rows).  Two products of the same form and a sum: a
// work-group takes an expert's choices and 16 rows (or eight times 16) of its weight; the matrix instruction's other operand are up to 16 choices' inputs.  Codes are exact in bf16; inputs are split into as
// many bf16 parts as hold them: bf16 one, fp16 two, fp32 three; so the products are those of the inputs as they are.  Hidden goes on in two parts, off by up to 2^-17 of itself beside results that are rounded by up
// to 2^-11 (fp16) or 2^-8 (bf16), or, for fp32, in three, which hold it: in three for all types the 33 tokens below take 158 us instead of 147, 64 tokens, 8 of 16 experts, 57 instead of 53.
// Measured: 33 tokens, 4 of 64 experts, 1024 x 4096 silu gate, bf16 147 to 153 us, 4.6 to 4.8 TB/s of weights; 64 tokens, 2 of 128, 640 x 1280 ReLU 42 us, 3.2 TB/s; 64 tokens, 8 of 16, 512 x 2048 ReLU fp16 54 us,
// 0.6 TB/s, where each work-group walks all choices for its own and reads weights once more for an expert's last ones; one token, 2 of 8, 512 x 2048 10.8 us in a graph, which is three launches
// that wait for each other (4.5, 5 and 2): each a chain of choices, addresses, weights and sums.  The sum in the second product's last work-group instead of a launch: 13 us in a graph, and 198 for the 33 tokens.
#include "block8.h"

#include <algorithm>

namespace {

constexpr int kMaxTokens = 64, kMaxChoices = 64, kMaxExperts = 1024, kMaxWidth = 1 << 20;
constexpr int kThreads = 512, kWaves = 8;
constexpr int kSets = 2;       // sets of 16 choices, a matrix instruction's, that are in work at a time (one: 33 tokens 170 us instead of 157)
// Codes go into the products 2^17 times smaller, and what is added up is as much larger: so the sum of a block's 128 products, each of up to 448 times an input, is finite where the inputs are.  The scale comes first: times
// 2^17 it would be infinite from 2^111 on, and a sum of zero times that no number.  (Inputs below 2^-80, and blocks that add less than 2^-109, may count with fewer bits.  A choice between both orders by the scale
// costs registers, and so a work-group: 33 tokens 148 -> 156 us.)
constexpr float kDown = 0x1p17f;
constexpr int kStretch = 256;  // of the width, in LDS at a time (512, which leaves room for half as many work-groups: 33 tokens 208 us instead of 158)

struct LayerArgs {
  const void* x;         // [tokens, d] rows of the layer's type, or hidden [parts, choices, width rounded up to 16] in bf16
  const uint8_t* codes;  // of the experts' weights
  const float* scales;
  const int32_t* ids;
  float* out;            // [choices, rows of the result] ...
  __bf16* hidden;        // ... or hidden, ld_hidden
  int64_t ld_hidden, ld_x, ld, stride, ld_scales, stride_scales;
  int n, experts, by_expert;  // choices; by_expert: a work-group's first index is an expert, not a choice
  int rows, width, piece;     // rows: of the result; width: of x; piece: blocks of it that a work-group of the second product takes
  Divisor by_k;               // choices of a token
};

template <int PARTS>
struct Input {  // eight elements of a row as bf16 parts that add up to them
  bf16x8_t part[PARTS];
};
// T: the type that the elements had.
template <typename T, int PARTS, int N>
__device__ __forceinline__ void split(const float (&x)[N], __bf16 (&part)[PARTS][N]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int e = 0; e < N; ++e) {
    float rest = x[e];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      float high = (float)(__bf16)rest;
      if (p + 1 < PARTS) {
        // (what is too large for bf16 keeps the rest of itself, an infinity or NaN has none)
        constexpr float kMax = 0x1.FEp127f;
        const bool number = fabsf(rest) < __builtin_inff();
        if (sizeof(T) == 4 && number) high = fminf(fmaxf(high, -kMax), kMax);
        part[p][e] = (__bf16)high;
        rest = number ? rest - high : 0.f;
      } else {
        part[p][e] = (__bf16)high;
      }
    }
  }
}

// Where a product's inputs come from.  Rows of T, which are split when they are loaded, RAGGED: of a width that is no multiple of 8; or parts that were split before.
template <typename T, int PARTS, bool RAGGED>
struct Rows {
  static constexpr bool SPLIT = false;
  static constexpr int kParts = PARTS;
  Eight<T, RAGGED> e;
  const T* row;
  __device__ __forceinline__ void set(const LayerArgs& a, int choice, bool up) {
    uint32_t j;
    row = static_cast<const T*>(a.x) + (int64_t)(up ? div_mod((uint32_t)choice, a.by_k, j) : (uint32_t)choice) * a.ld_x;
  }
  __device__ __forceinline__ void ask(const LayerArgs& a, int at) { e.load(row, min(at, RAGGED ? a.width - 1 : a.width - 8), a.width); }
  __device__ __forceinline__ Input<PARTS> get(const LayerArgs& a, int at) const {
    float v[8];
    __bf16 part[PARTS][8];
    e.get(v, min(at, a.width - 1), a.width);
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = at < a.width ? v[u] : 0.f;
    split<T, PARTS, 8>(v, part);
    Input<PARTS> in;
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
      for (int u = 0; u < 8; ++u) in.part[p][u] = part[p][u];
    return in;
  }
};
template <int PARTS>
struct Parts {
  static constexpr bool SPLIT = true;
  static constexpr int kParts = PARTS;
  Input<PARTS> in;
  const __bf16* row;
  __device__ __forceinline__ void set(const LayerArgs& a, int choice, bool) { row = static_cast<const __bf16*>(a.x) + (int64_t)choice * a.ld_x; }
  __device__ __forceinline__ void ask(const LayerArgs& a, int at) {
    const int64_t plane = (int64_t)a.n * a.ld_x;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) in.part[p] = *reinterpret_cast<const bf16x8_t*>(row + p * plane + min(at, (int)a.ld_x - 8));
  }
  __device__ __forceinline__ Input<PARTS> get(const LayerArgs& a, int at) const {
    Input<PARTS> x = in;
    if (at >= a.width)
#pragma unroll
      for (int p = 0; p < PARTS; ++p) x.part[p] = bf16x8_t{};
    return x;
  }
};

// The choices of an expert, in their order, in `list`; returns how many.  A token that chose it twice has one row, that of its first choice.
__device__ __forceinline__ int choices_of(const LayerArgs& a, int expert, int32_t* list, int32_t* found) {
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    int count = 0;
    for (int c0 = 0; c0 < a.n; c0 += 64) {
      const int c = c0 + lane;
      uint32_t j;
      div_mod((uint32_t)c, a.by_k, j);
      bool hit = a.ids[min(c, a.n - 1)] == expert && c < a.n;
      for (int back = (int)j; hit && back > 0; --back) hit = a.ids[c - back] != expert;
      const uint64_t hits = __ballot(hit);
      if (hit) list[count + __popcll(hits & ((1ull << lane) - 1))] = c;
      count += __popcll(hits);
    }
    if (lane == 0) *found = count;
  }
  __syncthreads();
  return *found;
}

// The matrix instruction's sums of 16 rows of W times 16 columns of inputs over the blocks of 128 that are at hand.
template <int PARTS, int HALVES>
struct Block {
  code4_t w[HALVES][2];  // a lane's codes: 16 from column 16 (L >> 4) of the block, and 64 further on
  float scale[HALVES][4];
  __device__ __forceinline__ void ask(const LayerArgs& a, const uint8_t* codes, const float* scales, int row0, int b) {
    const int lane = threadIdx.x & 63, group = lane >> 4;
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      const uint8_t* row = codes + (int64_t)(min(row0 + (lane & 15), a.rows - 1) + h * a.rows) * a.ld;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int k = b * kBlock8 + 64 * half + 16 * group;
        w[h][half] = *reinterpret_cast<const code4_t*>(row + (k < a.width ? k : 0));  // (16 bytes with a code of the row in them)
      }
      // 16 rows from a multiple of 16 on share a scale, other 16 may have two
      const float* at = scales + b * a.ld_scales;
      if (h * a.rows % 16 == 0) {
        const float s = at[(row0 + h * a.rows) >> 7];
#pragma unroll
        for (int e = 0; e < 4; ++e) scale[h][e] = s;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) scale[h][e] = at[(min(row0 + 4 * group + e, a.rows - 1) + h * a.rows) >> 7];
      }
    }
  }
  // Codes behind a row's end belong to nobody.
  __device__ __forceinline__ void cut(const LayerArgs& a, int b) {
    if ((b + 1) * kBlock8 <= a.width) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int keep = a.width - (b * kBlock8 + 64 * half + 16 * (int)((threadIdx.x & 63) >> 4));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t mask = keep >= 4 * i + 4 ? 0xFFFFFFFFu : keep <= 4 * i ? 0u : (1u << 8 * (keep - 4 * i)) - 1;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) w[h][half][i] &= mask;
      }
    }
  }
  // in(half, q, n): the inputs of eight codes from 64 half + 16 (L >> 4) + 8 q on, of the n-th 16 columns.
  template <int N, typename F>
  __device__ __forceinline__ void add(floatx4 (&acc)[N][HALVES], F in) const {
    floatx4 t[N][HALVES];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int h = 0; h < HALVES; ++h) t[n][h] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        bf16x8_t m[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) m[h] = widen8(w[h][half][2 * q], w[h][half][2 * q + 1], 1.f / kDown);
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const Input<PARTS> x = in(half, q, n);
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
            for (int h = 0; h < HALVES; ++h) t[n][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(m[h], x.part[p], t[n][h], 0, 0, 0);
        }
      }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][h][e] = __builtin_fmaf(t[n][h][e] * scale[h][e], kDown, acc[n][h][e]);
  }
};

// out[c] = W x for the choices c of an expert.  UP: c's row of x is its token's, and what comes of it is hidden, in HIDDEN bf16 parts for the next product, GATED: of rows r and
// rows + r of W together, silu(g) * u; ReLU otherwise.  Not UP: c's row is its own, and the result is left in fp32.
// ROWS: a wavefront of a work-group has 16 rows of its own, and inputs are split once for all of them, a stretch of kStretch at a time, in LDS.  Otherwise the work-group has 16 rows, each wavefront every
// kWaves-th block of them, and splits its own inputs: for layers that leave compute units idle.
template <typename Source, int HIDDEN, bool GATED, bool ROWS>
__global__ void __launch_bounds__(kThreads, ROWS ? 4 : 2) layer8_product_kernel(const LayerArgs a) {
  constexpr bool UP = HIDDEN > 0;
  constexpr int PARTS = Source::kParts, HALVES = GATED ? 2 : 1, PITCH = kStretch + 8, BLOCKS = kStretch / kBlock8;
  __shared__ int32_t list[kMaxTokens], found;
  __shared__ __attribute__((aligned(16))) __bf16 xs[ROWS ? PARTS : 1][ROWS ? 16 * kSets : 1][ROWS ? PITCH : 8];
  __shared__ float join[ROWS ? 1 : kWaves][HALVES][4][64];
  touch(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = lane >> 4;
  const int index = blockIdx.y;
  const int expert = a.by_expert ? index : __builtin_amdgcn_readfirstlane(a.ids[index]);
  if ((uint32_t)expert >= (uint32_t)a.experts) return;
  const int count = __builtin_amdgcn_readfirstlane(choices_of(a, expert, list, &found));
  if (count == 0 || (!a.by_expert && __builtin_amdgcn_readfirstlane(list[0]) != index)) return;  // (the expert's first choice has its work-groups)
  const int row0 = (ROWS ? blockIdx.x * kWaves + wave : blockIdx.x) * 16;
  const uint8_t* codes = a.codes + expert * a.stride;
  const float* scales = a.scales + expert * a.stride_scales;
  const int all = (a.width + kBlock8 - 1) / kBlock8, first = UP ? 0 : (int)blockIdx.z * a.piece, blocks = UP ? all : min(all, first + a.piece);
  // What comes of 16 columns, from the c0-th choice on.
  auto finish = [&](const floatx4 (&acc)[HALVES], int c0) {
    const int col = c0 + (lane & 15), row = row0 + 4 * group;
    if (col >= count) return;
    const int choice = list[col];
    if constexpr (UP) {
      float v[4];
      __bf16 part[HIDDEN][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float g = acc[0][e];
        v[e] = GATED ? g / (1.f + expf(-g)) * acc[HALVES - 1][e] : g < 0.f ? 0.f : g;
        if (row + e >= a.rows) v[e] = 0.f;  // (hidden rows are whole 16s)
      }
      split<float, HIDDEN, 4>(v, part);
#pragma unroll
      for (int p = 0; p < HIDDEN; ++p) {
        typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
        *reinterpret_cast<bf16x4_t*>(a.hidden + ((int64_t)p * a.n + choice) * a.ld_hidden + row) = bf16x4_t{part[p][0], part[p][1], part[p][2], part[p][3]};
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (row + e < a.rows) a.out[((int64_t)blockIdx.z * a.n + choice) * a.rows + row + e] = acc[0][e];
    }
  };
  if constexpr (ROWS) {
    for (int c0 = 0; c0 < count; c0 += 16 * kSets) {
      const int cols = min(count - c0, 16 * kSets);
      floatx4 acc[kSets][HALVES], (&acc_one)[1][HALVES] = reinterpret_cast<floatx4(&)[1][HALVES]>(acc);
#pragma unroll
      for (int n = 0; n < kSets; ++n)
#pragma unroll
        for (int h = 0; h < HALVES; ++h) acc[n][h] = floatx4{0.f, 0.f, 0.f, 0.f};
      for (int b0 = first; b0 < blocks; b0 += BLOCKS) {
        Block<PARTS, HALVES> w[BLOCKS];
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) w[i].ask(a, codes, scales, min(row0, a.rows - 1) & ~15, min(b0 + i, blocks - 1));
        __syncthreads();  // (the last stretch is done with)
        for (int i = threadIdx.x; i < cols * (kStretch / 8); i += kThreads) {
          const int c = i / (kStretch / 8), k = i % (kStretch / 8) * 8, at = b0 * kBlock8 + k;
          Source x;
          x.set(a, list[c0 + c], UP);
          x.ask(a, at);
          const Input<PARTS> in = x.get(a, at);
#pragma unroll
          for (int p = 0; p < PARTS; ++p) *reinterpret_cast<bf16x8_t*>(&xs[p][c][k]) = in.part[p];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
          if (b0 + i >= blocks) break;
          auto from = [&](int half, int q, int n) {
            Input<PARTS> in;  // (columns without a choice hold whatever was there: nothing of theirs is written)
#pragma unroll
            for (int p = 0; p < PARTS; ++p) in.part[p] = *reinterpret_cast<const bf16x8_t*>(&xs[p][16 * n + (lane & 15)][i * kBlock8 + 64 * half + 16 * group + 8 * q]);
            return in;
          };
          w[i].cut(a, b0 + i);
          if (cols > 16) w[i].add(acc, from);
          else w[i].add(acc_one, from);
        }
      }
      if (row0 < a.rows)
#pragma unroll
        for (int n = 0; n < kSets; ++n) finish(acc[n], c0 + 16 * n);
    }
  } else {
    for (int c0 = 0; c0 < count; c0 += 16) {
      const int choice = list[min(c0 + (lane & 15), count - 1)];
      floatx4 acc[1][HALVES];
#pragma unroll
      for (int h = 0; h < HALVES; ++h) acc[0][h] = floatx4{0.f, 0.f, 0.f, 0.f};
      for (int b = first + wave; b < blocks; b += kWaves) {
        const int at = b * kBlock8 + 16 * group;
        Block<PARTS, HALVES> w;
        w.ask(a, codes, scales, row0, b);
        Source x[2][2];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            x[half][q].set(a, choice, UP);
            x[half][q].ask(a, at + 64 * half + 8 * q);
          }
        w.cut(a, b);
        w.add(acc, [&](int half, int q, int) { return x[half][q].get(a, at + 64 * half + 8 * q); });
      }
      __syncthreads();  // (the last choices' sums are read)
#pragma unroll
      for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) join[wave][h][e][lane] = acc[0][h][e];
      __syncthreads();
      if (wave > 0) continue;
#pragma unroll
      for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = join[0][h][e][lane];
#pragma unroll
          for (int w = 1; w < kWaves; ++w) v += join[ROWS ? 0 : w][h][e][lane];
          acc[0][h][e] = v;
        }
      finish(acc[0], c0);
    }
  }
}

struct SumArgs {
  const float *y, *weights;
  const int32_t* ids;
  const void* add;
  void* out;
  int64_t ld_add, ld_out;
  int tokens, k, experts, d, pieces;
};
template <typename T>
__global__ void __launch_bounds__(kThreads) layer8_sum_kernel(const SumArgs a) {
  const int t = blockIdx.y, c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= a.d) return;
  float v = a.add ? (float)static_cast<const T*>(a.add)[t * a.ld_add + c] : 0.f;
  for (int j = 0; j < a.k; ++j) {
    const int e = a.ids[t * a.k + j];
    if ((uint32_t)e >= (uint32_t)a.experts) continue;
    int first = 0;  // (where a token chose an expert twice, the first choice has the row)
    while (a.ids[t * a.k + first] != e) ++first;
    const float* y = a.y + (int64_t)(t * a.k + first) * a.d + c;
    float sum = *y;
    for (int p = 1; p < a.pieces; ++p) sum += y[(int64_t)p * a.tokens * a.k * a.d];
    v = __builtin_fmaf(a.weights ? a.weights[t * a.k + j] : 1.f, sum, v);
  }
  static_cast<T*>(a.out)[t * a.ld_out + c] = (T)v;
}

// Whether a product's wavefronts have 16 rows each (ROWS).  They read a weight once for 32 choices, without them it is once for 16; but they must be enough: eight to a compute unit for the first product, four for
// the second, whose width can be cut.  With and without, microseconds of the layer: 33 tokens, 4 of 64 experts, 1024 x 4096 157, 236; 64 tokens, 8 of 16, 512 x 2048 (32 choices of an expert) 60, 70;
// 8 tokens, 2 of 64, 1024 x 4096 (1024 wavefronts for the second product) 32, 36; but one token, 4 of 16, 2048 x 4096 36, 28; 2 of 8, 512 x 2048 15, 11.
bool whole_rows(int rows, int n, int experts, bool up) {
  return (int64_t)ceil_div(rows, 16) * std::max(std::min(n, experts), n / 16) >= (int64_t)device_info().cus * kWaves / (up ? 1 : 2);
}
// Into how many pieces the second product's width is cut: a work-group waits for its weights stretch by stretch, so four to a compute unit are wanted (the 33 tokens: 158 us, 163 in one piece).
int pieces_of(int n, int experts, int d, int ff) {
  if (!whole_rows(d, n, experts, false)) return 1;
  const int64_t groups = (int64_t)ceil_div(ceil_div(d, 16), kWaves) * std::min(n, experts);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(4, ceil_div(ff, 2 * kStretch)), 4ll * device_info().cus / groups));
}
template <typename Source, int HIDDEN, bool GATED>
int launch_product(LayerArgs a, int pieces, hipStream_t stream) {
  const int tiles = ceil_div(a.rows, 16), experts = std::min(a.n, a.experts);
  a.by_expert = a.n > a.experts;
  a.piece = ceil_div(ceil_div(a.width, kStretch), pieces) * (kStretch / kBlock8);
  if (whole_rows(a.rows, a.n, a.experts, HIDDEN > 0)) hipLaunchKernelGGL((layer8_product_kernel<Source, HIDDEN, GATED, true>), dim3(ceil_div(tiles, kWaves), experts, pieces), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((layer8_product_kernel<Source, HIDDEN, GATED, false>), dim3(tiles, experts, pieces), dim3(kThreads), 0, stream, a);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}
// Floats of hidden, in three parts at most.
int64_t hidden_floats(int n, int ff) { return (int64_t)n * round_up(ff, 16) / 2 * 3; }

template <typename T, int PARTS, int HIDDEN>
int launch_layer(const nmt_expert_layer8* p, hipStream_t stream) {
  const int n = p->tokens * p->k;
  __bf16* hidden = reinterpret_cast<__bf16*>(p->d_scratch);
  float* y = p->d_scratch + hidden_floats(n, p->ff);
  LayerArgs a = {};
  a.ids = p->d_expert, a.n = n, a.by_k = divisor((uint32_t)p->k), a.experts = p->experts, a.hidden = hidden, a.ld_hidden = round_up(p->ff, 16);
  a.x = p->d_x, a.ld_x = p->ld_x, a.codes = static_cast<const uint8_t*>(p->d_up), a.ld = p->ld_up, a.stride = p->stride_up;
  a.scales = p->d_up_scales, a.ld_scales = p->ld_up_scales, a.stride_scales = p->stride_up_scales, a.rows = p->ff, a.width = p->d;
  const bool gate = p->act == NMT_ACT_SILU_GATE;
  int rc;
  if (p->d % 8) rc = gate ? launch_product<Rows<T, PARTS, true>, HIDDEN, true>(a, 1, stream) : launch_product<Rows<T, PARTS, true>, HIDDEN, false>(a, 1, stream);
  else rc = gate ? launch_product<Rows<T, PARTS, false>, HIDDEN, true>(a, 1, stream) : launch_product<Rows<T, PARTS, false>, HIDDEN, false>(a, 1, stream);
  if (rc != NMT_OK) return rc;
  a.x = hidden, a.ld_x = a.ld_hidden, a.codes = static_cast<const uint8_t*>(p->d_down), a.ld = p->ld_down, a.stride = p->stride_down;
  a.scales = p->d_down_scales, a.ld_scales = p->ld_down_scales, a.stride_scales = p->stride_down_scales, a.out = y, a.rows = p->d, a.width = p->ff;
  const int pieces = pieces_of(n, p->experts, p->d, p->ff);
  if (const int rc2 = launch_product<Parts<HIDDEN>, 0, false>(a, pieces, stream); rc2 != NMT_OK) return rc2;
  SumArgs s = {};
  s.y = y, s.weights = p->d_weights, s.ids = p->d_expert, s.add = p->d_add, s.out = p->d_out, s.ld_add = p->ld_add, s.ld_out = p->ld_out;
  s.tokens = p->tokens, s.k = p->k, s.experts = p->experts, s.d = p->d, s.pieces = pieces;
  hipLaunchKernelGGL(layer8_sum_kernel<T>, dim3(ceil_div(p->d, kThreads), p->tokens), dim3(kThreads), 0, stream, s);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}

int check_layer(const char* who, int tokens, int k, int experts, int d, int ff) {
  NMT_REQUIRE(tokens >= 0 && tokens <= kMaxTokens, "%s: %d tokens: at most %d, more go through the experts' products", who, tokens, kMaxTokens);
  NMT_REQUIRE(k >= 1 && k <= kMaxChoices, "%s: %d choices of a token outside [1, %d]", who, k, kMaxChoices);
  NMT_REQUIRE(experts >= 1 && experts <= kMaxExperts, "%s: %d experts outside [1, %d]", who, experts, kMaxExperts);
  NMT_REQUIRE(d >= 1 && d <= kMaxWidth && ff >= 1 && ff <= kMaxWidth, "%s: widths %d and %d outside [1, %d]", who, d, ff, kMaxWidth);
  return NMT_OK;
}

}  // namespace

extern "C" int64_t nmt_op_expert_layer8_scratch(int32_t tokens, int32_t k, int32_t experts, int32_t d, int32_t ff) {
  if (const int rc = check_layer("nmt_op_expert_layer8_scratch", tokens, k, experts, d, ff); rc != NMT_OK) return rc;
  return hidden_floats(tokens * k, ff) + (int64_t)tokens * k * d * (tokens ? pieces_of(tokens * k, experts, d, ff) : 1);
}

extern "C" int nmt_op_expert_layer8(const nmt_expert_layer8* p, void* stream_) {
  const char* who = "nmt_op_expert_layer8";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  NMT_REQUIRE(p, "%s: null argument", who);
  if (const int rc = check_layer(who, p->tokens, p->k, p->experts, p->d, p->ff); rc != NMT_OK) return rc;
  NMT_REQUIRE(row_type_ok(p->type), "%s: unknown type %d", who, p->type);
  NMT_REQUIRE(p->act == NMT_ACT_RELU || p->act == NMT_ACT_SILU_GATE, "%s: unknown activation %d", who, p->act);
  if (p->tokens == 0) return NMT_OK;
  NMT_REQUIRE(p->d_x && p->d_expert && p->d_up && p->d_up_scales && p->d_down && p->d_down_scales && p->d_out, "%s: null pointer", who);
  const int up_rows = p->act == NMT_ACT_SILU_GATE ? 2 * p->ff : p->ff;
  NMT_REQUIRE(p->tokens <= 1 || (p->ld_x >= p->d && p->ld_out >= p->d && (!p->d_add || p->ld_add >= p->d)), "%s: rows overlap", who);
  NMT_REQUIRE(!p->d_add || p->d_add != p->d_out || p->ld_add == p->ld_out, "%s: an addend in place has the result's distance", who);
  NMT_REQUIRE(aligned16(p->d_up) && aligned16(p->d_down) && p->ld_up % 16 == 0 && p->ld_down % 16 == 0 && p->stride_up % 16 == 0 && p->stride_down % 16 == 0,
              "%s: rows of the weights begin at multiples of 16 bytes", who);
  NMT_REQUIRE((up_rows <= 1 || p->ld_up >= p->d) && (p->d <= 1 || p->ld_down >= p->ff), "%s: rows of the weights overlap", who);
  NMT_REQUIRE(p->stride_up >= 0 && p->stride_down >= 0 && p->stride_up_scales >= 0 && p->stride_down_scales >= 0, "%s: a distance between experts is negative", who);
  NMT_REQUIRE((p->d <= kBlock8 || p->ld_up_scales >= ceil_div(up_rows, kBlock8)) && (p->ff <= kBlock8 || p->ld_down_scales >= ceil_div(p->d, kBlock8)),
              "%s: scales overlap", who);
  NMT_REQUIRE(aligned16(p->d_scratch), "%s: the scratch buffer must be 16-byte aligned", who);
  const int64_t need = nmt_op_expert_layer8_scratch(p->tokens, p->k, p->experts, p->d, p->ff);
  if (!p->d_scratch || p->scratch_floats < need) {
    nmt_set_error("%s: needs %lld floats of scratch", who, (long long)need);
    return NMT_ENOMEM;
  }
  if (p->type == NMT_F16) return launch_layer<half_t, 2, 2>(p, stream);
  if (p->type == NMT_BF16) return launch_layer<bf16_t, 1, 2>(p, stream);
  return launch_layer<float, 3, 3>(p, stream);
}
