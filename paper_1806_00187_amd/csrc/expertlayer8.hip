// A sparse layer over few tokens, its experts' weights held in 8 bits with a scale for each 128 x 128:
//   hidden[t, j] = act(up[e(t, j)] x[t]),  out[t] = add[t] + sum over j of weights[t, j] down[e(t, j)] hidden[t, j].
// Bound by the weights of the experts that have a token, which are read once.  Two products of the same form and a sum: a work-group takes an expert's choices and 16 rows (or four
// times 16) of its weight; the matrix instruction's other operand are up to 16 choices' inputs.  Codes are exact in bf16; inputs are split into as
// many bf16 parts as hold them: bf16 one, fp16 two, fp32 three; so the products are those of the inputs as they are.
#include "block8.h"

#include <algorithm>

namespace {

constexpr int kMaxTokens = 64, kMaxChoices = 64, kMaxExperts = 1024, kMaxWidth = 1 << 20;
constexpr int kThreads = 256, kWaves = 4;
constexpr int kMost = 16;  // choices of a matrix instruction

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

struct LayerArgs {
  const void* x;         // [tokens, d] rows of the layer's type, or hidden [choices, width] in fp32
  const uint8_t* codes;  // of the experts' weights
  const float* scales;
  const int32_t* ids;
  float* out;            // [choices, rows of the result]
  int64_t ld_x, ld, stride, ld_scales, stride_scales;
  int n, k, experts, by_expert;  // choices; of a token; by_expert: a work-group's first index is an expert, not a choice
  int rows, width, act;          // rows: of the result; width: of x
};

template <int PARTS>
struct Input {  // eight elements of a row as bf16 parts that add up to them
  bf16x8_t part[PARTS];
};
template <typename T, int PARTS>
__device__ __forceinline__ void split8(const float (&x)[8], Input<PARTS>& in) {
#pragma clang fp contract(off)
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
  for (int p = 0; p < PARTS; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      in.part[p][e] = (__bf16)rest[e];
      rest[e] -= (float)in.part[p][e];
    }
}

// out[c] = W x for the choices c of an expert.  UP: c's row of x is its token's, GATED: rows r and rows + r of W together, silu(g) * u; ReLU otherwise.  Not UP: c's row is
// its own, nothing is done to the result.  KS: the wavefronts of a work-group share 16 rows, each a part of the width; else each has 16 of its own.
template <typename T, int PARTS, bool UP, bool GATED, bool KS>
__global__ void __launch_bounds__(kThreads) layer8_product_kernel(const LayerArgs a) {
  __shared__ int32_t list[kMaxTokens];
  __shared__ int32_t found;
  __shared__ float join[KS ? kWaves : 1][GATED ? 2 : 1][4][64];
  touch(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int index = blockIdx.y;
  const int expert = a.by_expert ? index : a.ids[index];
  if ((uint32_t)expert >= (uint32_t)a.experts) return;
  // the expert's choices, in their order; a token that chose it twice has one row
  if (wave == 0) {
    int count = 0;
    for (int c0 = 0; c0 < a.n; c0 += 64) {
      const int c = c0 + lane;
      bool hit = c < a.n && a.ids[min(c, a.n - 1)] == expert;
      for (int j = c - c % a.k; hit && j < c; ++j) hit = a.ids[j] != expert;
      const uint64_t hits = __ballot(hit);
      if (hit) list[count + __popcll(hits & ((1ull << lane) - 1))] = c;
      count += __popcll(hits);
    }
    if (lane == 0) found = count;
  }
  __syncthreads();
  const int count = found;
  if (count == 0 || (!a.by_expert && list[0] != index)) return;  // (the expert's first choice has its work-groups)
  const int row0 = (KS ? blockIdx.x : blockIdx.x * kWaves + wave) * 16;
  if (!KS && row0 >= a.rows) return;
  const int group = lane >> 4;
  const uint8_t* codes = a.codes + expert * a.stride;
  const float* scales = a.scales + expert * a.stride_scales;
  const int blocks = (a.width + kBlock8 - 1) / kBlock8;
  for (int c0 = 0; c0 < count; c0 += kMost) {
    const int col = c0 + (lane & 15), choice = list[min(col, count - 1)];
    const bool there = col < count;
    const T* x = static_cast<const T*>(a.x) + (UP ? choice / a.k : choice) * a.ld_x;
    floatx4 acc[GATED ? 2 : 1];
#pragma unroll
    for (int h = 0; h < (GATED ? 2 : 1); ++h) acc[h] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int b = KS ? wave : 0; b < blocks; b += KS ? kWaves : 1) {
      const int k0 = b * kBlock8;
      floatx4 t[GATED ? 2 : 1];
#pragma unroll
      for (int h = 0; h < (GATED ? 2 : 1); ++h) t[h] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int k = k0 + 64 * half + 16 * group;  // this lane's 16 columns
        // 16 of the inputs
        Input<PARTS> in[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int at = k + 8 * q + e;
            const float w = (float)x[min(at, a.width - 1)];
            v[e] = there && at < a.width ? w : 0.f;
          }
          split8<T, PARTS>(v, in[q]);
        }
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h) {
          const int row = min(row0 + (lane & 15), a.rows - 1) + h * a.rows;
          // (16 bytes with a code of the row in them, or the row's first; codes behind the row's end belong to nobody)
          code4_t w = *reinterpret_cast<const code4_t*>(codes + row * a.ld + (k < a.width ? k : 0));
          const int keep = a.width - k;
          if (keep < 16)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] &= keep >= 4 * i + 4 ? 0xFFFFFFFFu : keep <= 4 * i ? 0u : (1u << 8 * (keep - 4 * i)) - 1;
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            bf16x8_t m;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int word = (int)w[2 * q + i];
              m[4 * i + 0] = (__bf16)__builtin_amdgcn_cvt_f32_fp8(word, 0);
              m[4 * i + 1] = (__bf16)__builtin_amdgcn_cvt_f32_fp8(word, 1);
              m[4 * i + 2] = (__bf16)__builtin_amdgcn_cvt_f32_fp8(word, 2);
              m[4 * i + 3] = (__bf16)__builtin_amdgcn_cvt_f32_fp8(word, 3);
            }
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p) t[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(m, in[q].part[p], t[h], 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int h = 0; h < (GATED ? 2 : 1); ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = min(row0 + 4 * group + e, a.rows - 1) + h * a.rows;
          acc[h][e] = __builtin_fmaf(t[h][e], scales[b * a.ld_scales + (row >> 7)], acc[h][e]);
        }
    }
    if (KS) {
      __syncthreads();
#pragma unroll
      for (int h = 0; h < (GATED ? 2 : 1); ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) join[wave][h][e][lane] = acc[h][e];
      __syncthreads();
      if (wave == 0)
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[h][e] = (join[0][h][e][lane] + join[1][h][e][lane]) + (join[KS ? 2 : 0][h][e][lane] + join[KS ? 3 : 0][h][e][lane]);
    }
    if (there && (!KS || wave == 0))
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = row0 + 4 * group + e;
        float v = acc[0][e];
        if (UP) v = GATED ? v / (1.f + expf(-v)) * acc[GATED ? 1 : 0][e] : v < 0.f ? 0.f : v;
        if (row < a.rows) a.out[(int64_t)choice * a.rows + row] = v;
      }
  }
}

struct SumArgs {
  const float *y, *weights;
  const int32_t* ids;
  const void* add;
  void* out;
  int64_t ld_add, ld_out;
  int tokens, k, experts, d;
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
    v = __builtin_fmaf(a.weights ? a.weights[t * a.k + j] : 1.f, a.y[(int64_t)(t * a.k + first) * a.d + c], v);
  }
  static_cast<T*>(a.out)[t * a.ld_out + c] = (T)v;
}

template <typename T, int PARTS, bool UP, bool GATED>
int launch_product(LayerArgs a, hipStream_t stream) {
  const int tiles = ceil_div(a.rows, 16), experts = std::min(a.n, a.experts);
  a.by_expert = a.n > a.experts;
  if ((int64_t)tiles * experts < 8192) hipLaunchKernelGGL((layer8_product_kernel<T, PARTS, UP, GATED, true>), dim3(tiles, experts), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((layer8_product_kernel<T, PARTS, UP, GATED, false>), dim3(ceil_div(tiles, kWaves), experts), dim3(kThreads), 0, stream, a);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}
template <typename T, int PARTS, int HIDDEN_PARTS>
int launch_layer(const nmt_expert_layer8* p, hipStream_t stream) {
  const int n = p->tokens * p->k;
  float *hidden = p->d_scratch, *y = p->d_scratch + (int64_t)n * p->ff;
  LayerArgs a = {};
  a.ids = p->d_expert, a.n = n, a.k = p->k, a.experts = p->experts, a.act = p->act;
  a.x = p->d_x, a.ld_x = p->ld_x, a.codes = static_cast<const uint8_t*>(p->d_up), a.ld = p->ld_up, a.stride = p->stride_up;
  a.scales = p->d_up_scales, a.ld_scales = p->ld_up_scales, a.stride_scales = p->stride_up_scales, a.out = hidden, a.rows = p->ff, a.width = p->d;
  const int rc = p->act == NMT_ACT_SILU_GATE ? launch_product<T, PARTS, true, true>(a, stream) : launch_product<T, PARTS, true, false>(a, stream);
  if (rc != NMT_OK) return rc;
  a.x = hidden, a.ld_x = p->ff, a.codes = static_cast<const uint8_t*>(p->d_down), a.ld = p->ld_down, a.stride = p->stride_down;
  a.scales = p->d_down_scales, a.ld_scales = p->ld_down_scales, a.stride_scales = p->stride_down_scales, a.out = y, a.rows = p->d, a.width = p->ff;
  if (const int rc2 = launch_product<float, HIDDEN_PARTS, false, false>(a, stream); rc2 != NMT_OK) return rc2;
  SumArgs s = {};
  s.y = y, s.weights = p->d_weights, s.ids = p->d_expert, s.add = p->d_add, s.out = p->d_out, s.ld_add = p->ld_add, s.ld_out = p->ld_out;
  s.tokens = p->tokens, s.k = p->k, s.experts = p->experts, s.d = p->d;
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
  return (int64_t)tokens * k * ((int64_t)ff + d);
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
