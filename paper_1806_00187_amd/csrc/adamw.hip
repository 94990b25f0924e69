// AdamW over many tensors in one launch, states in 32 bits or in 8.  Bound by memory: master weights and states read and written,
// gradients read, weights written once.  A table in device memory holds one record for each piece of kPiece elements of
// every tensor, so that a work-group finds its pointers in one trip.
#include "common.h"

#include <cmath>
#include <new>
#include <vector>

namespace {

constexpr int kThreads = 256;
constexpr int kStateBlock = 256;           // elements that share a scale: a wavefront's, four a lane
constexpr int kPiece = 4 * kThreads;       // elements of a work-group's turn
constexpr int kMaxGroups = 65536;
constexpr float kTop = 448.f;              // the largest e4m3 value
constexpr float kTiny = 0x1p-100f;         // blocks of nothing larger are zero

struct Piece {
  float* master;
  void *m, *v;
  float *m_scale, *v_scale;
  const void* grad;
  void* weights;
  int32_t n;
  float decay, lr_factor;
  int32_t pad;
};
static_assert(sizeof(Piece) == 72, "");

struct Hyper {
  float lr, b1, c1, b2, c2, eps, inv_bc1, inv_bc2, grad_scale;  // c = 1 - b
};

template <typename T, int N>
struct Any {  // N elements at any address the type allows
  typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// One element.  Operations are spelled out: each rounds once, so that the states' 8-bit codes follow from the inputs and not from what the compiler contracts.
struct Moments { float m, v; };
__device__ __forceinline__ float adamw_element(Moments& s, float w, float g, const Hyper& h, float lr, float decay) {
#pragma clang fp contract(off)
  g = g * h.grad_scale;
  s.m = s.m * h.b1 + g * h.c1;
  s.v = s.v * h.b2 + (g * g) * h.c2;
  const float step = (s.m * h.inv_bc1) / (sqrtf(s.v * h.inv_bc2) + h.eps);
  return w - lr * (step + decay * w);
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// Four values of a lane to e4m3, the block's scale to *scale.  What is inf or NaN becomes NaN and does not count for the scale.
template <bool KEEP>
__device__ __forceinline__ uint32_t to_e4m3(const float (&x)[4], float* scale) {
#pragma clang fp contract(off)
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) top = fmaxf(top, finite(x[e]) ? fabsf(x[e]) : 0.f);
  top = wave_max(top);
  const float s = top * (1.f / kTop), inv = top > kTiny ? 1.f / s : 0.f;
  if ((threadIdx.x & 63) == 0) *scale = s;
  float q[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    q[e] = finite(x[e]) ? x[e] * inv : __uint_as_float(0x7FC00000u);
    if (KEEP && q[e] > 0.f) q[e] = fmaxf(q[e], 0x1p-9f);  // (the smallest that is not zero)
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
}
__device__ __forceinline__ void from_e4m3(uint32_t code, float scale, float (&x)[4]) {
  x[0] = __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * scale;
  x[1] = __builtin_amdgcn_cvt_f32_fp8((int)code, 1) * scale;
  x[2] = __builtin_amdgcn_cvt_f32_fp8((int)code, 2) * scale;
  x[3] = __builtin_amdgcn_cvt_f32_fp8((int)code, 3) * scale;
}

// Four elements from `p + i`; those behind the piece's end are 0.
template <typename T>
__device__ __forceinline__ void ld4(const void* p, int i, int n, float (&x)[4]) {
  const T* q = static_cast<const T*>(p) + i;
  if (i + 4 <= n) {
    const auto v = *reinterpret_cast<const typename Any<T, 4>::vec*>(q);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (float)v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = i + e < n ? (float)q[e] : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void st4(void* p, int i, int n, const float (&x)[4]) {
  T* q = static_cast<T*>(p) + i;
  if (i + 4 <= n) {
    typename Any<T, 4>::vec v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (T)x[e];
    *reinterpret_cast<typename Any<T, 4>::vec*>(q) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) q[e] = (T)x[e];
  }
}
__device__ __forceinline__ uint32_t ld_codes(const void* p, int i, int n) {
  const uint8_t* q = static_cast<const uint8_t*>(p) + i;
  if (i + 4 <= n) return __builtin_bit_cast(uint32_t, *reinterpret_cast<const Any<uint8_t, 4>::vec*>(q));
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) c |= i + e < n ? (uint32_t)q[e] << (8 * e) : 0u;
  return c;
}
__device__ __forceinline__ void st_codes(void* p, int i, int n, uint32_t c) {
  uint8_t* q = static_cast<uint8_t*>(p) + i;
  if (i + 4 <= n) {
    *reinterpret_cast<Any<uint8_t, 4>::vec*>(q) = __builtin_bit_cast(Any<uint8_t, 4>::vec, c);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) q[e] = (uint8_t)(c >> (8 * e));
  }
}

template <int BITS, typename G, typename W>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const Piece* __restrict__ table, int64_t pieces, const Hyper h, const int32_t* __restrict__ flag) {
  if (flag && *flag != 0) return;
  const int i = threadIdx.x * 4, block = threadIdx.x >> 6;
  for (int64_t at = blockIdx.x; at < pieces; at += gridDim.x) {
    const Piece p = table[at];
    const int n = p.n;
    if (block * kStateBlock >= n) continue;  // (whole wavefronts)
    float w[4], g[4], m[4], v[4];
    ld4<float>(p.master, i, n, w);
    ld4<G>(p.grad, i, n, g);
    if constexpr (BITS == 8) {
      from_e4m3(ld_codes(p.m, i, n), p.m_scale[block], m);
      from_e4m3(ld_codes(p.v, i, n), p.v_scale[block], v);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= v[e];
    } else {
      ld4<float>(p.m, i, n, m);
      ld4<float>(p.v, i, n, v);
    }
    const float lr = p.lr_factor * h.lr;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      Moments s = {m[e], v[e]};
      w[e] = adamw_element(s, w[e], g[e], h, lr, p.decay);
      m[e] = s.m;
      v[e] = s.v;
    }
    st4<float>(p.master, i, n, w);
    if (p.weights) st4<W>(p.weights, i, n, w);
    if constexpr (BITS == 8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = sqrtf(v[e]);
      st_codes(p.m, i, n, to_e4m3<false>(m, p.m_scale + block));
      st_codes(p.v, i, n, to_e4m3<true>(v, p.v_scale + block));
    } else {
      st4<float>(p.m, i, n, m);
      st4<float>(p.v, i, n, v);
    }
  }
}

template <int BITS, typename G>
void launch(const Piece* table, int64_t pieces, const Hyper& h, const int32_t* flag, int weights_type, hipStream_t stream) {
  const dim3 grid((uint32_t)(pieces < kMaxGroups ? pieces : kMaxGroups));
  if (weights_type == NMT_F16) hipLaunchKernelGGL((adamw_kernel<BITS, G, half_t>), grid, dim3(kThreads), 0, stream, table, pieces, h, flag);
  else if (weights_type == NMT_BF16) hipLaunchKernelGGL((adamw_kernel<BITS, G, __bf16>), grid, dim3(kThreads), 0, stream, table, pieces, h, flag);
  else hipLaunchKernelGGL((adamw_kernel<BITS, G, float>), grid, dim3(kThreads), 0, stream, table, pieces, h, flag);
}
template <int BITS>
void launch(const Piece* table, int64_t pieces, const Hyper& h, const int32_t* flag, int grad_type, int weights_type, hipStream_t stream) {
  if (grad_type == NMT_F16) launch<BITS, half_t>(table, pieces, h, flag, weights_type, stream);
  else if (grad_type == NMT_BF16) launch<BITS, __bf16>(table, pieces, h, flag, weights_type, stream);
  else launch<BITS, float>(table, pieces, h, flag, weights_type, stream);
}

int64_t pieces_of(int64_t n) { return (n + kPiece - 1) / kPiece; }
int count_pieces(const char* who, int32_t n, const nmt_adamw_tensor* tensors, int64_t* pieces) {
  NMT_REQUIRE(n >= 0 && (n == 0 || tensors), "%s: %d tensors", who, n);
  *pieces = 0;
  for (int32_t i = 0; i < n; ++i) {
    NMT_REQUIRE(tensors[i].n >= 0 && tensors[i].n <= (1ll << 40), "%s: tensor %d has %lld elements", who, i, (long long)tensors[i].n);
    *pieces += pieces_of(tensors[i].n);
  }
  return NMT_OK;
}
bool type_ok(int t) { return t == NMT_F16 || t == NMT_BF16 || t == NMT_F32; }
template <typename T>
bool aligned_as(const void* p, T size) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)size == 0; }

}  // namespace

struct nmt_adamw {
  const Piece* table;
  int64_t pieces;
  int state_bits, grad_type, weights_type;
};

extern "C" int64_t nmt_adamw_table_bytes(int32_t n, const nmt_adamw_tensor* tensors) {
  int64_t pieces = 0;
  if (const int rc = count_pieces("nmt_adamw_table_bytes", n, tensors, &pieces); rc != NMT_OK) return rc;
  return pieces * (int64_t)sizeof(Piece);
}

extern "C" int nmt_adamw_create(int32_t n, const nmt_adamw_tensor* tensors, int32_t state_bits, int32_t grad_type, int32_t weights_type,
                                void* d_table, int64_t table_bytes, void* stream_, nmt_adamw** out) {
  const char* who = "nmt_adamw_create";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  NMT_REQUIRE(out, "%s: null argument", who);
  *out = nullptr;
  NMT_REQUIRE(state_bits == 8 || state_bits == 32, "%s: states of %d bits: 8 or 32", who, state_bits);
  NMT_REQUIRE(type_ok(grad_type) && type_ok(weights_type), "%s: unknown type", who);
  int64_t pieces = 0;
  if (const int rc = count_pieces(who, n, tensors, &pieces); rc != NMT_OK) return rc;
  auto size = [](int t) { return t == NMT_F32 ? 4 : 2; };
  for (int32_t i = 0; i < n; ++i) {
    const nmt_adamw_tensor& t = tensors[i];
    NMT_REQUIRE(std::isfinite(t.weight_decay) && t.weight_decay >= 0.f && std::isfinite(t.lr_factor) && t.lr_factor >= 0.f,
                "%s: tensor %d: weight decay and learning-rate factor must be finite and not negative", who, i);
    if (t.n == 0) continue;
    NMT_REQUIRE(t.d_master && t.d_m && t.d_v && t.d_grad, "%s: tensor %d: null pointer", who, i);
    NMT_REQUIRE((state_bits == 8) == (t.d_m_scale != nullptr) && (state_bits == 8) == (t.d_v_scale != nullptr),
                "%s: tensor %d: scales belong to states of 8 bits", who, i);
    NMT_REQUIRE(aligned_as(t.d_master, 4) && aligned_as(t.d_grad, size(grad_type)) && aligned_as(t.d_weights, size(weights_type)) &&
                    (state_bits == 8 || (aligned_as(t.d_m, 4) && aligned_as(t.d_v, 4))) && aligned_as(t.d_m_scale, 4) && aligned_as(t.d_v_scale, 4),
                "%s: tensor %d: an address is no multiple of its element's size", who, i);
  }
  if (pieces * (int64_t)sizeof(Piece) > table_bytes || (pieces && !d_table)) {
    nmt_set_error("%s: a table of %lld bytes, %lld needed", who, (long long)(d_table ? table_bytes : 0), (long long)(pieces * (int64_t)sizeof(Piece)));
    return NMT_ENOMEM;
  }
  NMT_REQUIRE(aligned16(d_table), "%s: the table must be 16-byte aligned", who);
  try {
    std::vector<Piece> host;
    host.reserve((size_t)pieces);
    for (int32_t i = 0; i < n; ++i) {
      const nmt_adamw_tensor& t = tensors[i];
      const int state = state_bits / 8, grad = size(grad_type), weights = size(weights_type);
      for (int64_t at = 0; at < t.n; at += kPiece) {
        auto plus = [](const void* p, int64_t bytes) { return p ? (char*)p + bytes : nullptr; };
        const int64_t block = at / kStateBlock * 4;
        host.push_back(Piece{t.d_master + at, plus(t.d_m, at * state), plus(t.d_v, at * state), (float*)plus(t.d_m_scale, block),
                             (float*)plus(t.d_v_scale, block), plus(t.d_grad, at * grad), plus(t.d_weights, at * weights),
                             (int32_t)(t.n - at < kPiece ? t.n - at : kPiece), t.weight_decay, t.lr_factor, 0});
      }
    }
    if (pieces) {
      hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
      NMT_HIP_CHECK(hipStreamIsCapturing(stream, &capturing));
      NMT_REQUIRE(capturing == hipStreamCaptureStatusNone, "%s: the stream is being captured", who);
      NMT_HIP_CHECK(hipMemcpyAsync(d_table, host.data(), host.size() * sizeof(Piece), hipMemcpyHostToDevice, stream));
      NMT_HIP_CHECK(hipStreamSynchronize(stream));
    }
    *out = new nmt_adamw{static_cast<const Piece*>(d_table), pieces, state_bits, grad_type, weights_type};
  } catch (const std::bad_alloc&) {
    nmt_set_error("%s: no host memory for a table of %lld pieces", who, (long long)pieces);
    return NMT_ENOMEM;
  }
  return NMT_OK;
}

extern "C" void nmt_adamw_destroy(nmt_adamw* plan) { delete plan; }

extern "C" int nmt_adamw_step(const nmt_adamw* plan, double lr, double beta1, double beta2, double eps, int32_t t, float grad_scale,
                              const int32_t* d_flag, void* stream_) {
  const char* who = "nmt_adamw_step";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  NMT_REQUIRE(plan, "%s: null argument", who);
  NMT_REQUIRE(std::isfinite(lr) && lr >= 0, "%s: the learning rate must be finite and not negative", who);
  NMT_REQUIRE(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1, "%s: beta outside [0, 1)", who);
  NMT_REQUIRE(std::isfinite(eps) && eps > 0 && t >= 1 && std::isfinite(grad_scale), "%s: bad eps, t or grad_scale", who);
  if (plan->pieces == 0) return NMT_OK;
  const Hyper h = {(float)lr, (float)beta1, (float)(1 - beta1), (float)beta2, (float)(1 - beta2), (float)eps,
                   (float)(1 / (1 - pow(beta1, (double)t))), (float)(1 / (1 - pow(beta2, (double)t))), grad_scale};
  if (plan->state_bits == 8) launch<8>(plan->table, plan->pieces, h, d_flag, plan->grad_type, plan->weights_type, stream);
  else launch<32>(plan->table, plan->pieces, h, d_flag, plan->grad_type, plan->weights_type, stream);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}
