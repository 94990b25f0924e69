// AdamW over many tensors in one launch, states in 32 bits or in 8.  Bound by memory: master weights and states read and written,
// gradients read, weights written once.  A table in device memory holds one record for each piece of kPiece elements of
// every tensor, so that a work-group finds its pointers in one trip.
// 61 million parameters, states in 32 bits, fp32 gradients: 299 us, 6.1 TB/s.  210 million, states in 8 bits, fp16 gradients: 593 us, 5.7 TB/s (a copy of a
// gigabyte: 5.2), one step after another; from an idle card the first three take 555 to 585, the next up to 900, and some fifty later they are back.  In turn with other forms: past the caches 303
// and 588 us, through them 355 and 657; one block of 256 elements a wavefront, two, four: 318, 303, 312 us.
#include "common.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

namespace {

constexpr int kThreads = 256;
constexpr int kStateBlock = 256;           // elements that share a scale: a wavefront's, four a lane
constexpr int kAhead = 2;                  // blocks that a wavefront has in flight
constexpr int kPiece = 4 * kThreads * kAhead;  // elements of a work-group, which takes one piece
constexpr int64_t kStreamFrom = 16 << 20;  // elements from which master weights and states of 32 bits exceed the last-level cache
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

}  // namespace

struct nmt_adamw {
  const Piece* table;
  int64_t pieces;
  int state_bits, grad_type, weights_type;
  bool stream;
};

namespace {

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

// Four elements from `p + i`; those behind the piece's end are 0.  FULL: there are none.
template <typename T, bool FULL, bool STREAM>
__device__ __forceinline__ void ld4(const void* p, int i, int n, float (&x)[4]) {
  const T* q = static_cast<const T*>(p) + i;
  if (FULL || i + 4 <= n) {
    const auto* a = reinterpret_cast<const typename Any<T, 4>::vec*>(q);
    const auto v = STREAM ? __builtin_nontemporal_load(a) : *a;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (float)v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = i + e < n ? (float)q[e] : 0.f;
  }
}
template <typename T, bool FULL, bool STREAM>
__device__ __forceinline__ void st4(void* p, int i, int n, const float (&x)[4]) {
  T* q = static_cast<T*>(p) + i;
  if (FULL || i + 4 <= n) {
    typename Any<T, 4>::vec v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (T)x[e];
    auto* a = reinterpret_cast<typename Any<T, 4>::vec*>(q);
    if (STREAM) __builtin_nontemporal_store(v, a);
    else *a = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) q[e] = (T)x[e];
  }
}
template <bool FULL, bool STREAM>
__device__ __forceinline__ uint32_t ld_codes(const void* p, int i, int n) {
  const uint8_t* q = static_cast<const uint8_t*>(p) + i;
  if (FULL || i + 4 <= n) {
    const auto* a = reinterpret_cast<const Any<uint8_t, 4>::vec*>(q);
    return __builtin_bit_cast(uint32_t, STREAM ? __builtin_nontemporal_load(a) : *a);
  }
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) c |= i + e < n ? (uint32_t)q[e] << (8 * e) : 0u;
  return c;
}
template <bool FULL, bool STREAM>
__device__ __forceinline__ void st_codes(void* p, int i, int n, uint32_t c) {
  uint8_t* q = static_cast<uint8_t*>(p) + i;
  if (FULL || i + 4 <= n) {
    auto* a = reinterpret_cast<Any<uint8_t, 4>::vec*>(q);
    const auto v = __builtin_bit_cast(Any<uint8_t, 4>::vec, c);
    if (STREAM) __builtin_nontemporal_store(v, a);
    else *a = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) q[e] = (uint8_t)(c >> (8 * e));
  }
}

// A work-group's piece.  A wavefront has kAhead blocks of 256 elements in flight, four elements a lane.
template <int BITS, bool FULL, bool STREAM, typename G, typename W>
__device__ __forceinline__ void adamw_piece(const Piece& p, const Hyper& h) {
  const int block0 = threadIdx.x >> 6, lane = threadIdx.x & 63, n = p.n;
  float w[kAhead][4], g[kAhead][4], m[kAhead][4], v[kAhead][4], ms[kAhead], vs[kAhead];
  uint32_t mc[kAhead], vc[kAhead];
  auto first = [&](int u) { return (block0 + u * (kThreads / 64)) * kStateBlock; };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int i = first(u) + 4 * lane;
    if (!FULL && first(u) >= n) break;  // (whole wavefronts)
    ld4<float, FULL, STREAM>(p.master, i, n, w[u]);
    ld4<G, FULL, STREAM>(p.grad, i, n, g[u]);
    if constexpr (BITS == 8) {
      mc[u] = ld_codes<FULL, STREAM>(p.m, i, n), vc[u] = ld_codes<FULL, STREAM>(p.v, i, n);
      ms[u] = p.m_scale[first(u) / kStateBlock], vs[u] = p.v_scale[first(u) / kStateBlock];
    } else {
      ld4<float, FULL, STREAM>(p.m, i, n, m[u]);
      ld4<float, FULL, STREAM>(p.v, i, n, v[u]);
    }
  }
  __builtin_amdgcn_sched_barrier(0);
  const float lr = p.lr_factor * h.lr;
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int i = first(u) + 4 * lane;
    if (!FULL && first(u) >= n) break;
    if constexpr (BITS == 8) {
      from_e4m3(mc[u], ms[u], m[u]);
      from_e4m3(vc[u], vs[u], v[u]);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[u][e] *= v[u][e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      Moments s = {m[u][e], v[u][e]};
      w[u][e] = adamw_element(s, w[u][e], g[u][e], h, lr, p.decay);
      m[u][e] = s.m;
      v[u][e] = s.v;
    }
    st4<float, FULL, STREAM>(p.master, i, n, w[u]);
    if (p.weights) st4<W, FULL, STREAM>(p.weights, i, n, w[u]);
    if constexpr (BITS == 8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[u][e] = sqrtf(v[u][e]);
      st_codes<FULL, STREAM>(p.m, i, n, to_e4m3<false>(m[u], p.m_scale + first(u) / kStateBlock));
      st_codes<FULL, STREAM>(p.v, i, n, to_e4m3<true>(v[u], p.v_scale + first(u) / kStateBlock));
    } else {
      st4<float, FULL, STREAM>(p.m, i, n, m[u]);
      st4<float, FULL, STREAM>(p.v, i, n, v[u]);
    }
  }
}

// STREAM: past the caches, which could not hold the state until the next update.
template <int BITS, bool STREAM, typename G, typename W>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const Piece* __restrict__ table, const Hyper h, const int32_t* __restrict__ flag) {
  if (flag && *flag != 0) return;
  const Piece p = table[blockIdx.x];
  if (p.n == kPiece) adamw_piece<BITS, true, STREAM, G, W>(p, h);
  else adamw_piece<BITS, false, STREAM, G, W>(p, h);
}

template <int BITS, bool STREAM, typename G>
void launch(const nmt_adamw& a, const Hyper& h, const int32_t* flag, hipStream_t stream) {
  const dim3 grid((uint32_t)a.pieces);
  if (a.weights_type == NMT_F16) hipLaunchKernelGGL((adamw_kernel<BITS, STREAM, G, half_t>), grid, dim3(kThreads), 0, stream, a.table, h, flag);
  else if (a.weights_type == NMT_BF16) hipLaunchKernelGGL((adamw_kernel<BITS, STREAM, G, __bf16>), grid, dim3(kThreads), 0, stream, a.table, h, flag);
  else hipLaunchKernelGGL((adamw_kernel<BITS, STREAM, G, float>), grid, dim3(kThreads), 0, stream, a.table, h, flag);
}
template <int BITS, bool STREAM>
void launch(const nmt_adamw& a, const Hyper& h, const int32_t* flag, hipStream_t stream) {
  if (a.grad_type == NMT_F16) launch<BITS, STREAM, half_t>(a, h, flag, stream);
  else if (a.grad_type == NMT_BF16) launch<BITS, STREAM, __bf16>(a, h, flag, stream);
  else launch<BITS, STREAM, float>(a, h, flag, stream);
}

int64_t pieces_of(int64_t n) { return (n + kPiece - 1) / kPiece; }
int count_pieces(const char* who, int32_t n, const nmt_adamw_tensor* tensors, int64_t* pieces) {
  NMT_REQUIRE(n >= 0 && (n == 0 || tensors), "%s: %d tensors", who, n);
  *pieces = 0;
  for (int32_t i = 0; i < n; ++i) {
    NMT_REQUIRE(tensors[i].n >= 0 && tensors[i].n <= (1ll << 40), "%s: tensor %d has %lld elements", who, i, (long long)tensors[i].n);
    *pieces += pieces_of(tensors[i].n);
  }
  NMT_REQUIRE(*pieces < (1 << 24), "%s: more than 2^24 pieces of %d elements", who, kPiece);  // (a grid has less than 2^32 threads)
  return NMT_OK;
}
// What a step writes overlaps neither what else it writes nor what it reads.
struct Range {
  uintptr_t begin, end;
  bool written;
};
bool overlap(std::vector<Range>& ranges) {
  std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t end = 0, written_end = 0;
  for (const Range& r : ranges) {
    if (r.begin < (r.written ? end : written_end)) return true;
    end = std::max(end, r.end);
    if (r.written) written_end = std::max(written_end, r.end);
  }
  return false;
}
bool type_ok(int t) { return t == NMT_F16 || t == NMT_BF16 || t == NMT_F32; }
template <typename T>
bool aligned_as(const void* p, T size) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)size == 0; }

}  // namespace

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
  int64_t elements = 0;
  for (int32_t i = 0; i < n; ++i) {
    const nmt_adamw_tensor& t = tensors[i];
    NMT_REQUIRE(std::isfinite(t.weight_decay) && t.weight_decay >= 0.f && std::isfinite(t.lr_factor) && t.lr_factor >= 0.f,
                "%s: tensor %d: weight decay and learning-rate factor must be finite and not negative", who, i);
    if (t.n == 0) continue;
    elements += t.n;
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
    std::vector<Range> ranges;
    ranges.reserve(7 * (size_t)n + 1);
    auto add = [&](const void* p, int64_t bytes, bool written) {
      if (p && bytes) ranges.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes, written});
    };
    add(d_table, pieces * (int64_t)sizeof(Piece), true);  // (gradients, which others write, must not lie there either)
    for (int32_t i = 0; i < n; ++i) {
      const nmt_adamw_tensor& t = tensors[i];
      const int64_t scales = (t.n + kStateBlock - 1) / kStateBlock * 4;
      add(t.d_master, 4 * t.n, true), add(t.d_m, t.n * (state_bits / 8), true), add(t.d_v, t.n * (state_bits / 8), true);
      add(t.d_m_scale, scales, true), add(t.d_v_scale, scales, true);
      add(t.d_weights, t.n * size(weights_type), true), add(t.d_grad, t.n * size(grad_type), false);
    }
    NMT_REQUIRE(!overlap(ranges), "%s: the table or what a step writes overlaps another buffer of the list", who);
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
    *out = new nmt_adamw{static_cast<const Piece*>(d_table), pieces, state_bits, grad_type, weights_type, elements >= kStreamFrom};
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
  NMT_REQUIRE(std::isfinite((float)lr) && lr >= 0, "%s: the learning rate must be finite and not negative", who);
  NMT_REQUIRE(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1, "%s: beta outside [0, 1)", who);
  NMT_REQUIRE(std::isfinite((float)eps) && (float)eps > 0 && t >= 1 && std::isfinite(grad_scale), "%s: bad eps, t or grad_scale", who);
  if (plan->pieces == 0) return NMT_OK;
  const Hyper h = {(float)lr, (float)beta1, (float)(1 - beta1), (float)beta2, (float)(1 - beta2), (float)eps,
                   (float)(1 / (1 - pow(beta1, (double)t))), (float)(1 / (1 - pow(beta2, (double)t))), grad_scale};
  if (plan->state_bits == 8 && plan->stream) launch<8, true>(*plan, h, d_flag, stream);
  else if (plan->state_bits == 8) launch<8, false>(*plan, h, d_flag, stream);
  else if (plan->stream) launch<32, true>(*plan, h, d_flag, stream);
  else launch<32, false>(*plan, h, d_flag, stream);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}
