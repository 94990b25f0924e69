// Products of matrices held in 8 bits with a scale for each block of 128:
//   C[m, n] = sum over the blocks of k of sa[block, m] sb[block, n] (sum over k in the block of A[m, k] B[n, k]) + bias[n] + add[m, n].
// A block of 128 is one matrix instruction (16 x 16 x 128) of codes as they are, whose sums are multiplied by the scales and added up in fp32.  That instruction
// adds up eight products at a time to 13 bits below the largest's power of two (measured; the sums of eight are added in fp32): 1.5e-5 of a result's size for
// normally distributed codes, which a rounding to 16 bits (2^-12, 2^-9) hides.  Results in fp32 are to be better than that: their codes go through the bf16
// instruction, at half the rate, which adds up in fp32 what are exact products.
#include "block8.h"

#include <algorithm>

namespace {

constexpr int kMaxSize = 0x7FFFFFFF - 65536;
constexpr int64_t kMaxLd = 1 << 27;      // bytes from row to row: eight rows within 32-bit offsets
constexpr int kMaxBatch = 1024;
constexpr uint32_t kOob = 0x80000000u;   // a byte offset that no operand reaches: such loads return 0
constexpr int BK = kBlock8;              // bytes of a row of a stage
constexpr int kGridX = 1 << 21;

typedef int frag_t __attribute__((ext_vector_type(8)));  // 32 codes of a lane
typedef __attribute__((address_space(3))) void* lds_void_ptr;

struct Gemm8Args {
  const uint8_t *a, *b;
  const float *sa, *sb;
  const void *bias, *add;
  void* c;
  float* partial;  // sums of the pieces of a product cut along k
  const int32_t* ranges;
  int64_t lda, ldb, ldc, ld_add, ld_sa, ld_sb, stride_a, stride_b, stride_c, stride_add, stride_bias, stride_sa, stride_sb;
  int M, N, K, batch, type, shift_a, shift_b;  // shift: 7 where 128 rows share a scale
  int k_chunk, splits, tiles_m, tiles_n;
  int64_t groups;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

// An operand's tile: R rows of 128 bytes in LDS, chunk p of 16 bytes of row r at p ^ (r >> 1 & 7), so that the 16 rows that a read touches lie on all banks.
// One wave instruction brings eight rows; its descriptor starts where it reads and ends with the rows, so what lies behind them arrives as zero.
template <int R, int NW>
struct Operand {
  static constexpr int BYTES = R * BK, NV = R / (8 * NW);  // wave instructions of a wavefront and stage
  static_assert(NV >= 1, "");
  const uint8_t* base;  // of the tile's first row, k = 0
  int64_t ld;
  int rows, K, wave;
  uint32_t voff, chunk;
  __device__ __forceinline__ void init(const uint8_t* first, int64_t ld_, int rows_, int K_) {
    base = first, ld = ld_, rows = rows_, K = K_;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, row = lane >> 3;
    chunk = ((lane & 7) ^ (((8 * wave + row) >> 1) & 7)) * 16;
    voff = (uint32_t)(row * ld) + chunk;
  }
  __device__ __forceinline__ void request(unsigned char* stage, int k, int it) const {
    const int r0 = 8 * (wave + NW * it), left = min(rows - r0, 8), k_left = K - k;
    // (to the end of the 16 bytes in which the last row's last code lies)
    const uint32_t bytes = left > 0 && k_left > 0 ? (uint32_t)((left - 1) * ld) + (uint32_t)((min(k_left, BK) + 15) & ~15) : 0u;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(base + r0 * ld + k, bytes), (lds_void_ptr)(stage + (wave + NW * it) * 1024), 16,
                                             (int)((int)chunk < k_left ? voff : kOob), 0, 0, 0);
  }
  __device__ __forceinline__ static frag_t fragment(const unsigned char* stage, int row0, int lane) {
    const int row = row0 + (lane & 15), s = (row >> 1) & 7, g = lane >> 4;
    const code4_t lo = *reinterpret_cast<const code4_t*>(stage + row * BK + ((g ^ s) << 4));
    const code4_t hi = *reinterpret_cast<const code4_t*>(stage + row * BK + (((g + 4) ^ s) << 4));
    return frag_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  }
  // The codes behind K of the 16 bytes in which K ends become zero: they belong to nobody.
  __device__ __forceinline__ static void clear_tail(unsigned char* stage, int k_left) {
    for (int row = threadIdx.x; row < R; row += 64 * NW) {
      code4_t* at = reinterpret_cast<code4_t*>(stage + row * BK + (((k_left >> 4) ^ ((row >> 1) & 7)) << 4));
      code4_t v = *at;
      const int keep = k_left & 15;
#pragma unroll
      for (int w = 0; w < 4; ++w) v[w] &= keep >= 4 * w + 4 ? 0xFFFFFFFFu : keep <= 4 * w ? 0u : (1u << 8 * (keep - 4 * w)) - 1;
      *at = v;
    }
  }
};

// Scales of R rows for one block of k, in LDS; 64 to a wave instruction.
template <int R>
__device__ __forceinline__ void request_scales(const float* s, int64_t ld, int shift, int row0, int rows, int block, bool there, float* lds, int part) {
  const int lane = threadIdx.x & 63, r = 64 * part + lane;
  const uint32_t at = (uint32_t)(((row0 + r) >> shift) - (row0 >> shift)) * 4u;
  __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(s + block * ld + (row0 >> shift), there ? 4u * R : 0u), (lds_void_ptr)(lds + 64 * part), 4,
                                           (int)(r < rows ? at : kOob), 0, 0, 0);
}

// Which tile a work-group takes.
struct Place {
  int batch, split, m0, n0, rows, first;  // rows of the tile; first row of the expert's range
};
__device__ __forceinline__ bool place(const Gemm8Args& g, int64_t id, int BM, int BN, Place& p) {
  // work-groups go round the eight dies; each gets a contiguous run of tiles
  const int64_t run = g.groups / 8, rest = g.groups % 8, die = id % 8;
  int64_t t = die * run + min(die, rest) + id / 8;
  p.n0 = (int)(t % g.tiles_n) * BN;
  t /= g.tiles_n;
  p.first = 0;
  if (!g.ranges) {
    p.m0 = (int)(t % g.tiles_m) * BM;
    t /= g.tiles_m;
    p.split = (int)(t % g.splits);
    p.batch = (int)(t / g.splits);
    p.rows = min(g.M - p.m0, BM);
    return true;
  }
  p.split = 0;
  const int lane = threadIdx.x & 63, per = (g.batch + 63) / 64;
  auto range = [&](int e, int& first, int& count) {
    first = max(0, min(g.ranges[2 * e], g.M));
    count = max(0, min(g.ranges[2 * e + 1], g.M - first));
  };
  int64_t mine = 0;
  int first, count;
  for (int i = 0; i < per; ++i) {
    const int e = lane * per + i;
    if (e < g.batch) {
      range(e, first, count);
      mine += (count + BM - 1) / BM;
    }
  }
  int64_t sum = mine;
  for (int step = 1; step < 64; step *= 2) {
    const int64_t up = __shfl_up(sum, step);
    sum += lane >= step ? up : 0;
  }
  const uint64_t behind = __ballot(sum > t);
  if (!behind) return false;
  const int at = __builtin_ctzll(behind);
  t -= __shfl(sum - mine, at);
  for (int e = at * per;; ++e) {
    range(e, first, count);
    const int tiles = (count + BM - 1) / BM;
    if (t < tiles) {
      p.batch = e;
      p.m0 = (int)t * BM;
      p.rows = min(count - p.m0, BM);
      p.first = first;
      return true;
    }
    t -= tiles;
  }
}

template <typename T>
__device__ __forceinline__ void store4(const Gemm8Args& g, T* c, const T* bias, const T* add, int64_t row, int n, floatx4 v) {
  typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  if (n + 4 <= g.N) {
    if (bias) {
      const vec b = *reinterpret_cast<const vec*>(bias + n);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += (float)b[e];
    }
    if (add) {
      const vec b = *reinterpret_cast<const vec*>(add + row * g.ld_add + n);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += (float)b[e];
    }
    vec out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (T)v[e];
    *reinterpret_cast<vec*>(c + row * g.ldc + n) = out;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < g.N) {
        float x = v[e];
        if (bias) x += (float)bias[n + e];
        if (add) x += (float)add[row * g.ld_add + n + e];
        c[row * g.ldc + n + e] = (T)x;
      }
  }
}

// Sixteen codes of one wavefront's rows as bf16, which holds them exactly.
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ bf16x8_t widen(int lo, int hi) {
  union {
    bf16x2_t two[4];
    bf16x8_t all;
  } u;
  u.two[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
  u.two[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
  u.two[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
  u.two[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
  return u.all;
}
template <bool EXACT>
struct Codes;
template <>
struct Codes<false> {  // as they are
  frag_t f;
  __device__ __forceinline__ void set(const frag_t& v) { f = v; }
  __device__ __forceinline__ floatx4 times(const Codes& o) const {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f, o.f, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
  }
};
template <>
struct Codes<true> {
  bf16x8_t f[4];
  __device__ __forceinline__ void set(const frag_t& v) {
#pragma unroll
    for (int q = 0; q < 4; ++q) f[q] = widen(v[2 * q], v[2 * q + 1]);
  }
  __device__ __forceinline__ floatx4 times(const Codes& o) const {
    floatx4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4; ++q) t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[q], o.f[q], t, 0, 0, 0);
    return t;
  }
};

// BM x BN of C by NW wavefronts, two of them along m.  Results lie transposed in the registers: lane L has row L & 15 of a 16 x 16 tile, columns 4 (L >> 4) to + 3.
template <int BM, int BN, int NW, bool EXACT>
__global__ void __launch_bounds__(64 * NW) gemm8_kernel(const Gemm8Args g) {
  constexpr int WM = BM / 2, WN = BN / (NW / 2), TM = WM / 16, TN = WN / 16;
  using OpA = Operand<BM, NW>;
  using OpB = Operand<BN, NW>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  constexpr int STAGE = OpA::BYTES + OpB::BYTES;
  auto stage = [&](int i) { return lds + i * STAGE; };
  auto scales = [&](int i) { return reinterpret_cast<float*>(lds + 2 * STAGE) + i * (BM + BN); };
  touch(g);
  const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  Place p;
  if (id >= g.groups || !place(g, id, BM, BN, p)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % 2 * WM, wn = wave / 2 * WN;
  const int k_begin = p.split * g.k_chunk, k_end = min(g.K, k_begin + g.k_chunk);
  const int cols = min(g.N - p.n0, BN);
  const int64_t row0 = (int64_t)p.first + p.m0;
  OpA a;
  OpB b;
  a.init(g.a + (g.ranges ? 0 : p.batch * g.stride_a) + row0 * g.lda, g.lda, p.rows, k_end);
  b.init(g.b + p.batch * g.stride_b + p.n0 * g.ldb, g.ldb, cols, k_end);
  const float *sa = g.sa + (g.ranges ? 0 : p.batch * g.stride_sa), *sb = g.sb + p.batch * g.stride_sb;
  auto request = [&](int s, int k) {
#pragma unroll
    for (int it = 0; it < OpA::NV; ++it) a.request(stage(s), k, it);
#pragma unroll
    for (int it = 0; it < OpB::NV; ++it) b.request(stage(s) + OpA::BYTES, k, it);
    for (int part = wave; part < (BM + BN) / 64; part += NW) {
      if (part < BM / 64) request_scales<BM>(sa, g.ld_sa, g.shift_a, (int)row0, p.rows, k / BK, k < k_end, scales(s), part);
      else request_scales<BN>(sb, g.ld_sb, g.shift_b, p.n0, cols, k / BK, k < k_end, scales(s) + BM, part - BM / 64);
    }
  };
  auto arrived = [&](int s, int k) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (k_end - k < BK && k_end - k > 0 && (k_end & 15)) {
      OpA::clear_tail(stage(s), k_end - k);
      OpB::clear_tail(stage(s) + OpA::BYTES, k_end - k);
      __syncthreads();
    }
  };
  floatx4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  request(0, k_begin);
  arrived(0, k_begin);
  int s = 0;
  for (int k = k_begin; k < k_end; k += BK, s ^= 1) {
    if (k + BK < k_end) request(s ^ 1, k + BK);
    Codes<EXACT> fb[TN];
    float4 sn[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      fb[j].set(OpB::fragment(stage(s) + OpA::BYTES, wn + 16 * j, lane));
      sn[j] = *reinterpret_cast<const float4*>(scales(s) + BM + wn + 16 * j + 4 * (lane >> 4));
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      Codes<EXACT> fa;
      fa.set(OpA::fragment(stage(s), wm + 16 * i, lane));
      const float sm = scales(s)[wm + 16 * i + (lane & 15)];
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const floatx4 t = fb[j].times(fa);
        acc[i][j][0] = __builtin_fmaf(t[0], sn[j].x * sm, acc[i][j][0]);
        acc[i][j][1] = __builtin_fmaf(t[1], sn[j].y * sm, acc[i][j][1]);
        acc[i][j][2] = __builtin_fmaf(t[2], sn[j].z * sm, acc[i][j][2]);
        acc[i][j][3] = __builtin_fmaf(t[3], sn[j].w * sm, acc[i][j][3]);
      }
    }
    arrived(s ^ 1, k + BK);
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = wm + 16 * i + (lane & 15);
    if (m >= p.rows) continue;
    const int64_t row = row0 + m;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int n = p.n0 + wn + 16 * j + 4 * (lane >> 4);
      if (n >= g.N) continue;
      if (g.partial) {
        float* to = g.partial + (((int64_t)p.batch * g.splits + p.split) * g.M + row) * g.N + n;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < g.N) to[e] = acc[i][j][e];
        continue;
      }
      auto out = [&](auto type) {
        using T = decltype(type);
        const int64_t own = g.ranges ? 0 : p.batch;
        store4<T>(g, static_cast<T*>(g.c) + own * g.stride_c, g.bias ? static_cast<const T*>(g.bias) + p.batch * g.stride_bias : nullptr,
                  g.add ? static_cast<const T*>(g.add) + own * g.stride_add : nullptr, row, n, acc[i][j]);
      };
      if (g.type == NMT_F16) out(half_t());
      else if (g.type == NMT_BF16) out(bf16_t());
      else out(float());
    }
  }
}

// The pieces' sums in increasing k, and what comes behind a product.
template <typename T>
__global__ void __launch_bounds__(256) gemm8_sums_kernel(const Gemm8Args g) {
  const int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x, per_row = (g.N + 3) / 4;
  const int64_t line = i / per_row;
  if (line >= (int64_t)g.batch * g.M) return;
  const int n = (int)(i % per_row) * 4;
  const int64_t batch = line / g.M, row = line % g.M;
  floatx4 v = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < g.splits; ++s) {
    const float* from = g.partial + ((batch * g.splits + s) * g.M + row) * g.N + n;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += from[min(e, g.N - 1 - n)];
  }
  store4<T>(g, static_cast<T*>(g.c) + batch * g.stride_c, g.bias ? static_cast<const T*>(g.bias) + batch * g.stride_bias : nullptr,
            g.add ? static_cast<const T*>(g.add) + batch * g.stride_add : nullptr, row, n, v);
}

struct Plan {
  int tile, splits;  // tile: 256, 128 or 64
};
Plan plan(int M, int N, int K, int batch, bool ranges) {
  auto tiles = [&](int t) { return ((int64_t)ceil_div(M, t) + (ranges ? batch : 0)) * ceil_div(N, t) * (ranges ? 1 : batch); };
  const int cus = 256;
  Plan p = {64, 1};
  if (tiles(256) >= cus) p.tile = 256;
  else if (tiles(128) >= cus) p.tile = 128;
  if (!ranges && tiles(p.tile) < cus) {
    const int blocks = ceil_div(K, BK);
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(blocks / 8, 2 * cus / std::max<int64_t>(1, tiles(p.tile))));
  }
  return p;
}

template <int BM, int BN, int NW, bool EXACT>
int launch_tiles(Gemm8Args g, hipStream_t stream) {
  g.tiles_m = ceil_div(g.M, BM), g.tiles_n = ceil_div(g.N, BN);
  g.groups = g.ranges ? ((int64_t)g.tiles_m + g.batch) * g.tiles_n : (int64_t)g.tiles_m * g.tiles_n * g.splits * g.batch;
  const dim3 grid((uint32_t)std::min<int64_t>(g.groups, kGridX), (uint32_t)((g.groups + kGridX - 1) / kGridX));
  constexpr size_t kLds = 2 * (BM + BN) * (BK + 4);
  if (kLds > (64 << 10))
    if (const int rc = allow_lds(reinterpret_cast<const void*>(gemm8_kernel<BM, BN, NW, EXACT>), kLds)) return rc;
  hipLaunchKernelGGL((gemm8_kernel<BM, BN, NW, EXACT>), grid, dim3(64 * NW), kLds, stream, g);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}

int check_sizes(const char* who, int M, int N, int K, int batch) {
  NMT_REQUIRE(M >= 0 && M <= kMaxSize && N >= 0 && N <= kMaxSize && K >= 0 && K <= kMaxSize, "%s: a product of %d x %d x %d", who, M, N, K);
  NMT_REQUIRE(batch >= 0 && batch <= kMaxBatch, "%s: %d products, at most %d", who, batch, kMaxBatch);
  NMT_REQUIRE(((int64_t)ceil_div(M, 64) + batch) * ceil_div(N, 64) <= (1ll << 40), "%s: a product of %d x %d is too large", who, M, N);
  return NMT_OK;
}

}  // namespace

extern "C" int64_t nmt_op_gemm8_scratch(int32_t M, int32_t N, int32_t K, int32_t batch, int32_t ranges) {
  if (const int rc = check_sizes("nmt_op_gemm8_scratch", M, N, K, batch); rc != NMT_OK) return rc;
  const Plan p = plan(M, N, K, batch, ranges != 0);
  return p.splits > 1 ? (int64_t)p.splits * batch * M * N : 0;
}

extern "C" int nmt_op_gemm8(const nmt_gemm8* p, void* stream_) {
  const char* who = "nmt_op_gemm8";
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  NMT_REQUIRE(p, "%s: null argument", who);
  if (const int rc = check_sizes(who, p->M, p->N, p->K, p->batch); rc != NMT_OK) return rc;
  NMT_REQUIRE(row_type_ok(p->type), "%s: unknown type %d", who, p->type);
  NMT_REQUIRE(!p->d_ranges || !p->a_square, "%s: experts' rows have a scale each", who);
  if (p->M == 0 || p->N == 0 || p->batch == 0) return NMT_OK;
  NMT_REQUIRE(p->d_c && (p->K == 0 || (p->d_a && p->d_b && p->d_sa && p->d_sb)), "%s: null pointer", who);
  const int blocks = ceil_div(p->K, BK), a_lines = p->a_square ? ceil_div(p->M, BK) : p->M, b_lines = p->b_square ? ceil_div(p->N, BK) : p->N;
  NMT_REQUIRE(p->K == 0 || (aligned16(p->d_a) && aligned16(p->d_b) && p->lda % 16 == 0 && p->ldb % 16 == 0 && (p->batch <= 1 || (p->stride_a % 16 == 0 && p->stride_b % 16 == 0))),
              "%s: rows of A and B begin at multiples of 16 bytes", who);
  NMT_REQUIRE(p->K == 0 || p->M <= 1 || (p->lda >= p->K && p->lda <= kMaxLd), "%s: lda = %lld", who, (long long)p->lda);
  NMT_REQUIRE(p->K == 0 || p->N <= 1 || (p->ldb >= p->K && p->ldb <= kMaxLd), "%s: ldb = %lld", who, (long long)p->ldb);
  NMT_REQUIRE(p->M <= 1 || p->ldc >= p->N, "%s: rows of C overlap", who);
  NMT_REQUIRE(!p->d_add || p->M <= 1 || p->ld_add >= p->N, "%s: rows of the addend overlap", who);
  NMT_REQUIRE(blocks <= 1 || (p->ld_sa >= a_lines && p->ld_sb >= b_lines), "%s: scales of a block of k overlap the next one's", who);
  NMT_REQUIRE(!p->d_add || p->d_add != p->d_c || (p->ld_add == p->ldc && p->stride_add == p->stride_c), "%s: an addend in place has C's distances", who);
  NMT_REQUIRE(p->stride_a >= 0 && p->stride_b >= 0 && p->stride_c >= 0 && p->stride_add >= 0 && p->stride_bias >= 0 && p->stride_sa >= 0 && p->stride_sb >= 0,
              "%s: a distance between products is negative", who);
  NMT_REQUIRE(p->d_ranges || p->batch <= 1 || p->stride_c > 0, "%s: products of a batch write the same C", who);
  NMT_REQUIRE(aligned16(p->d_scratch), "%s: the scratch buffer must be 16-byte aligned", who);
  const Plan how = plan(p->M, p->N, p->K, p->batch, p->d_ranges != nullptr);
  const int64_t need = how.splits > 1 ? (int64_t)how.splits * p->batch * p->M * p->N : 0;
  if (need > 0 && (!p->d_scratch || p->scratch_floats < need)) {
    nmt_set_error("%s: needs %lld floats of scratch", who, (long long)need);
    return NMT_ENOMEM;
  }
  Gemm8Args g = {};
  g.a = static_cast<const uint8_t*>(p->d_a), g.b = static_cast<const uint8_t*>(p->d_b), g.sa = p->d_sa, g.sb = p->d_sb;
  g.bias = p->d_bias, g.add = p->d_add, g.c = p->d_c, g.ranges = p->d_ranges;
  g.lda = p->lda, g.ldb = p->ldb, g.ldc = p->ldc, g.ld_add = p->ld_add, g.ld_sa = p->ld_sa, g.ld_sb = p->ld_sb;
  g.stride_a = p->stride_a, g.stride_b = p->stride_b, g.stride_c = p->stride_c, g.stride_add = p->stride_add, g.stride_bias = p->stride_bias;
  g.stride_sa = p->stride_sa, g.stride_sb = p->stride_sb;
  if (p->K == 0 || p->M == 1) g.lda = round_up(p->K, 16);  // (one row: no distance)
  if (p->K == 0 || p->N == 1) g.ldb = round_up(p->K, 16);
  g.M = p->M, g.N = p->N, g.K = p->K, g.batch = p->batch, g.type = p->type, g.shift_a = p->a_square ? 7 : 0, g.shift_b = p->b_square ? 7 : 0;
  g.splits = how.splits, g.k_chunk = ceil_div(ceil_div(p->K, BK), how.splits) * BK;
  g.partial = how.splits > 1 ? p->d_scratch : nullptr;
  int rc;
  if (g.type == NMT_F32) rc = how.tile >= 128 ? launch_tiles<128, 128, 4, true>(g, stream) : launch_tiles<64, 64, 4, true>(g, stream);
  else rc = how.tile == 256 ? launch_tiles<256, 256, 8, false>(g, stream) : how.tile == 128 ? launch_tiles<128, 128, 4, false>(g, stream) : launch_tiles<64, 64, 4, false>(g, stream);
  if (rc != NMT_OK || !g.partial) return rc;
  const int64_t groups = ((int64_t)g.batch * g.M * ((g.N + 3) / 4) + 255) / 256;
  const dim3 grid((uint32_t)std::min<int64_t>(groups, kGridX), (uint32_t)((groups + kGridX - 1) / kGridX));
  if (g.type == NMT_F16) hipLaunchKernelGGL(gemm8_sums_kernel<half_t>, grid, dim3(256), 0, stream, g);
  else if (g.type == NMT_BF16) hipLaunchKernelGGL(gemm8_sums_kernel<bf16_t>, grid, dim3(256), 0, stream, g);
  else hipLaunchKernelGGL(gemm8_sums_kernel<float>, grid, dim3(256), 0, stream, g);
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}
