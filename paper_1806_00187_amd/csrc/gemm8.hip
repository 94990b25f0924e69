// Products of matrices held in 8 bits with a scale for each block of 128:
//   C[m, n] = sum over the blocks of k of sa[block, m] sb[block, n] (sum over k in the block of A[m, k] B[n, k]) + bias[n] + add[m, n].
// A block of 128 is one matrix instruction (16 x 16 x 128) of codes as they are, whose sums are multiplied by the scales and added up in fp32.  That instruction
// adds up eight products at a time to 13 bits below the largest's power of two (measured; the sums of eight are added in fp32): 1.5e-5 of a result's size for
// normally distributed codes, at most 2^-10 of the sum of the terms' magnitudes, beside which results are rounded to 16 bits (by up to 2^-11, 2^-8).  Results in fp32 are to be better than that: their codes go through the bf16
// instruction, at half the rate, which adds up in fp32 what are exact products.
//
// Bound by the matrix units and the card's power: 8192^3 with 16-bit results 466 to 480 us, 2300 TFLOP/s, the matrix units at work in 60 % of the cycles of a clock that falls to 1.8 GHz (the library's product of the
// same codes without scales of blocks 360 us); 52701 x 4096 x 1024 236 to 248 us; 52012 rows of 128 experts, 1024 x 1024, 88 to 103 us.  Short sizes wait for memory and LDS once per block of k: 3584 x 2048 x 512 10 us, 5 x 2048 x 512 5 us.
// fp32 results: 8192^3 1000 to 1060 us, 1040 to 1100 TFLOP/s (bf16 library product 790); 1024 x 4096 x 26001 230 us and the sums of its two pieces 13; with 16-bit results, B's rows with a scale each, 140 in all.  The widening itself is 55 us of the 1000; the same instructions with A's operand
// held constant take 750: most of the rest is what changing operands cost, in power.
#include "block8.h"

#include <algorithm>

namespace {

constexpr int kMaxSize = 0x7FFFFFFF - 65536;
constexpr int64_t kMaxLd = 1 << 22;      // bytes from row to row: a tile's rows within 31-bit offsets
constexpr int kMaxBatch = 1024;
constexpr uint32_t kOob = 0x80000000u;   // a byte offset that no operand reaches: such loads return 0
constexpr int BK = kBlock8;              // bytes of a row of a stage
constexpr int kGridX = 1 << 21;
constexpr int kPatch = 4;                // rows of tiles that are swept together, column by column

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
  int k_chunk, splits;
  uint32_t groups, run, rest, launched;  // tiles; a die's of them (rest: how many dies have one more); work-groups, which take one after the other
  int tiles_m;
  Divisor by_n, by_tiles, by_splits, by_patch, by_rows, by_last;  // columns of tiles; tiles; ...; tiles of kPatch rows; kPatch, and what is left of rows behind the last whole patch
};

__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(lds_void_ptr)p; }
// The kernel's arguments, fetched anew: kept from a tile to the next they would fill the scalar registers.
__device__ __forceinline__ Gemm8Args arguments() {
#ifdef __HIP_DEVICE_COMPILE__
  auto* p = (const __attribute__((address_space(4))) Gemm8Args*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *p;
#else
  return {};
#endif
}
// One wave instruction: lane L's SIZE bytes, `at` bytes from base on, land at lds + SIZE L; zeros where `at` is kOob.  Written as an instruction because the compiler holds every read of LDS up
// until all such requests have arrived; whoever reads what this brings waits for it (arrived()).  The waits are those that the compiler would put behind a vector instruction that has written one of the scalars.
// m0 is one of the registers that the compiler reserves and takes no word of a change of: nothing else in these kernels may use it, which is checked on the built library.
template <int SIZE>
__device__ __forceinline__ void request_to_lds(uint64_t base, uint32_t lds, uint32_t at) {
  typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));
  const rsrc_t s = {(uint32_t)base, (uint32_t)(base >> 32), kOob, 0x00020000u};  // (no address has more than 48 bits)
  if constexpr (SIZE == 16) asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(at), "s"(s), "s"(lds) : "memory");
  else asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(at), "s"(s), "s"(lds) : "memory");
}
__device__ __forceinline__ uint64_t scalar(const void* p) {
  auto one = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
  return (uint64_t)one((uint32_t)((uint64_t)p >> 32)) << 32 | one((uint32_t)(uint64_t)p);
}
// All of a wavefront's requests and reads of LDS have arrived, but for the last BUT accesses; with the barrier behind it, all wavefronts'.
template <int BUT = 0>
__device__ __forceinline__ void arrived() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(BUT) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// An operand's tile: R rows of 128 bytes in LDS, chunk p of 16 bytes of row r at p ^ (r >> 1 & 7), so that the 16 rows that a read touches lie on all banks.
// One wave instruction brings eight rows, from the block of k at hand on; rows that the tile does not have and 16 bytes without a code of their row arrive as zeros.
template <int R, int NW>
struct Operand {
  static constexpr int BYTES = R * BK, NV = R / (8 * NW);  // wave instructions of a wavefront and stage
  static_assert(NV >= 1, "");
  uint64_t at;  // the tile's first row at the block of k at hand
  uint32_t voff[NV];
  int chunk;
  __device__ __forceinline__ void init(const uint8_t* first, int64_t ld, int rows, int wave) {
    const int lane = threadIdx.x & 63, row = 8 * wave + (lane >> 3);
    chunk = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    at = scalar(first);
#pragma unroll
    for (int it = 0; it < NV; ++it) voff[it] = row + 8 * NW * it < rows ? (uint32_t)((row + 8 * NW * it) * ld) + (uint32_t)chunk : kOob;
  }
  // k_left: codes of a row from the block at hand on
  __device__ __forceinline__ void request(uint32_t stage, int k_left, int wave, int it) const {
    request_to_lds<16>(at, stage + (uint32_t)(wave + NW * it) * 1024u, chunk < k_left ? voff[it] : kOob);
  }
  __device__ __forceinline__ void next() { at += BK; }
  // Where a lane reads its part of the fragment of 16 rows; rows 16 on lie 16 * BK on.
  __device__ __forceinline__ static int fragment_at(int row0, int lane) {
    const int row = row0 + (lane & 15);
    return row * BK + (((lane >> 4) ^ ((row >> 1) & 7)) << 4);
  }
  __device__ __forceinline__ static frag_t fragment(const unsigned char* stage, int at, int i) {
    const code4_t lo = *reinterpret_cast<const code4_t*>(stage + at + i * 16 * BK);
    const code4_t hi = *reinterpret_cast<const code4_t*>(stage + (at ^ 64) + i * 16 * BK);
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

// The scales of both operands' rows for one block of k, in LDS, A's first; 64 to a wave instruction, of which a wavefront has one at most.
template <int BM, int BN, int NW>
struct Scales {
  static constexpr int PARTS = (BM + BN) / 64;
  static_assert(PARTS <= NW, "");
  uint64_t at;
  int64_t step;
  uint32_t voff;
  __device__ __forceinline__ void init(const float* sa, int64_t ld_sa, int shift_a, int64_t row_a, int rows_a, const float* sb, int64_t ld_sb, int shift_b,
                                       int row_b, int rows_b, int wave) {
    const bool of_a = wave < BM / 64;
    const int r = 64 * (of_a ? wave : wave - BM / 64) + (int)(threadIdx.x & 63), shift = of_a ? shift_a : shift_b;
    const int64_t row = of_a ? row_a : row_b;
    at = scalar((of_a ? sa : sb) + (row >> shift));
    step = (of_a ? ld_sa : ld_sb) * 4;
    voff = r < (of_a ? rows_a : rows_b) ? (uint32_t)(((row + r) >> shift) - (row >> shift)) * 4u : kOob;
  }
  __device__ __forceinline__ void request(uint32_t lds, int k_left, int wave) const {
    if (wave < PARTS) request_to_lds<4>(at, lds + 256u * wave, k_left > 0 ? voff : kOob);
  }
  __device__ __forceinline__ void next() { at += step; }
};

// Which tile a work-group takes.
struct Place {
  int batch, split, m0, n0, rows, first;  // rows of the tile; first row of the expert's range
};
__device__ __forceinline__ bool place(const Gemm8Args& g, uint32_t id, int BM, int BN, Place& p) {
  // work-groups go round the eight dies; each die gets a contiguous run of tiles
  const uint32_t die = id & 7, turn = id >> 3;
  p.first = 0;
  if (!g.ranges) {
    if (id >= g.groups) return false;
    // splits of a product apart, and its tiles in patches: what the compute units of a die work on at a time are a few rows and columns of tiles, whose operands its cache holds
    uint32_t t = die * g.run + min(die, g.rest) + turn, col, row, split;
    t = div_mod(t, g.by_tiles, row);
    p.batch = (int)div_mod(t, g.by_splits, split);
    p.split = (int)split;
    const int first = (int)div_mod(row, g.by_patch, col) * kPatch;
    p.n0 = (int)div_mod(col, first + kPatch <= g.tiles_m ? g.by_rows : g.by_last, row) * BN;
    p.m0 = (first + (int)row) * BM;
    p.rows = min(g.M - p.m0, BM);
    return true;
  }
  p.split = 0;
  const int lane = threadIdx.x & 63, per = (g.batch + 63) / 64;
  // (cut at both ends: what lies below row 0 is no part of the count; no sum leaves 32 bits)
  auto range = [&](int e, int& first, int& count) {
    const int from = g.ranges[2 * e], rows = g.ranges[2 * e + 1];
    first = max(0, min(from, g.M));
    count = max(0, min(max(rows, 0) + min(from, 0), g.M - first));
  };
  uint32_t mine = 0;
  int first, count;
  for (int i = 0; i < per; ++i) {
    const int e = lane * per + i;
    if (e < g.batch) {
      range(e, first, count);
      mine += (uint32_t)(count + BM - 1) / BM;
    }
  }
  uint32_t sum = mine;
#pragma unroll
  for (int step = 1; step < 64; step *= 2) {
    const uint32_t up = __shfl_up(sum, step);
    sum += lane >= step ? up : 0;
  }
  const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)sum, 63) * g.by_n.d;
  if (id >= all) return false;
  uint32_t col, t = div_mod(die * (all >> 3) + min(die, all & 7) + turn, g.by_n, col);
  p.n0 = (int)col * BN;
  const uint64_t behind = __ballot(sum > t);
  if (!behind) return false;
  const int at = __builtin_ctzll(behind);
  t -= (uint32_t)__builtin_amdgcn_readlane((int)(sum - mine), at);
  for (int e = at * per; e < g.batch; ++e) {
    range(e, first, count);
    const uint32_t tiles = (uint32_t)(count + BM - 1) / BM;
    if (t < tiles) {
      p.batch = e;
      p.m0 = (int)t * BM;
      p.rows = min(count - p.m0, BM);
      p.first = first;
      return true;
    }
    t -= tiles;
  }
  return false;
}
// The same for all lanes, which the compiler does not see.
__device__ __forceinline__ bool place_scalar(const Gemm8Args& g, uint32_t id, int BM, int BN, Place& p) {
  const int there = __builtin_amdgcn_readfirstlane(place(g, id, BM, BN, p));
  for (int* v : {&p.batch, &p.split, &p.m0, &p.n0, &p.rows, &p.first}) *v = __builtin_amdgcn_readfirstlane(*v);
  return there != 0;
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

// A fragment as bf16.
struct Codes {
  bf16x8_t f[4];
  __device__ __forceinline__ void set(const frag_t& v) {
#pragma unroll
    for (int q = 0; q < 4; ++q) f[q] = widen8((uint32_t)v[2 * q], (uint32_t)v[2 * q + 1]);
  }
};

// What a work-group needs of its product.
template <int BM, int BN, int NW>
struct Product {
  static constexpr int WM = BM / 2, WN = BN / (NW / 2), TM = WM / 16, TN = WN / 16, STAGE = (BM + BN) * BK, ROWS_OF_TILE = BM, COLS_OF_TILE = BN, WAVES = NW;
  using OpA = Operand<BM, NW>;
  using OpB = Operand<BN, NW>;
  OpA a;
  OpB b;
  Scales<BM, BN, NW> s;
  int wave, lane, wm, wn;
  int left, length;  // codes of a row from the block that is asked for next on, and in all
  __device__ __forceinline__ void start() {
    lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wm = wave % 2 * WM, wn = wave / 2 * WN;
  }
  // The requests go to this tile's operands.
  __device__ __forceinline__ void aim(const Gemm8Args& g, const Place& p) {
    const int k_begin = p.split * g.k_chunk, k_end = min(g.K, k_begin + g.k_chunk), block = k_begin / BK;
    const int64_t own = g.ranges ? 0 : p.batch, row0 = (int64_t)p.first + p.m0;
    const int cols = min(g.N - p.n0, BN);
    left = length = max(k_end - k_begin, 0);
    a.init(g.a + own * g.stride_a + row0 * g.lda + k_begin, g.lda, p.rows, wave);
    b.init(g.b + p.batch * g.stride_b + p.n0 * g.ldb + k_begin, g.ldb, cols, wave);
    s.init(g.sa + own * g.stride_sa + block * g.ld_sa, g.ld_sa, g.shift_a, row0, p.rows, g.sb + p.batch * g.stride_sb + block * g.ld_sb, g.ld_sb, g.shift_b, p.n0, cols, wave);
  }
  static constexpr int REQUESTS = OpA::NV + OpB::NV + 1;
  // The q-th of the requests of a block of k; behind the last, the next block's are at hand.  Behind the last block nothing is asked for.
  __device__ __forceinline__ void request(uint32_t stage, uint32_t scales, int q) {
    if (q < OpA::NV) a.request(stage, left, wave, q);
    else if (q < OpA::NV + OpB::NV) b.request(stage + OpA::BYTES, left, wave, q - OpA::NV);
    else s.request(scales, left, wave);
    if (q < REQUESTS - 1) return;
    a.next(), b.next(), s.next();
    left -= BK;
  }
  __device__ __forceinline__ void request_all(uint32_t stage, uint32_t scales) {
#pragma unroll
    for (int q = 0; q < REQUESTS; ++q) request(stage, scales, q);
  }
  // Behind the barrier that publishes a stage; codes: of a row from its block on.
  __device__ __forceinline__ static void tail(unsigned char* stage, int codes) {
    if (__builtin_expect(codes > 0 && codes < BK && (codes & 15), 0)) {
      OpA::clear_tail(stage, codes);
      OpB::clear_tail(stage + OpA::BYTES, codes);
      __syncthreads();
    }
  }
};

// Codes as they are.  Results lie transposed in the registers: lane L has row L & 15 of a 16 x 16 tile, columns 4 (L >> 4) to + 3.
//
// A wavefront has TM strips of 16 rows and TN columns of tiles.  B's fragments of a block of k stay in registers, A's pass through G of them.  The first strips are multiplied one after the
// other; then comes the barrier behind which the stage is free and the next one is there, and the last G strips are multiplied column by column, so that one of B's fragments after the other is done
// with and can be fetched for the next block long before it is needed.  What a matrix instruction leaves is multiplied by its scales and added up LAG instructions later, which is the
// vector units' work beside the matrix units'.  The requests for the block after next are spread over the last strips.
// BFINE: B's rows have a scale each; else the wavefront's columns share one.  (Tiles of 256 x 256 leave registers for a LAG of 2 then: 8192^3 540 us, with 3 770.)
template <int BM, int BN, int NW, bool BFINE>
struct Strips : Product<BM, BN, NW> {
  using P = Product<BM, BN, NW>;
  using typename P::OpA;
  using typename P::OpB;
  static constexpr int TM = P::TM, TN = P::TN, G = TM < 3 ? TM : 3, ROWS = TM - G, SLOTS = TM * TN, LAG = BFINE && TM == 8 ? 2 : 3, RING = 4;
  static constexpr bool PER_STRIP = !BFINE && TM % 4 == 0;  // (of the strips in work at a time no two are the same modulo 4)
  static_assert(SLOTS % RING == 0, "");
  static_assert(P::WN <= BK, "a wavefront's columns share a scale");
  float acc[TM][TN][4];  // (apart, so that each is added to where it is)
  floatx4 t[RING];
  frag_t fa[G], fb[TN];
  float sm[G], sn[BFINE ? 1 : 2];
  float4 sn4[BFINE ? TN : 1];
  floatx4 by4[BFINE ? RING : 1];
  float by[BFINE ? 1 : RING];    // of a slot, or (PER_STRIP) of a strip
  int at_a, at_b, at_sm, at_sn;

  static constexpr int strip_of(int g) {  // of the last strips the one in register g
    for (int i = ROWS; i < TM; ++i)
      if (i % G == g) return i;
    return 0;
  }
  static constexpr int slot_i(int q) { return q < ROWS * TN ? q / TN : strip_of((q - ROWS * TN) % G); }
  static constexpr int slot_j(int q) { return q < ROWS * TN ? q % TN : (q - ROWS * TN) / G; }

  __device__ __forceinline__ void begin() {
    at_a = OpA::fragment_at(this->wm, this->lane), at_b = OpA::BYTES + OpB::fragment_at(this->wn, this->lane);
    at_sm = this->wm + (this->lane & 15), at_sn = BM + this->wn + 4 * (this->lane >> 4);
    clear();
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.f;
#pragma unroll
    for (int r = 0; r < RING; ++r) {
      t[r] = floatx4{0.f, 0.f, 0.f, 0.f};
      if constexpr (BFINE) by4[r] = t[r];
      else by[r] = 0.f;
    }
  }
  __device__ __forceinline__ void fetch_a(const unsigned char* stage, const float* scales, int i) {
    fa[i % G] = OpA::fragment(stage, at_a, i);
    sm[i % G] = scales[at_sm + 16 * i];
  }
  __device__ __forceinline__ void fetch_b(const unsigned char* stage, const float* scales, int j) {
    fb[j] = OpB::fragment(stage, at_b, j);
    if constexpr (BFINE) sn4[j] = *reinterpret_cast<const float4*>(scales + at_sn + 16 * j);
  }
  __device__ __forceinline__ void first(const unsigned char* stage, const float* scales) {
#pragma unroll
    for (int j = 0; j < TN; ++j) fetch_b(stage, scales, j);
    if constexpr (!BFINE) sn[0] = scales[BM + this->wn];
#pragma unroll
    for (int i = 0; i < G; ++i) fetch_a(stage, scales, i);
  }
  __device__ __forceinline__ void add(int q) {  // the sums of slot q, of this block or (q < 0) the one before
    const int slot = (q + SLOTS) % SLOTS, r = (q + SLOTS) % RING;
    float(&c)[4] = acc[slot_i(slot)][slot_j(slot)];
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = __builtin_fmaf(t[r][e], BFINE ? by4[BFINE ? r : 0][e] : by[BFINE ? 0 : PER_STRIP ? slot_i(slot) % 4 : r], c[e]);
    asm volatile("" : "+v"(c[0]), "+v"(c[1]), "+v"(c[2]), "+v"(c[3]));  // (here and not behind a branch)
  }
  __device__ __forceinline__ void multiply(int q) {
    const int i = slot_i(q), j = slot_j(q), r = q % RING;
    t[r] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[j], fa[i % G], floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
    if constexpr (BFINE) by4[r] = floatx4{sn4[j].x * sm[i % G], sn4[j].y * sm[i % G], sn4[j].z * sm[i % G], sn4[j].w * sm[i % G]};
    else if (!PER_STRIP) by[r] = sm[i % G] * sn[0];
    add(q - LAG);
    if (PER_STRIP && j == 0) by[i % 4] = sm[i % G] * sn[0];
    __builtin_amdgcn_sched_barrier(0);
  }
  // One block of k from stage `from`; the next is in or on its way to `to`, where a row has `codes` from there on; the one after goes to `from`.  aim(): the requests go on to the next tile's operands, if
  // there is one.  The wavefront may have STORES stores behind those requests under way, which need not be waited for.
  template <int STORES, typename Aim>
  __device__ __forceinline__ void block(unsigned char* from, float* scales_from, unsigned char* to, float* scales_to, int codes, bool stores, Aim aim) {
    const uint32_t to_stage = lds_address(from), to_scales = lds_address(scales_from);
#pragma unroll
    for (int q = 0; q < ROWS * TN; ++q) {
      multiply(q);
      if (slot_j(q) == TN - 1) fetch_a(from, scales_from, slot_i(q) + G);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (STORES > 0 && stores) arrived<STORES>();
    else arrived();  // (the next stage's requests, this one's fragments)
    this->tail(to, codes);
    if (__builtin_expect(this->left <= 0, 0)) aim();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!BFINE) sn[1] = scales_to[BM + this->wn];
#pragma unroll
    for (int c = 0; c < G * TN; ++c) {
      const int q = ROWS * TN + c, j = slot_j(q);
      multiply(q);
      if (j == TN - 1) fetch_a(to, scales_to, c % G);
      if (c % G == G - 1) fetch_b(to, scales_to, j);
#pragma unroll
      for (int x = c * P::REQUESTS / (G * TN); x < (c + 1) * P::REQUESTS / (G * TN); ++x) this->request(to_stage, to_scales, x);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (!BFINE) sn[0] = sn[1];
  }
  // One tile after the other, from work-group to work-group of the grid: the requests of a tile's last blocks are the next one's first, which arrive while results are written.
  // finish(place): writes acc; returns whether that took STORES stores.
  template <int STORES, typename Finish>
  __device__ __forceinline__ void run(const Gemm8Args& g, uint32_t id, Place& at, unsigned char* stages, float* scales, Finish finish) {
    this->start();
    this->aim(g, at);
    begin();
    this->request_all(lds_address(stages), lds_address(scales));
    __builtin_amdgcn_sched_barrier(0);
    int codes = this->length;
    this->request_all(lds_address(stages + P::STAGE), lds_address(scales + BM + BN));
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(P::REQUESTS - 1) : "memory");  // (the first stage's; a wavefront may have no scales to bring)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    this->tail(stages, codes);
    first(stages, scales);
    Place next = at;
    bool more = false, stores = false;
    auto aim = [&] {
      if constexpr (STORES > 0) {
        const Gemm8Args g = arguments();
        if (id + g.launched >= g.groups) return;
        more = place_scalar(g, id + g.launched, BM, BN, next);
        if (!more) return;
        id += g.launched;
        this->aim(g, next);
      }
    };
    int s = 0;
    auto one = [&] {
      const int behind = codes > BK ? codes - BK : more ? this->length : 0;
      block<STORES>(stages + s * P::STAGE, scales + s * (BM + BN), stages + (s ^ 1) * P::STAGE, scales + (s ^ 1) * (BM + BN), behind, stores, aim);
      codes -= BK, s ^= 1;
    };
    auto rest = [&] {
#pragma unroll
      for (int q = -LAG; q < 0; ++q) add(q);
    };
    if constexpr (STORES == 0) {
      while (codes > 0) one();
      rest();
      finish(at);
    } else {
      for (;;) {  // (one loop: of one in another the compiler keeps two sets of sums)
        if (__builtin_expect(codes > 0, 1)) one();
        stores = false;
        if (__builtin_expect(codes > 0, 1)) continue;
        rest();
        stores = finish(at);
        if (!more) break;
        clear();
        first(stages + s * P::STAGE, scales + s * (BM + BN));  // (once more: registers do not hold them while results are written)
        at = next, more = false, codes = this->length;
      }
    }
    arrived();  // (requests past the end, of nothing, which write zeros)
  }
};

// Codes as bf16, for results in fp32.  B's fragments of a block of k are widened once, A's strip by strip; a strip's sums are multiplied by their scales while the next strip's are formed.
template <int BM, int BN, int NW, bool BFINE>
struct Wide : Product<BM, BN, NW> {
  using P = Product<BM, BN, NW>;
  using typename P::OpA;
  using typename P::OpB;
  static constexpr int TM = P::TM, TN = P::TN;
  float acc[TM][TN][4];
  int at_a, at_b, at_sm, at_sn;
  __device__ __forceinline__ void block(const unsigned char* stage, const float* scales) {
    Codes fb[TN];
    float4 sn[TN];
    floatx4 t[2][TN];
    frag_t raw = OpA::fragment(stage, at_a, 0);
    float sm[2];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      fb[j].set(OpB::fragment(stage, at_b, j));
      sn[j] = *reinterpret_cast<const float4*>(scales + at_sn + 16 * j);
    }
    auto add = [&](int i) {
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const floatx4& v = t[i % 2][j];
        acc[i][j][0] = __builtin_fmaf(v[0], sn[j].x * sm[i % 2], acc[i][j][0]);
        acc[i][j][1] = __builtin_fmaf(v[1], sn[j].y * sm[i % 2], acc[i][j][1]);
        acc[i][j][2] = __builtin_fmaf(v[2], sn[j].z * sm[i % 2], acc[i][j][2]);
        acc[i][j][3] = __builtin_fmaf(v[3], sn[j].w * sm[i % 2], acc[i][j][3]);
      }
    };
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      Codes fa;
      fa.set(raw);
      sm[i % 2] = scales[at_sm + 16 * i];
      if (i + 1 < TM) raw = OpA::fragment(stage, at_a, i + 1);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int j = 0; j < TN; ++j) t[i % 2][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j].f[q], fa.f[q], q ? t[i % 2][j] : floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
      if (i > 0) add(i - 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    add(TM - 1);
  }
  template <int, typename Finish>
  __device__ __forceinline__ void run(const Gemm8Args& g, uint32_t, Place& at, unsigned char* stages, float* scales, Finish finish) {
    this->start();
    this->aim(g, at);
    at_a = OpA::fragment_at(this->wm, this->lane), at_b = OpA::BYTES + OpB::fragment_at(this->wn, this->lane);
    at_sm = this->wm + (this->lane & 15), at_sn = BM + this->wn + 4 * (this->lane >> 4);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.f;
    this->request_all(lds_address(stages), lds_address(scales));
    arrived();
    this->tail(stages, this->length);
    int s = 0;
    for (int codes = this->length; codes > 0; codes -= BK, s ^= 1) {
      this->request_all(lds_address(stages + (s ^ 1) * P::STAGE), lds_address(scales + (s ^ 1) * (BM + BN)));
      __builtin_amdgcn_sched_barrier(0);
      block(stages + s * P::STAGE, scales + s * (BM + BN));
      arrived();
      this->tail(stages + (s ^ 1) * P::STAGE, codes - BK);
    }
    finish(at);
  }
};

// A wavefront's share of C: strips of 16 rows turn round in LDS, so that lanes write 16 bytes each and a row's lie side by side.
template <typename Loop, typename T>
struct Result {
  static constexpr int TM = Loop::TM, TN = Loop::TN, WN = Loop::WN, E = 16 / sizeof(T), LANES = WN / E, ROWS = 64 / LANES, N = 16 / ROWS, PITCH = WN + E;
  static constexpr int BYTES = 16 * PITCH * sizeof(T), STORES = TM * N;
  static_assert(N >= 1, "");
  typedef T vec __attribute__((ext_vector_type(E), aligned(sizeof(T))));
  typedef T lds_vec __attribute__((ext_vector_type(E)));
  typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  typedef T lds_four __attribute__((ext_vector_type(4)));
  // Of n columns those that are there, from `from` on.
  static __device__ __forceinline__ four ask(const T* from, int n) {
    four v = {};
    if (n >= 4) {
      v = *reinterpret_cast<const four*>(from);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < n) v[e] = from[e];
    }
    return v;
  }
  // ALL: all of the share is there.  ADD: something may be added to it.
  template <bool ALL, bool ADD>
  static __device__ __forceinline__ void strips(const Loop& l, int rows, int cols, T* c, int64_t ldc, const T* add, int64_t ld_add, T* turn) {
    // as results lie in registers ...
    const int m = l.lane & 15, n = 4 * (l.lane >> 4);
    four plus[TN], next[TN];
    auto ask_strip = [&](int i) {
#pragma unroll
      for (int j = 0; j < TN; ++j) next[j] = ask(add + (int64_t)(16 * i + m) * ld_add + n + 16 * j, 16 * i + m < rows ? cols - (n + 16 * j) : 0);
    };
    if (ADD && add) ask_strip(0);
    // ... and as they are written
    const int row = l.lane / LANES, col = l.lane % LANES * E;
    T* to = c + (int64_t)row * ldc + col;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      if (ADD && add) {
#pragma unroll
        for (int j = 0; j < TN; ++j) plus[j] = next[j];
        if (i + 1 < TM) ask_strip(i + 1);
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        lds_four o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (T)(ADD && add ? l.acc[i][j][e] + (float)plus[j][e] : l.acc[i][j][e]);
        *reinterpret_cast<lds_four*>(turn + m * PITCH + 16 * j + n) = o;
      }
      wave_sync();
#pragma unroll
      for (int x = 0; x < N; ++x) {
        const lds_vec o = *reinterpret_cast<const lds_vec*>(turn + (ROWS * x + row) * PITCH + col);
        if (ALL || (16 * i + ROWS * x + row < rows && col + E <= cols)) {
          __builtin_nontemporal_store((vec)o, reinterpret_cast<vec*>(to));
        } else if (16 * i + ROWS * x + row < rows) {
#pragma unroll
          for (int e = 0; e < E - 1; ++e)
            if (col + e < cols) to[e] = o[e];
        }
        to += ROWS * ldc;
      }
      wave_sync();
    }
  }
  // c, add: of the product; bias: of its columns.  Returns whether all of the share was there, and written with STORES stores.
  template <bool ADD = true>
  static __device__ __forceinline__ bool store(Loop& l, const Place& p, int all_cols, T* c, int64_t ldc, const T* bias, const T* add, int64_t ld_add, unsigned char* turn_) {
    T* turn = reinterpret_cast<T*>(turn_);
    const int n0 = p.n0 + l.wn, rows = p.rows - l.wm, cols = all_cols - n0;  // of the share
    const int64_t row0 = (int64_t)p.first + p.m0 + l.wm;
    if (bias) {
      const int n = 4 * (l.lane >> 4);
      four b[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) b[j] = ask(bias + n0 + n + 16 * j, cols - (n + 16 * j));
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) l.acc[i][j][e] += (float)b[j][e];
    }
    c += row0 * ldc + n0;
    if (rows >= 16 * TM && cols >= WN && (!ADD || !add)) {
      strips<true, false>(l, rows, cols, c, ldc, nullptr, 0, turn);
      return true;
    }
    strips<false, ADD>(l, rows, cols, c, ldc, add ? add + row0 * ld_add + n0 : nullptr, ld_add, turn);
    return false;
  }
};

// BM x BN of C by NW wavefronts, two of them along m.  WIDE: codes as bf16, C in fp32.  TURNS, a type and not void: C is of that type, nothing is added to it, and a work-group takes one tile after the
// other: the next one's first blocks arrive while results are written, which turn round in LDS of their own.
template <int BM, int BN, int NW, bool BFINE, bool WIDE, typename TURNS>
__global__ void __launch_bounds__(64 * NW, BM == 64 ? 4 : 2) gemm8_kernel(const Gemm8Args g) {
  using Loop = std::conditional_t<WIDE, Wide<BM, BN, NW, BFINE>, Strips<BM, BN, NW, BFINE>>;
  __shared__ __attribute__((aligned(1024))) unsigned char stages[2 * Loop::STAGE];
  __shared__ __attribute__((aligned(16))) float scales[2 * (BM + BN)];
  touch(g);
  const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x;
  Place p;
  if (!place_scalar(g, id, BM, BN, p)) return;
  Loop l;
  if constexpr (!std::is_same_v<TURNS, void>) {
    using R = Result<Loop, TURNS>;
    __shared__ __attribute__((aligned(16))) unsigned char turns[NW * R::BYTES];
    l.template run<R::STORES>(g, id, p, stages, scales, [&](const Place& at) {
      const Gemm8Args g = arguments();
      const int64_t own = g.ranges ? 0 : at.batch;
      return R::template store<false>(l, at, g.N, static_cast<TURNS*>(g.c) + own * g.stride_c, g.ldc, g.bias ? static_cast<const TURNS*>(g.bias) + at.batch * g.stride_bias : nullptr,
                                      nullptr, 0, turns + l.wave * R::BYTES);
    });
  } else {
    static_assert(NW * Result<Loop, float>::BYTES <= 2 * Loop::STAGE, "");
    l.template run<0>(g, id, p, stages, scales, [&](const Place& at) {
      const int64_t own = g.ranges ? 0 : at.batch;
      arrived();  // (the stages are free)
      auto out = [&](auto type, void* c, int64_t ldc, bool whole) {
        using T = decltype(type);
        using R = Result<Loop, T>;
        R::store(l, at, g.N, static_cast<T*>(c), ldc, whole && g.bias ? static_cast<const T*>(g.bias) + at.batch * g.stride_bias : nullptr,
                 whole && g.add ? static_cast<const T*>(g.add) + own * g.stride_add : nullptr, g.ld_add, stages + l.wave * R::BYTES);
      };
      if (g.partial) out(float(), g.partial + ((int64_t)at.batch * g.splits + at.split) * g.M * g.N, g.N, false);
      else if constexpr (WIDE) out(float(), static_cast<float*>(g.c) + own * g.stride_c, g.ldc, true);
      else if (g.type == NMT_F16) out(half_t(), static_cast<half_t*>(g.c) + own * g.stride_c, g.ldc, true);
      else out(bf16_t(), static_cast<bf16_t*>(g.c) + own * g.stride_c, g.ldc, true);
    });
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

// How a product is cut up: tiles of 256 x 256, 128 x 128 or 64 x 64, of which a compute unit holds one, two or four, and pieces along k.  What it takes is estimated from what was measured, microseconds: a
// block of k with that many tiles on a compute unit, what a tile takes besides, and the sums of pieces.  Of 65 products (5 to 52701 rows, 512 to 52701 k, fp32 and bf16 results, B's scales by squares and by
// rows) timed in all forms 52 take the fastest, eleven one that is up to 11 % slower, two (6000 x 2900 x 1000 bf16, 777 x 5000 x 1000 fp32) one that is 24 % slower.  What the forms are for,
// microseconds: 8192^3 in tiles of 256 and 128 480, 600 (B's rows with a scale each 540, 660); 3584 x 2048 x 512 of 256, 128 and 64 16, 10, 14; 300 x 1024 x 1024 20, 12, 8; 512 x 512 x 52701 whole and in 16 pieces,
// of 128, 367, 41.
struct Form {
  int tile, held;
  double block[4], besides;
};
constexpr Form kNarrow[] = {{256, 1, {1.6}, 5.0}, {128, 2, {0.9, 1.22}, 3.5}, {64, 4, {0.56, 0.66, 0.85, 1.1}, 2.5}};
// (B's rows with a scale each)
constexpr Form kFine[] = {{256, 1, {1.85}, 13.0}, {128, 2, {0.94, 1.27}, 3.5}, {64, 4, {0.6, 0.7, 0.9, 1.15}, 2.5}};
constexpr Form kWide[] = {{128, 2, {1.36, 2.1}, 3.5}, {64, 4, {0.65, 0.8, 1.1, 1.4}, 2.5}};
constexpr double kSums = 4.0, kSumsRate = 4e6;  // microseconds; bytes of pieces, written and read, in a microsecond
struct Plan {
  int tile, splits;
  double us;
};
Plan plan(int M, int N, int K, int batch, bool ranges, bool wide, bool b_square) {
  const int cus = device_info().cus, blocks = std::max(1, ceil_div(K, BK));
  Plan best = {64, 1, 1e30};
  auto look = [&](const Form& f, int splits) {
    if (splits > 1 && (ranges || blocks / splits < 2)) return;
    // (of experts' rows the last tile is half full)
    const double tiles = (ranges ? ceil_div(M, f.tile) + 0.5 * batch : (double)ceil_div(M, f.tile) * batch) * ceil_div(N, f.tile);
    const int64_t each = (int64_t)((tiles * splits + cus - 1) / cus), rest = each % f.held;
    auto set = [&](int n) { return n ? ceil_div(blocks, splits) * f.block[n - 1] + f.besides : 0.0; };
    double us = (double)(each / f.held) * set(f.held) + set((int)rest);
    if (splits > 1) us += kSums + 8.0 * splits * batch * M * N / kSumsRate;
    if (us < best.us) best = {f.tile, splits, us};
  };
  for (int splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
    if (wide)
      for (const Form& f : kWide) look(f, splits);
    else
      for (const Form& f : b_square ? kNarrow : kFine) look(f, splits);
  }
  return best;
}

template <int BM, int BN, int NW, bool WIDE>
int launch_tiles(Gemm8Args g, hipStream_t stream) {
  const int64_t tiles_m = ceil_div(g.M, BM), tiles_n = ceil_div(g.N, BN);
  const int64_t groups = g.ranges ? (tiles_m + g.batch) * tiles_n : tiles_m * tiles_n * g.splits * g.batch;
  g.groups = (uint32_t)groups, g.run = g.groups / 8, g.rest = g.groups % 8;
  g.tiles_m = (int)tiles_m, g.by_n = divisor((uint32_t)tiles_n), g.by_tiles = divisor((uint32_t)(tiles_m * tiles_n)), g.by_splits = divisor((uint32_t)g.splits);
  g.by_patch = divisor((uint32_t)(kPatch * tiles_n)), g.by_rows = divisor(kPatch), g.by_last = divisor((uint32_t)std::max<int64_t>(1, tiles_m % kPatch));
  // Tiles of 256 x 256: a work-group on each compute unit takes one after the other, where the requests of two blocks are of one tile or of two.
  const bool turns = BM == 256 && g.shift_b && g.splits == 1 && g.K > BK && !g.add;
  const int64_t launched = turns ? std::min<int64_t>(groups, device_info().cus / 8 * 8) : groups;
  g.launched = (uint32_t)launched;
  const dim3 grid((uint32_t)std::min<int64_t>(launched, kGridX), (uint32_t)((launched + kGridX - 1) / kGridX)), threads(64 * NW);
  if constexpr (BM == 256) {
    if (!g.shift_b) hipLaunchKernelGGL((gemm8_kernel<BM, BN, NW, true, false, void>), grid, threads, 0, stream, g);
    else if (turns && g.type == NMT_F16) hipLaunchKernelGGL((gemm8_kernel<BM, BN, NW, false, false, half_t>), grid, threads, 0, stream, g);
    else if (turns) hipLaunchKernelGGL((gemm8_kernel<BM, BN, NW, false, false, bf16_t>), grid, threads, 0, stream, g);
    else hipLaunchKernelGGL((gemm8_kernel<BM, BN, NW, false, false, void>), grid, threads, 0, stream, g);
  } else if (!WIDE && g.shift_b) {
    hipLaunchKernelGGL((gemm8_kernel<BM, BN, NW, false, WIDE, void>), grid, threads, 0, stream, g);
  } else {
    hipLaunchKernelGGL((gemm8_kernel<BM, BN, NW, true, WIDE, void>), grid, threads, 0, stream, g);
  }
  NMT_LAUNCH_CHECK();
  return NMT_OK;
}

int check_sizes(const char* who, int M, int N, int K, int batch) {
  NMT_REQUIRE(M >= 0 && M <= kMaxSize && N >= 0 && N <= kMaxSize && K >= 0 && K <= kMaxSize, "%s: a product of %d x %d x %d", who, M, N, K);
  NMT_REQUIRE(batch >= 0 && batch <= kMaxBatch, "%s: %d products, at most %d", who, batch, kMaxBatch);
  NMT_REQUIRE((double)(ceil_div(M, 64) + 1) * ceil_div(N, 64) * std::max(batch, 1) < 1e9, "%s: %d products of %d x %d are too large", who, batch, M, N);
  return NMT_OK;
}

}  // namespace

extern "C" int64_t nmt_op_gemm8_scratch(int32_t M, int32_t N, int32_t K, int32_t batch, int32_t ranges) {
  if (const int rc = check_sizes("nmt_op_gemm8_scratch", M, N, K, batch); rc != NMT_OK) return rc;
  int splits = 0;
  for (int kind = 0; kind < 3; ++kind) splits = std::max(splits, plan(M, N, K, batch, ranges != 0, kind == 0, kind == 1).splits);
  return splits > 1 ? (int64_t)splits * batch * M * N : 0;
}

extern "C" int nmt_debug_gemm8_form(int32_t M, int32_t N, int32_t K, int32_t batch, int32_t ranges, int32_t type, int32_t b_square, int32_t* tile, int32_t* splits) {
  const char* who = "nmt_debug_gemm8_form";
  if (const int rc = check_sizes(who, M, N, K, batch); rc != NMT_OK) return rc;
  NMT_REQUIRE(row_type_ok(type) && tile && splits, "%s: bad argument", who);
  const Plan p = plan(M, N, K, batch, ranges != 0, type == NMT_F32, b_square != 0);
  *tile = p.tile, *splits = p.splits;
  return NMT_OK;
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
  const Plan how = plan(p->M, p->N, p->K, p->batch, p->d_ranges != nullptr, p->type == NMT_F32, p->b_square != 0);
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
  if (g.type == NMT_F32) rc = how.tile == 128 ? launch_tiles<128, 128, 4, true>(g, stream) : launch_tiles<64, 64, 4, true>(g, stream);
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
