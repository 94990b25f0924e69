// Matrices held in 8 bits: e4m3 codes (4 exponent and 3 mantissa bits, no infinity), a scale in fp32 for each block of 128, value = code * scale.
#pragma once

#include "rowtypes.h"

constexpr int kBlock8 = 128;          // elements that share a scale
constexpr float kTop8 = 448.f;        // the largest code
constexpr float kTiny8 = 0x1p-100f;   // blocks of nothing larger are zero

typedef uint8_t byte8_t __attribute__((ext_vector_type(8), aligned(1)));
typedef uint32_t code4_t __attribute__((ext_vector_type(4)));                       // 16 codes
typedef uint32_t code4_any __attribute__((ext_vector_type(4), aligned(1)));         // at any address
typedef uint32_t code2_any __attribute__((ext_vector_type(2), aligned(1)));         // 8 codes at any address

// An element's part in its block's largest magnitude, in an order that unsigned integers have: twice its bits without the sign, and one more in the exponent, which
// wraps round for what is inf or NaN: that is less than any number's.
__device__ __forceinline__ uint32_t magnitude8(float x) { return (__float_as_uint(x) << 1) + 0x01000000u; }
template <int N>
__device__ __forceinline__ uint32_t magnitude8(const float (&x)[N]) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) top = max(top, magnitude8(x[e]));
  return top;
}
// The magnitude itself; 0 if there are no numbers.
__device__ __forceinline__ float magnitude8_value(uint32_t top) { return top < 0x01000000u ? 0.f : __uint_as_float((top - 0x01000000u) >> 1); }
// Largest over groups of 16 lanes; every lane gets its group's.
__device__ __forceinline__ uint32_t lanes16_max(uint32_t v) {
  auto meet = [](uint32_t x, auto ctrl) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, true)); };
  v = meet(v, std::integral_constant<int, 0x128>{});  // row_ror:8
  v = meet(v, std::integral_constant<int, 0x124>{});  // row_ror:4
  v = meet(v, std::integral_constant<int, 0x4E>{});   // quad_perm:[2,3,0,1]
  return meet(v, std::integral_constant<int, 0xB1>{});  // quad_perm:[1,0,3,2]
}

// A block's scale, rounded once, and its reciprocal; nothing is left of a block that is next to nothing.
struct Scale8 { float scale, back; };
__device__ __forceinline__ Scale8 scale8(uint32_t magnitude) {
#pragma clang fp contract(off)
  const float top = magnitude8_value(magnitude);
  Scale8 s = {0.f, 0.f};
  if (top > kTiny8) {
    s.scale = top * (1.f / kTop8);
    const float near = __builtin_amdgcn_rcpf(s.scale);  // (no scale is subnormal: one step of Newton's makes it the nearest but for a last bit now and then)
    s.back = __builtin_fmaf(__builtin_fmaf(-s.scale, near, 1.f), near, near);
  }
  return s;
}
// Four codes, nearest, ties to even.  |x back| exceeds 448 by two roundings at most, which the nearest code hides; an infinity has no code and becomes NaN, as NaN does.
__device__ __forceinline__ uint32_t codes8(float a, float b, float c, float d, float back) {
#pragma clang fp contract(off)
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * back, b * back, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * back, d * back, w, true);
}

// Eight elements from column c of a row of d on; what is behind the row's end is 0.  No access hangs on a branch that lanes take differently: where eight from c on are not there
// (RAGGED), the row's last eight are loaded, and moved down.
template <typename T, bool RAGGED>
struct Eight {
  static constexpr int WORDS = 2 * sizeof(T);
  typedef T vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  vec v;
  __device__ __forceinline__ void load(const T* row, int c, int d) {
    if (!RAGGED) {
      v = *reinterpret_cast<const vec*>(row + c);
    } else if (d >= 8) {
      v = *reinterpret_cast<const vec*>(row + min(c, d - 8));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < d ? row[e] : T(0);
    }
  }
  // What was loaded, where it belongs.
  __device__ __forceinline__ vec settled(int c, int d) const {
    if constexpr (!RAGGED) {
      return v;
    } else {
      struct Words {
        uint32_t w[WORDS];
      };
      Words t = __builtin_bit_cast(Words, v);
      const int up = d >= 8 ? min(max(c - (d - 8), 0), 8) : min(c, 8);
      auto down = [&](bool on, int words) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) t.w[i] = on ? (i + words < WORDS ? t.w[(i + words) % WORDS] : 0u) : t.w[i];
      };
      down(up & 8, WORDS);
      down(up & 4, WORDS / 2);
      down(up & 2, WORDS / 4);
      if constexpr (sizeof(T) == 4) {
        down(up & 1, 1);
      } else {
        const uint32_t by = (up & 1) * 16;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) t.w[i] = __builtin_amdgcn_alignbit(i + 1 < WORDS ? t.w[(i + 1) % WORDS] : 0u, t.w[i], by);
      }
      return __builtin_bit_cast(vec, t);
    }
  }
  __device__ __forceinline__ void get(float (&x)[8], int c, int d) const {
    const vec t = settled(c, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)t[e];
  }
  // Of the n (0 to 8) that are there.
  static __device__ __forceinline__ void store(T* to, const vec& t, int n) {
    if (!RAGGED || n >= 8) {
      *reinterpret_cast<vec*>(to) = t;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) to[e] = t[e];
    }
  }
};
// Eight codes, n (0 to 8) of which are there.
template <bool RAGGED>
__device__ __forceinline__ void store8(uint8_t* to, uint32_t lo, uint32_t hi, int n) {
  if (!RAGGED || n >= 8) {
    *reinterpret_cast<code2_any*>(to) = code2_any{lo, hi};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) to[e] = (uint8_t)((e < 4 ? lo : hi) >> 8 * (e & 3));
  }
}

// Eight codes times a power of two as bf16, which holds them exactly.
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ bf16x8_t widen8(uint32_t lo, uint32_t hi, float by = 1.f) {
  union {
    bf16x2_t two[4];
    bf16x8_t all;
  } u;
  u.two[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, false);
  u.two[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, true);
  u.two[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, false);
  u.two[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, true);
  return u.all;
}
