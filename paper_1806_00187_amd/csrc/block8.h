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

// Largest magnitude over groups of 16 lanes; every lane gets its group's.
__device__ __forceinline__ float lanes16_max(float v) {
  auto meet = [](float x, auto ctrl) {
    return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true)));
  };
  v = meet(v, std::integral_constant<int, 0x128>{});  // row_ror:8
  v = meet(v, std::integral_constant<int, 0x124>{});  // row_ror:4
  v = meet(v, std::integral_constant<int, 0x4E>{});   // quad_perm:[2,3,0,1]
  return meet(v, std::integral_constant<int, 0xB1>{});  // quad_perm:[1,0,3,2]
}

// An element's part in its block's largest magnitude: what is inf or NaN has none.
__device__ __forceinline__ float magnitude8(float x) {
  const float a = fabsf(x);
  return a < __builtin_inff() ? a : 0.f;
}
// A block's scale and the scale's reciprocal, each rounded once; nothing is left of a block that is next to nothing.
struct Scale8 { float scale, back; };
__device__ __forceinline__ Scale8 scale8(float top) {
#pragma clang fp contract(off)
  Scale8 s = {0.f, 0.f};
  if (top > kTiny8) {
    s.scale = top * (1.f / kTop8);
    s.back = 1.f / s.scale;
  }
  return s;
}
// Four codes, nearest, ties to even.  |x back| exceeds 448 by two roundings at most, which the nearest code hides; what is inf or NaN becomes NaN.
__device__ __forceinline__ uint32_t codes8(float a, float b, float c, float d, float back) {
#pragma clang fp contract(off)
  auto q = [back](float x) { return fabsf(x) < __builtin_inff() ? x * back : __uint_as_float(0x7FC00000u); };
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(q(a), q(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q(c), q(d), w, true);
}

// Eight elements from column c of a row of d on, which may end before them (what is behind it is 0) or before c.  No access hangs on a branch that lanes take differently: of a row of
// at least 8 columns the last 8 are loaded, and moved up.
template <typename T, bool RAGGED>
struct Eight {
  typedef T vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  vec v;
  __device__ __forceinline__ void load(const T* row, int c, int d) {
    if (!RAGGED) {
      v = *reinterpret_cast<const vec*>(row + c);
    } else if (d >= 8) {
      v = *reinterpret_cast<const vec*>(row + min(c, d - 8));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = row[min(e, d - 1)];
    }
  }
  __device__ __forceinline__ void get(float (&x)[8], int c, int d) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
    if (RAGGED) {
      const int up = d >= 8 ? c - min(c, d - 8) : 0;
#pragma unroll
      for (int by = 4; by >= 1; by /= 2)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (up & by) && e + by < 8 ? x[(e + by) & 7] : x[e];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = c + e < d ? x[e] : 0.f;
    }
  }
  static __device__ __forceinline__ void store(T* row, const float (&x)[8], int c, int d) {
    vec t;
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = (T)x[e];
    if (!RAGGED || c + 8 <= d) {
      *reinterpret_cast<vec*>(row + c) = t;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < d) row[c + e] = t[e];
    }
  }
};

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
