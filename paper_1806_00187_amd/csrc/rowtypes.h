// Rows of fp16, bf16 or fp32 elements for the kernels that take all three: 16 bytes a lane and access, whatever the address (the
// hardware takes global accesses at any address that the element type allows), held as fp32.
#pragma once

#include "common.h"

#include <type_traits>

typedef __bf16 bf16_t;

template <typename T>
struct Row {
  static constexpr int kVec = 16 / sizeof(T);  // elements of one access
  typedef T vec __attribute__((ext_vector_type(kVec), aligned(sizeof(T))));
};

// STREAM: past the caches.
template <bool STREAM = false, typename T>
__device__ __forceinline__ typename Row<T>::vec ld_vec(const T* p) {
  const auto* v = reinterpret_cast<const typename Row<T>::vec*>(p);
  return STREAM ? __builtin_nontemporal_load(v) : *v;
}
template <bool STREAM = false, typename T>
__device__ __forceinline__ void st_vec(T* p, const typename Row<T>::vec& x) {
  auto* v = reinterpret_cast<typename Row<T>::vec*>(p);
  if (STREAM) __builtin_nontemporal_store(x, v);
  else *v = x;
}

// Sum over a wavefront's groups of 8, 16, 32 or 64 lanes; every lane gets its group's.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (LANES == 64) {
    return wave_sum(v);
  } else {
    auto plus = [](float x, auto ctrl) {
      return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    if constexpr (LANES == 32) {
      const auto h = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
      v = __builtin_bit_cast(float, (unsigned)h[0]) + __builtin_bit_cast(float, (unsigned)h[1]);
    }
    if constexpr (LANES == 8) {
      v = plus(v, std::integral_constant<int, 0x141>{});  // row_half_mirror
    } else {
      v = plus(v, std::integral_constant<int, 0x128>{});  // row_ror:8
      v = plus(v, std::integral_constant<int, 0x124>{});  // row_ror:4
    }
    v = plus(v, std::integral_constant<int, 0x4E>{});     // quad_perm:[2,3,0,1]
    return plus(v, std::integral_constant<int, 0xB1>{});  // quad_perm:[1,0,3,2]
  }
}

static inline bool row_type_ok(int type) { return type == NMT_F16 || type == NMT_BF16 || type == NMT_F32; }
static inline int row_type_bytes(int type) { return type == NMT_F32 ? 4 : 2; }
