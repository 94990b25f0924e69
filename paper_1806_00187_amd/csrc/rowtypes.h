// Rows of fp16, bf16 or fp32 elements for the kernels that take all three: 16 bytes a lane and access, whatever the address (the
// hardware takes global accesses at any address that the element type allows), held as fp32.
#pragma once

#include "common.h"

typedef __bf16 bf16_t;

template <typename T>
struct Row {
  static constexpr int kVec = 16 / sizeof(T);  // elements of one access
  typedef T vec __attribute__((ext_vector_type(kVec), aligned(sizeof(T))));
};

template <typename T>
__device__ __forceinline__ typename Row<T>::vec ld_vec(const T* p) { return *reinterpret_cast<const typename Row<T>::vec*>(p); }
template <typename T>
__device__ __forceinline__ void st_vec(T* p, const typename Row<T>::vec& x) { *reinterpret_cast<typename Row<T>::vec*>(p) = x; }
static inline bool row_type_ok(int type) { return type == NMT_F16 || type == NMT_BF16 || type == NMT_F32; }
static inline int row_type_bytes(int type) { return type == NMT_F32 ? 4 : 2; }
