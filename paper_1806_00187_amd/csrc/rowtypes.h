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

// Elements [c, c + kVec) of a row of d; those behind its end are 0.  RAGGED: d need not be a multiple of kVec.
template <bool RAGGED, typename T>
__device__ __forceinline__ void ld_row(const T* row, int c, int d, float* v) {
  constexpr int N = Row<T>::kVec;
  if (c + N <= d) {
    const typename Row<T>::vec x = *reinterpret_cast<const typename Row<T>::vec*>(row + c);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (float)x[e];
    return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = RAGGED && c + e < d ? (float)row[c + e] : 0.f;
}
template <bool RAGGED, typename T>
__device__ __forceinline__ void st_row(T* row, int c, int d, const float* v) {
  constexpr int N = Row<T>::kVec;
  if (c + N <= d) {
    typename Row<T>::vec x;
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = (T)v[e];
    *reinterpret_cast<typename Row<T>::vec*>(row + c) = x;
    return;
  }
  if (RAGGED) {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (c + e < d) row[c + e] = (T)v[e];
  }
}

static inline bool row_type_ok(int type) { return type == NMT_F16 || type == NMT_BF16 || type == NMT_F32; }
static inline int row_type_bytes(int type) { return type == NMT_F32 ? 4 : 2; }
