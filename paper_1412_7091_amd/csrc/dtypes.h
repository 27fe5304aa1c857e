// Element types of the operators around the output layer: float32, bfloat16 and
// float16 in memory, float32 in registers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "lst.h"

namespace lst {

// N elements at any address that an element may have, in accesses of up to 16 bytes,
// which global memory takes without further alignment.
template <class T, int N>
__device__ inline void load_vec(const T* p, T (&v)[N]) {
  if constexpr (N == 1) {
    v[0] = *p;
  } else {
    constexpr int M = (int)sizeof(T) * N > 16 ? 16 / (int)sizeof(T) : N;
    typedef T vec __attribute__((ext_vector_type(M), aligned(sizeof(T))));
#pragma unroll
    for (int j = 0; j < N; j += M) {
      const vec w = *reinterpret_cast<const vec*>(p + j);
#pragma unroll
      for (int i = 0; i < M; ++i) v[j + i] = w[i];
    }
  }
}

// N elements of a row of `cols`, from column `col`; zeros behind the last.  The loads at the
// end do not depend on each other: with a branch for each they wait for one another.
template <class T, int N>
__device__ inline void load_part(const T* row, int col, int cols, T (&v)[N]) {
  if (col + N <= cols) {
    load_vec(row + col, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (T)0.f;
    if (col < cols) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = row[min(col + i, cols - 1)];
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = col + i < cols ? v[i] : (T)0.f;
    }
  }
}

template <class T, int N>
__device__ inline void store_vec(T* p, const T (&v)[N]) {
  if constexpr (N == 1) {
    *p = v[0];
  } else {
    constexpr int M = (int)sizeof(T) * N > 16 ? 16 / (int)sizeof(T) : N;
    typedef T vec __attribute__((ext_vector_type(M), aligned(sizeof(T))));
#pragma unroll
    for (int j = 0; j < N; j += M) {
      vec w;
#pragma unroll
      for (int i = 0; i < M; ++i) w[i] = v[j + i];
      *reinterpret_cast<vec*>(p + j) = w;
    }
  }
}

// Calls f with a value of the element type that dtype names.
template <class F>
inline int with_dtype(int dtype, F f) {
  switch (dtype) {
    case LST_F32: return f(float{});
    case LST_BF16: return f(__bf16{});
    case LST_F16: return f(_Float16{});
    default: return LST_EINVAL;
  }
}

inline bool known_dtype(int dtype) {
  return dtype == LST_F32 || dtype == LST_BF16 || dtype == LST_F16;
}

inline int launched() { return hipGetLastError() == hipSuccess ? LST_OK : LST_EHIP; }

}  // namespace lst
