// Rows of numbers taken E at a time, at any address their type allows (internal header). gfx950 loads and stores 16 bytes
// at any alignment; whole, aligned 16-byte pieces are the fastest.
#pragma once

#include "rows.h"

namespace snn {
namespace vectors {

using rows::Bf16;
using rows::F16;
using rows::from_float;
using rows::to_float;

template <class T, int E>
__device__ __forceinline__ void load(const T* p, float (&x)[E]) {
  T v[E];
  __builtin_memcpy(v, p, sizeof(v));
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] = to_float(v[i]);
}

template <class T, int E>
__device__ __forceinline__ void store(T* p, const float (&x)[E]) {
  T v[E];
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = from_float<T>(x[i]);
  __builtin_memcpy(p, v, sizeof(v));
}

// Elements [i, i + E) of a row of n, those past its end as 0 and not stored. A row that ends inside is taken element
// by element.
template <class T, int E>
__device__ __forceinline__ void load_in(const T* row, int i, int n, float (&x)[E]) {
  if (i + E <= n) {
    load<T, E>(row + i, x);
  } else {
#pragma unroll
    for (int u = 0; u < E; ++u) x[u] = i + u < n ? to_float(row[i + u]) : 0.0f;
  }
}

template <class T, int E>
__device__ __forceinline__ void store_in(T* row, int i, int n, const float (&x)[E]) {
  if (i + E <= n) {
    store<T, E>(row + i, x);
  } else {
#pragma unroll
    for (int u = 0; u < E; ++u)
      if (i + u < n) row[i + u] = from_float<T>(x[u]);
  }
}

}  // namespace vectors

// Size in bytes of an snn_dtype's values, 0 for an unknown one; whether an address suits it.
inline size_t dtype_size(int dtype) { return dtype == SNN_F32 ? 4 : dtype == SNN_BF16 || dtype == SNN_F16 ? 2 : 0; }
inline bool misaligned(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % dtype_size(dtype) != 0; }

}  // namespace snn
