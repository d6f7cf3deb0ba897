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

// Elements [i, i + E) of a row of n as they lie in memory, those past its end as 0. Not yet converted: several such loads
// are then under way together (a conversion inside the branch would wait for its load there: rows of 1024 float32 picked
// by token 170 -> 140 us for 128000). A row that ends inside is taken element by element.
// The words are kept as words: of an array of 16-bit values the compiler keeps one a register.
template <class T, int E>
struct Raw {
  static constexpr int kWords = E * (int)sizeof(T) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void to(float (&x)[E]) const {
#pragma unroll
    for (int u = 0; u < E; ++u) {
      if constexpr (sizeof(T) == 4) x[u] = __uint_as_float(w[u]);
      else if constexpr (std::is_same<T, Bf16>::value) x[u] = __uint_as_float(u & 1 ? w[u / 2] & 0xffff0000u : w[u / 2] << 16);
      else x[u] = to_float(F16{(uint16_t)(u & 1 ? w[u / 2] >> 16 : w[u / 2])});
    }
  }
};

template <class T, int E>
__device__ __forceinline__ Raw<T, E> raw_in(const T* row, int i, int n) {
  static_assert(E * sizeof(T) % 4 == 0, "whole words");
  Raw<T, E> r;
  // the zeros first and by themselves: written beside the load, in another branch, they would wait for it
#pragma unroll
  for (int q = 0; q < Raw<T, E>::kWords; ++q) r.w[q] = 0;
  if (i + E <= n) __builtin_memcpy(r.w, row + i, sizeof(r.w));
  if (i < n && i + E > n) {
#pragma unroll
    for (int u = 0; u < E; ++u)
      if (i + u < n) {
        if constexpr (sizeof(T) == 4) r.w[u] = __float_as_uint(row[i + u]);
        else r.w[u / 2] |= (uint32_t)row[i + u].bits << (16 * (u & 1));
      }
  }
  return r;
}

template <class T, int E>
__device__ __forceinline__ void load_in(const T* row, int i, int n, float (&x)[E]) {
  raw_in<T, E>(row, i, n).to(x);
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

// A lane's vector of a row without a branch around its load: the vector at i where it lies inside the row, else the row's last
// E elements, of which the first skip_of() are other lanes' (all E past the row's end). A branch for the last vector would
// hold up every load before it. Rows shorter than E (SHORT: there may be such) are taken by raw_in, where element u is i + u.
__device__ __forceinline__ int start_of(int i, int n, int E) { return n >= E ? min(i, n - E) : i; }
__device__ __forceinline__ int skip_of(int i, int n, int E) { return n >= E ? min(max(i + E - n, 0), E) : 0; }

template <class T, int E, bool SHORT = true>
__device__ __forceinline__ Raw<T, E> span_load(const T* row, int i, int n) {
  if (SHORT && n < E) return raw_in<T, E>(row, i, n);
  Raw<T, E> r;
  __builtin_memcpy(r.w, row + start_of(i, n, E), sizeof(r.w));
  return r;
}

// Whether the elements of such a vector are the lane's own, not those of others or past the row.
template <int E, bool SHORT = true>
__device__ __forceinline__ void span_own(int i, int n, bool (&own)[E]) {
  const int skip = skip_of(i, n, E);
#pragma unroll
  for (int u = 0; u < E; ++u) own[u] = SHORT && n < E ? i + u < n : u >= skip;
}

// store_in past the caches, for results much larger than they are.
template <class T, int E>
__device__ __forceinline__ void store_past_in(T* row, int i, int n, const float (&x)[E]) {
  typedef uint32_t Words __attribute__((ext_vector_type(E * sizeof(T) / 4), aligned(sizeof(T))));
  if (i + E <= n) {
    T v[E];
#pragma unroll
    for (int u = 0; u < E; ++u) v[u] = from_float<T>(x[u]);
    Words w;
    __builtin_memcpy(&w, v, sizeof(v));
    __builtin_nontemporal_store(w, reinterpret_cast<Words*>(row + i));
  } else {
    store_in<T, E>(row, i, n, x);
  }
}

// The lane's own elements of such a vector to a row, past the caches or not.
template <class T, int E, bool PAST, bool SHORT = true>
__device__ __forceinline__ void span_store(T* row, int i, int n, const float (&x)[E]) {
  if (i + E <= n || (SHORT && n < E)) {
    if constexpr (PAST) store_past_in<T, E>(row, i, n, x);
    else store_in<T, E>(row, i, n, x);
  } else if (i < n) {
    const int skip = skip_of(i, n, E);
#pragma unroll
    for (int u = 0; u < E; ++u)
      if (u >= skip) row[n - E + u] = from_float<T>(x[u]);
  }
}

}  // namespace vectors

// Size in bytes of an snn_dtype's values, 0 for an unknown one; whether an address suits it.
inline size_t dtype_size(int dtype) { return dtype == SNN_F32 ? 4 : dtype == SNN_BF16 || dtype == SNN_F16 ? 2 : 0; }
inline bool misaligned(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % dtype_size(dtype) != 0; }

}  // namespace snn
