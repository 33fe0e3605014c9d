// Vectors of a row's columns for kernels that pass over rows in float32, of
// float32 or bf16 (gfx950).
#pragma once

#include "tiles.h"

namespace tfg {

template <typename T> using any8_t = x8_t<T> __attribute__((aligned(sizeof(T))));
template <typename T> using any4_t = x4_t<T> __attribute__((aligned(sizeof(T))));

// V consecutive columns as float32, at any address of an element (16-byte accesses need
// no alignment here).
template <typename T, int V>
__device__ __forceinline__ void load_cols(const T* p, float (&x)[V]) {
  if constexpr (V == 8) {
    const any8_t<T> t = *reinterpret_cast<const any8_t<T>*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)t[i];
  } else if constexpr (V == 4) {
    const any4_t<T> t = *reinterpret_cast<const any4_t<T>*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)t[i];
  } else {
    x[0] = (float)*p;
  }
}

template <typename T, int V>
__device__ __forceinline__ void store_cols(T* p, const float (&x)[V]) {
  if constexpr (V == 8) {
    x8_t<T> t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = to_type<T>(x[i]);
    any8_t<T> u = t;
    __builtin_nontemporal_store(u, reinterpret_cast<any8_t<T>*>(p));
  } else if constexpr (V == 4) {
    x4_t<T> t;
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = to_type<T>(x[i]);
    any4_t<T> u = t;
    __builtin_nontemporal_store(u, reinterpret_cast<any4_t<T>*>(p));
  } else {
    *p = to_type<T>(x[0]);
  }
}

// Columns in 16 bytes.
template <typename T> constexpr int vector_cols() { return 16 / (int)sizeof(T); }

}  // namespace tfg
