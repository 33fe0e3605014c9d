// Vectors of a row's columns for kernels that pass over rows in float32, of
// float32 or bf16 (gfx950).
#pragma once

#include "tiles.h"

namespace tfg {

// V consecutive columns as float32. V elements at a time: rows start at multiples
// of V elements' bytes.
template <typename T, int V>
__device__ __forceinline__ void load_cols(const T* p, float (&x)[V]) {
  if constexpr (V == 8) {
    const x8_t<T> t = *reinterpret_cast<const x8_t<T>*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)t[i];
  } else if constexpr (V == 4) {
    const x4_t<T> t = *reinterpret_cast<const x4_t<T>*>(p);
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
    __builtin_nontemporal_store(t, reinterpret_cast<x8_t<T>*>(p));
  } else if constexpr (V == 4) {
    x4_t<T> t;
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = to_type<T>(x[i]);
    __builtin_nontemporal_store(t, reinterpret_cast<x4_t<T>*>(p));
  } else {
    *p = to_type<T>(x[0]);
  }
}

// Columns a lane takes: as many as 16 bytes hold, half of that, or one, by what the
// width, the leading dimensions and the addresses allow.
template <typename T> inline bool cols_fit(int v, const void* p, int64_t ld, int64_t F) {
  return reinterpret_cast<uintptr_t>(p) % (v * sizeof(T)) == 0 && ld % v == 0 && F % v == 0;
}

}  // namespace tfg
