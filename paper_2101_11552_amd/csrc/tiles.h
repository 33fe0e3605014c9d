// Matrix tiles for the operators over a BatchGraph's nodes (gfx950): element
// types, 16x16 matrix products and the layouts their operands take.
//
// One product step multiplies a 16 x 32 by a 32 x 16 tile. Lane l holds eight
// consecutive k of row (operand A) or column (operand B) l % 16, starting at
// k = 8 * (l / 16); the result has column l % 16 and rows 4 * (l / 16) + i in
// register i. bf16 takes one v_mfma_f32_16x16x32_bf16, float32 eight
// v_mfma_f32_16x16x4_f32 (element e of every lane is one step of four k), so
// both types share every index.
//
// A result becomes the operand of the next product without leaving its
// registers: the 32 k of a step are numbered so that the lane group g = l / 16
// owns k = 16 a + 4 g + i (a = 0, 1 the two result tiles, i the register),
// and the other operand is stored in LDS in that order ("interleaved": k =
// 16 a + 4 g + i at place 8 g + 4 a + i), read as eight consecutive elements.
#pragma once

#include "wave.h"

namespace tfg {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

template <typename T> struct Vec;
template <> struct Vec<float> {
  typedef f32x8 x8;
  typedef f32x4 x4;
};
template <> struct Vec<__bf16> {
  typedef bf16x8 x8;
  typedef bf16x4 x4;
};
template <typename T> using x8_t = typename Vec<T>::x8;
template <typename T> using x4_t = typename Vec<T>::x4;

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f32x8 a, f32x8 b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// Heads of at most 16 columns: a 16 x 16 by 16 x 16 step, four consecutive k a lane.
__device__ __forceinline__ f32x4 mma(bf16x4 a, bf16x4 b, f32x4 c) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a),
                                                   __builtin_bit_cast(s16x4, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// Rounded to nearest even.
template <typename T> __device__ __forceinline__ T to_type(float x) { return (T)x; }

// Place, inside 32, of the k that result register i of tile a holds in group g:
// for the four rows 4 * quad .. + 3 of a tile of 32, the first of their places.
__device__ __forceinline__ int interleaved_quad(int quad) {
  return (quad & ~7) * 4 + (quad & 3) * 8 + ((quad >> 2) & 1) * 4;
}

// How rows may be read: 8 elements at a time (every row starts at a multiple of
// 16 bytes and has a multiple of 16 bytes of columns), 4 (of 8 bytes; bf16 only)
// or one.
template <typename T> __host__ inline int row_vector(const void* p, int64_t ld, int64_t D) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  const int per = (int)(16 / sizeof(T));  // elements in 16 bytes
  if (a % 16 == 0 && ld % per == 0 && D % per == 0) return 8;
  if (sizeof(T) == 2 && a % 8 == 0 && ld % 4 == 0 && D % 4 == 0) return 4;
  return 1;
}

// Elements d0 .. d0 + 7 of a row of D, zeros from D on. d0 is a multiple of 8.
template <typename T>
__device__ __forceinline__ x8_t<T> load8(const T* row, int d0, int D, int vec) {
  x8_t<T> v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (T)0.0f;
  if (d0 >= D) return v;
  if (vec == 8) {
    if constexpr (sizeof(T) == 2) {
      v = *reinterpret_cast<const bf16x8*>(row + d0);
    } else {
      const f32x4 lo = *reinterpret_cast<const f32x4*>(row + d0);
      f32x4 hi = {0.0f, 0.0f, 0.0f, 0.0f};
      if (d0 + 4 < D) hi = *reinterpret_cast<const f32x4*>(row + d0 + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = lo[e];
        v[4 + e] = hi[e];
      }
    }
  } else if (vec == 4) {
    const x4_t<T> lo = *reinterpret_cast<const x4_t<T>*>(row + d0);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = lo[e];
    if (d0 + 4 < D) {
      const x4_t<T> hi = *reinterpret_cast<const x4_t<T>*>(row + d0 + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 + e] = hi[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (d0 + e < D) v[e] = row[d0 + e];
  }
  return v;
}

// Elements d0 .. d0 + 3 (d0 a multiple of 4) of a row of D, rounded once. vec > 1:
// the row starts at a multiple of four elements and D is one.
template <typename T>
__device__ __forceinline__ void store4(T* row, int d0, int D, int vec, f32x4 x) {
  if (d0 >= D) return;
  if (vec > 1) {
    x4_t<T> v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = to_type<T>(x[e]);
    *reinterpret_cast<x4_t<T>*>(row + d0) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (d0 + e < D) row[d0 + e] = to_type<T>(x[e]);
  }
}

// Eight consecutive elements of an LDS row (16-byte aligned).
template <typename T>
__device__ __forceinline__ x8_t<T> lds8(const T* p) {
  if constexpr (sizeof(T) == 2) {
    return *reinterpret_cast<const bf16x8*>(p);
  } else {
    const f32x4 lo = *reinterpret_cast<const f32x4*>(p);
    const f32x4 hi = *reinterpret_cast<const f32x4*>(p + 4);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

// Columns added to an LDS row that is read one row a lane at a time.
template <typename T> constexpr int lds_pad() { return 16 / (int)sizeof(T); }

// A lane's part of a head's DP columns as an operand: KC chunks of 32 (of 16 for DP =
// 16), eight (four) consecutive columns of each.
template <typename T, int DP> struct Frag {
  static constexpr int N = DP == 16 ? 4 : 8, KC = DP == 16 ? 1 : DP / 32, W = 4 * N;
  typedef T type __attribute__((ext_vector_type(N)));
};
template <typename T, int DP> using frag_t = typename Frag<T, DP>::type;

template <typename T, int DP>
__device__ __forceinline__ frag_t<T, DP> zero_frag() {
  frag_t<T, DP> v;
#pragma unroll
  for (int e = 0; e < Frag<T, DP>::N; ++e) v[e] = (T)0.0f;
  return v;
}
// Chunk c of lane group g of a row of D columns in memory (see load8).
template <typename T, int DP>
__device__ __forceinline__ frag_t<T, DP> load_frag(const T* row, int c, int g, int D, int vec) {
  if constexpr (DP == 16) {
    frag_t<T, DP> v = zero_frag<T, DP>();
    const int d0 = g * 4;
    if (d0 >= D) return v;
    if (vec > 1) return *reinterpret_cast<const frag_t<T, DP>*>(row + d0);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (d0 + e < D) v[e] = row[d0 + e];
    return v;
  } else {
    return load8<T>(row, c * 32 + g * 8, D, vec);
  }
}

// A tile of LDS rows of COLS elements that operands are read from: lane l row l % 16,
// 16 bytes at column chunk l / 16 of a step. Of 64 such lanes the LDS serves 0..3, 12..15
// and 20..27 together, then 4..11, 16..19 and 28..31, and so on, so padded rows, without
// conflicts among 16 neighbouring lanes, meet in these groups: 8.1 cycles a read against
// 4.4 without conflicts. Here chunk j of a row is kept at j ^ key(row), no padding, with
// keys that put each such group into different banks (attention forward, bf16, width 128:
// 236 -> 200 us; float32's products take longer than its reads: padded). 16 bf16 columns
// are read 8 bytes a lane, from padded rows.
template <typename T, int COLS, bool SWAP = sizeof(T) == 2> struct Tile {
  static constexpr int PER = 16 / (int)sizeof(T), CHUNKS = COLS / PER;
  static constexpr bool PAD = !SWAP || CHUNKS == 2;
  static constexpr int LD = PAD ? COLS + PER : COLS;
  static __device__ __forceinline__ int key(int row) {
    if constexpr (PAD) return 0;
    if constexpr (CHUNKS >= 16) return row & 15;
    // rows 0-3 and 12-15 the keys 0..3, rows 4-11 the keys 4..7: both sets are closed under
    // ^ 1 and ^ 2, the difference between the lane groups' chunks
    if constexpr (CHUNKS == 8) return ((row >> 1) & 1) | ((row >> 2) & 2) | ((row ^ (row >> 1)) & 4);
    if constexpr (CHUNKS == 4) return -(row >> 2) & 3;
    return 0;
  }
  static __device__ __forceinline__ int at(int row, int col) {
    return row * LD + ((col / PER) ^ key(row)) * PER + col % PER;
  }
  // Eight columns from col on, a multiple of eight.
  static __device__ __forceinline__ x8_t<T> get8(const T* tile, int row, int col) {
    if constexpr (sizeof(T) == 2) {
      return *reinterpret_cast<const bf16x8*>(tile + at(row, col));
    } else {
      const f32x4 lo = *reinterpret_cast<const f32x4*>(tile + at(row, col));
      const f32x4 hi = *reinterpret_cast<const f32x4*>(tile + at(row, col + 4));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
  static __device__ __forceinline__ void put8(T* tile, int row, int col, x8_t<T> v) {
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<bf16x8*>(tile + at(row, col)) = v;
    } else {
      *reinterpret_cast<f32x4*>(tile + at(row, col)) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
      *reinterpret_cast<f32x4*>(tile + at(row, col + 4)) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
    }
  }
  // Four rows of eight columns of another tile as columns of this one, places interleaved.
  static __device__ __forceinline__ void put_columns(T* tile, int quad, int d0, const x8_t<T> (&v)[4]) {
    const int place = interleaved_quad(quad);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x4_t<T> w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i][e];
      *reinterpret_cast<x4_t<T>*>(tile + at(d0 + e, place)) = w;
    }
  }
  // Chunk c of lane group g of a row of this many columns as an operand.
  static __device__ __forceinline__ frag_t<T, COLS> frag(const T* tile, int row, int c, int g) {
    if constexpr (COLS == 16) return *reinterpret_cast<const frag_t<T, 16>*>(tile + at(row, g * 4));
    else return get8(tile, row, c * 32 + g * 8);
  }
};

// Two result tiles (a = 0, 1) as one operand of 32 k.
template <typename T>
__device__ __forceinline__ x8_t<T> as_operand(f32x4 lo, f32x4 hi) {
  x8_t<T> v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = to_type<T>(lo[i]);
    v[4 + i] = to_type<T>(hi[i]);
  }
  return v;
}

}  // namespace tfg
