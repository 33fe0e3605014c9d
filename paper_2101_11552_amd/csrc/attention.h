// Attention inside each graph of a BatchGraph: what the forward and the
// gradient kernels share (gfx950).
#pragma once

#include <type_traits>

#include "spans.h"
#include "tiles.h"

namespace tfg {

// Entries of the bias table that one key/value head's query heads may have: its
// copy in LDS (16 KB).
constexpr int kMaxBiasEntries = 4096;
constexpr int kMaxHeadDim = 128;

// A query tile's graph. Rows: the rows of one key/value head of graph g are the
// pairs (query, query head of the group), query-major: row r is query r / grp
// and head kvh * grp + r % grp, so that shared heads read their keys once.
struct Span {
  int g, tile;             // graph, tile of it; g < 0: no tile here
  int q0, nq, k0, nk;      // its queries and keys
};

// The tile of slot t among tiles of TILE rows (see spans.h), and its graph's
// queries and keys.
template <int TILE>
__device__ __forceinline__ Span find_span(const AttnShape& a, const int* off, int n_off, int grp,
                                          int64_t slot) {
  const Run r = find_run<TILE>(off, a.G, n_off, grp, slot);
  if (r.g < 0) return Span{-1, 0, 0, 0, 0, 0};
  Span s;
  s.g = r.g;
  s.tile = r.tile;
  s.q0 = clamp_off(uniform(a.qoff[r.g]), a.Nq);
  s.nq = max(clamp_off(uniform(a.qoff[r.g + 1]), a.Nq) - s.q0, 0);
  s.k0 = clamp_off(uniform(a.koff[r.g]), a.Nk);
  s.nk = max(clamp_off(uniform(a.koff[r.g + 1]), a.Nk) - s.k0, 0);
  return s;
}

// Beside the launch over small graphs (attention_small.h), kRestBlocks blocks take the tiles
// of the graphs that have more than `small` queries or keys: block b the tiles b, +
// kRestBlocks, .. in the graphs' order. 64 lanes look at 64 graphs at a time, and a block
// goes on where it was. A batch without such graphs is seen at once, by all threads.
constexpr int kRestBlocks = 512;
__device__ __forceinline__ bool any_rest(const AttnShape& a, int small) {
  bool any = false;
  for (int g0 = 0; g0 < a.G; g0 += 16 * (int)blockDim.x) {
    int q[16][2], k[16][2];
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      const int g = min(g0 + u * (int)blockDim.x + (int)threadIdx.x, a.G - 1);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        q[u][e] = a.qoff[g + e];
        k[u][e] = a.koff[g + e];
      }
    }
#pragma unroll
    for (int u = 0; u < 16; ++u)
      any = any || clamp_off(q[u][1], a.Nq) - clamp_off(q[u][0], a.Nq) > small ||
            clamp_off(k[u][1], a.Nk) - clamp_off(k[u][0], a.Nk) > small;
  }
  return __syncthreads_or(any) != 0;
}
struct RestScan {
  int base = 0, count = 0;  // graphs before base have `count` tiles
};
template <int TILE, bool KEYS>
__device__ __forceinline__ Span next_span(const AttnShape& a, int grp, int small, int index, RestScan& st) {
  for (; st.base < a.G; st.base += kWave) {
    const int g = min(st.base + lane_id(), a.G - 1);
    Span s;
    s.q0 = clamp_off(a.qoff[g], a.Nq);
    s.nq = max(clamp_off(a.qoff[g + 1], a.Nq) - s.q0, 0);
    s.k0 = clamp_off(a.koff[g], a.Nk);
    s.nk = max(clamp_off(a.koff[g + 1], a.Nk) - s.k0, 0);
    const bool rest = st.base + lane_id() < a.G && (s.nq > small || s.nk > small);
    const int64_t rows = KEYS ? (int64_t)s.nk : (int64_t)s.nq * grp;
    const int tiles = rest ? (int)((rows + TILE - 1) / TILE) : 0;
    const int incl = wave_incl_scan(tiles), total = __shfl(incl, kWave - 1);
    if (index < st.count + total) {
      const int l = uniform(__ffsll((long long)__ballot(index < st.count + incl)) - 1);
      s.g = uniform(st.base + l);
      s.tile = uniform(index - st.count - __shfl(incl - tiles, l));
      s.q0 = uniform(__shfl(s.q0, l));
      s.nq = uniform(__shfl(s.nq, l));
      s.k0 = uniform(__shfl(s.k0, l));
      s.nk = uniform(__shfl(s.nk, l));
      return s;
    }
    st.count = uniform(st.count + total);
  }
  return Span{-1, 0, 0, 0, 0, 0};
}

// The distance bytes [nq, nk] of a span's graph, or NULL where they would not
// lie inside the array (every pair is then masked).
__device__ __forceinline__ const uint8_t* dist_block(const AttnShape& a, const Span& s) {
  const int64_t o = a.doff[s.g];
  if (o < 0 || o > a.dist_bytes || (int64_t)s.nq * s.nk > a.dist_bytes - o) return nullptr;
  return a.dist + o;
}

typedef unsigned u32_u __attribute__((aligned(1)));

// Four buckets of a row of n from j on (255, masked, from n on); any alignment.
__device__ __forceinline__ unsigned load_buckets(const uint8_t* row, int j, int n) {
  if (j + 4 <= n) return *reinterpret_cast<const u32_u*>(row + j);
  unsigned v = 0xFFFFFFFFu;
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (j + i < n) v = (v & ~(0xFFu << (8 * i))) | ((unsigned)row[j + i] << (8 * i));
  return v;
}

// f * tanh(x * to_tanh) + add, with to_exp = 2 log2(e) to_tanh.
// bf16 features: f + add - 2 f / (1 + exp(2 x to_tanh)) on the hardware's exponential
// and reciprocal, add given with f in it; the tanh's absolute error of some 2^-22 is
// far below the features' rounding.
// float32 features: below 0.65 the odd polynomial x + x z P(z), z = x^2, P fitted to
// (tanh(x) / x - 1) / z for the least relative error (8e-8 with its roundings), above it
// the same form, whose error is a step or two there.
template <typename T>
__device__ __forceinline__ float capped(float x, float to_tanh, float to_exp, float f, float add) {
  if constexpr (sizeof(T) == 4) {
    x *= to_tanh;
    const float z = x * x;
    float q = -0.005528633017092943f;
    q = __builtin_fmaf(q, z, 0.020483314990997314f);
    q = __builtin_fmaf(q, z, -0.05369296669960022f);
    q = __builtin_fmaf(q, z, 0.1333089917898178f);
    q = __builtin_fmaf(q, z, -0.3333326280117035f);
    const float low = __builtin_fmaf(x * z, q, x);
    const float e = __builtin_amdgcn_exp2f(fabsf(x) * (2.0f * kLog2e));
    const float high = __builtin_copysignf(1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + e), x);
    return __builtin_fmaf(f, fabsf(x) < 0.65f ? low : high, add);  // (NaN: high, NaN)
  } else {
    return __builtin_fmaf(-2.0f * f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * to_exp)), add);
  }
}
// What `add` carries beside the bias.
template <typename T> __device__ __forceinline__ float cap_offset(float f) {
  return sizeof(T) == 2 ? f : 0.0f;
}

// The biases of the group's heads to LDS, plus `offset`, B + 1 a head: bucket B and
// above are masked, -inf.
template <typename T>
__device__ __forceinline__ void load_bias(const AttnShape& a, int kvh, int grp, float offset,
                                          float* tab, int threads, int tid) {
  const T* b = static_cast<const T*>(a.bias) + (int64_t)kvh * grp * a.B;
  for (int i = tid; i < grp * (a.B + 1); i += threads) {
    const int h = i / (a.B + 1), j = i - h * (a.B + 1);
    tab[i] = j < a.B ? (float)b[h * a.B + j] + offset : -INFINITY;
  }
}
inline size_t bias_table_bytes(const AttnShape& a) {
  return a.B > 0 ? sizeof(float) * (size_t)(a.H / a.Hk) * (a.B + 1) : 0;
}

// Capped scores are at most cap: up to this one their exponentials need no running
// maximum (e^60 times 2^31 terms is far inside float32).
constexpr float kBoundedCap = 60.0f;
// Scores beyond this are differences of large numbers: see the kernels.
constexpr float kHugeScore = 1.0e37f;

// Eight columns from d0 on of the row at element `at` past base (the same in every lane;
// below 64 rows of less than 2^23 elements, so bytes fit 32 bits and the address takes one
// register). VEC 8: D is a multiple of 16 bytes, the row of one element (16-byte loads at
// any address); 4: D is a multiple of four. Columns past D are read from the row's last
// ones: finite where the row is, and the other operand of their product is zero.
template <typename V, typename T>
__device__ __forceinline__ V load_at(const T* base, unsigned at) {
  return *reinterpret_cast<const V*>(reinterpret_cast<const char*>(base) + at * (unsigned)sizeof(T));
}
template <typename T, int VEC>
__device__ __forceinline__ x8_t<T> load8_within(const T* base, unsigned at, int d0, int D) {
  if constexpr (VEC == 8 && sizeof(T) == 2) {
    typedef bf16x8 any8 __attribute__((aligned(2)));
    return load_at<any8>(base, at + min(d0, D - 8));
  } else if constexpr (VEC >= 4) {
    typedef x4_t<T> any4 __attribute__((aligned(sizeof(T))));
    const x4_t<T> lo = load_at<any4>(base, at + min(d0, D - 4));
    const x4_t<T> hi = load_at<any4>(base, at + min(d0 + 4, D - 4));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  } else {
    x8_t<T> v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = load_at<T>(base, at + min(d0 + e, D - 1));
    return v;
  }
}
// Whether a kernel's loads may be VEC = 8: a choice for the whole kernel, since a branch
// around loads would make every tile wait for them.
template <typename T> inline bool whole_vectors(int D) { return D % (16 / (int)sizeof(T)) == 0; }

// Calls f with the vector length as a constant: 8, or (VEC 0) by the width, where each tile
// waits for its loads.
template <typename T, int VEC, typename F>
__device__ __forceinline__ void with_vector(int D, F f) {
  if constexpr (VEC == 8) {
    f(std::integral_constant<int, 8>{});
  } else {
    if (D % 4 == 0) f(std::integral_constant<int, 4>{});
    else f(std::integral_constant<int, 1>{});
  }
}

// A thread's units of a tile of ROWS rows: unit c is eight columns of row row8(c), or of
// the four rows of quad(c).
template <int ROWS, int DP>
struct Units {
  static constexpr int C = DP / 8;
  static __device__ __forceinline__ int row8(int c) { return c / C; }
  static __device__ __forceinline__ int col8(int c) { return (c % C) * 8; }
  static __device__ __forceinline__ int quad(int c) { return c % (ROWS / 4); }
  static __device__ __forceinline__ int quad_col(int c) { return (c / (ROWS / 4)) * 8; }
};

}  // namespace tfg
