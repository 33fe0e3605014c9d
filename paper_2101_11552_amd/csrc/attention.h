// Attention inside each graph of a BatchGraph: what the forward and the
// gradient kernels share (gfx950).
#pragma once

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

// tanh. bf16 features: 1 - 2 / (1 + exp(2 x)) on the hardware's exponential and
// reciprocal; its absolute error of some 2^-22 is far below the features' rounding.
// float32 features: below 0.65 the odd polynomial x + x z P(z), z = x^2, P fitted to
// (tanh(x) / x - 1) / z for the least relative error (8e-8 with its roundings), above it
// the same form, whose error is a step or two there.
template <typename T> __device__ __forceinline__ float cap_tanh(float x) {
  if constexpr (sizeof(T) == 4) {
    const float z = x * x;
    float q = -0.005528633017092943f;
    q = __builtin_fmaf(q, z, 0.020483314990997314f);
    q = __builtin_fmaf(q, z, -0.05369296669960022f);
    q = __builtin_fmaf(q, z, 0.1333089917898178f);
    q = __builtin_fmaf(q, z, -0.3333326280117035f);
    const float low = __builtin_fmaf(x * z, q, x);
    const float e = __builtin_amdgcn_exp2f(fabsf(x) * (2.0f * kLog2e));
    const float high = __builtin_copysignf(1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + e), x);
    return fabsf(x) < 0.65f ? low : high;  // (NaN: high, NaN)
  } else {
    const float e = __builtin_amdgcn_exp2f(x * (2.0f * kLog2e));
    return 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + e);
  }
}

// The biases of the group's heads to LDS, B + 1 a head: bucket B and above are
// masked, -inf.
template <typename T>
__device__ __forceinline__ void load_bias(const AttnShape& a, int kvh, int grp, float* tab,
                                          int threads, int tid) {
  const T* b = static_cast<const T*>(a.bias) + (int64_t)kvh * grp * a.B;
  for (int i = tid; i < grp * (a.B + 1); i += threads) {
    const int h = i / (a.B + 1), j = i - h * (a.B + 1);
    tab[i] = j < a.B ? (float)b[h * a.B + j] : -INFINITY;
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

// ROWS rows of D columns to LDS (row-major, leading dimension LD), zeros from
// column D and row n on. at(r): a row's first element.
template <typename T, int ROWS, int DP, int LD, int THREADS, typename At>
__device__ __forceinline__ void stage_rows(T* dst, int n, int D, int vec, At at) {
  constexpr int C = DP / 8;
  for (int c = threadIdx.x; c < ROWS * C; c += THREADS) {
    const int r = c / C, d0 = (c % C) * 8;
    x8_t<T> v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (T)0.0f;
    if (r < n) v = load8<T>(at(r), d0, D, vec);
    put8<T>(dst + r * LD + d0, v);
  }
}

// ROWS rows to LDS as columns: dst[d][place of the row], places interleaved (see
// tiles.h), and with nat also row-major there.
template <typename T, int ROWS, int DP, int LDT, int LD, int THREADS, typename At>
__device__ __forceinline__ void stage_columns(T* dst, T* nat, int n, int D, int vec, At at) {
  constexpr int Q = ROWS / 4;
  for (int c = threadIdx.x; c < Q * (DP / 8); c += THREADS) {
    const int quad = c % Q, d0 = (c / Q) * 8;
    x8_t<T> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = (T)0.0f;
      if (quad * 4 + i < n) v[i] = load8<T>(at(quad * 4 + i), d0, D, vec);
      if (nat != nullptr) put8<T>(nat + (quad * 4 + i) * LD + d0, v[i]);
    }
    const int place = interleaved_quad(quad);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x4_t<T> w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i][e];
      *reinterpret_cast<x4_t<T>*>(dst + (d0 + e) * LDT + place) = w;
    }
  }
}

}  // namespace tfg
