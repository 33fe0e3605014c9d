// Group norm with an activation over the graphs of a BatchGraph, channels last
// (gfx950): every graph is a sample, its nodes the positions; the F channels fall
// into K groups of C = F / K.
//
//   xh = (x - mean) * rstd,  z = xh * gamma + beta,  out = act(z)
//   dz = dout * act'(z), dgamma = sum dz xh, dbeta = sum dz (over all nodes),
//   dh = dz * gamma, dx = rstd (dh - mean(dh) - xh mean(dh xh)) (means over the
//   graph's nodes and the group's channels)
//
// Both directions are a sum of two terms per channel (x, x^2; dz, dz xh) over the
// graph's nodes, a small step per group, and a pass that applies it. Sums are
// double: x^2 of a float32 is then exact and var = E[x^2] - mean^2 keeps some 15
// digits where the mean is far from zero; the kernels stay bound by memory.
// Small graphs take a wavefront each for all three steps (their rows are read again
// from the caches); larger ones are cut into tiles of rows.
//
// What bounds it: one graph of 169,343 nodes, 128 channels, float32, both directions: 151 us
// for 436 MB needed once (2.9 TB/s; x and dout are read twice, 4.6 TB/s with that); 4,096
// graphs of 35 nodes, 128 channels, bf16: 101 us, the latency of a graph's chain of sums,
// statistics and apply in its wavefront.
#include "columns.h"
#include "rows.h"
#include "spans.h"

namespace tfg {

namespace {

constexpr int kThreads = 256;
constexpr int kNormTile = 128;  // rows of a tile
constexpr int kU = 4;           // rows in flight per thread (eight: fewer wavefronts, 62 -> 78 us)

struct NormArgs {
  const void *x, *gi, *gamma, *beta, *dout;
  void *out, *dx;
  float *mean, *rstd;   // [G, K]
  const int* goff;      // [G + 1] (tiles)
  double* sums;         // [tiles or wavefronts][F][2] channels' sums (backward)
  double* groups;       // [tiles][K + slabs][2] groups' sums: slab s has group k at k + s
  float* coef;          // [G, K][2] (backward, tiles)
  int slab, slabs;      // columns a block of the tiles takes, and how many make a row
  int64_t ldx;
  int Nb, G, F, K, C, act;
  int lpr, rp;          // lanes a row, rows a block and step
  float eps;
};

// 1 + erf(z / sqrt 2) and exp(-z^2 / 2): the rational form 7.1.26 of Abramowitz and
// Stegun's handbook (error 1.5e-7 of the unit), whose exponential the slope needs too.
__device__ __forceinline__ float one_plus_erf(float z, float* gauss) {
  const float x = fabsf(z) * 0.70710678118654752440f;
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, x, 1.0f));
  const float e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * z * z);
  float q = __builtin_fmaf(1.061405429f, t, -1.453152027f);
  q = __builtin_fmaf(q, t, 1.421413741f);
  q = __builtin_fmaf(q, t, -0.284496736f);
  q = __builtin_fmaf(q, t, 0.254829592f);
  q *= t * e;  // 1 - erf(|x|)
  *gauss = e;
  return z < 0.0f ? q : 2.0f - q;
}
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * z));
}
// act(z) and act'(z).
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == TFG_ACT_RELU) return z > 0.0f ? z : (z == z ? 0.0f : z);
  if (act == TFG_ACT_SILU) return z * sigmoid(z);
  if (act == TFG_ACT_GELU) {
    float e;
    return 0.5f * z * one_plus_erf(z, &e);
  }
  return z;
}
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == TFG_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
  if (act == TFG_ACT_SILU) {
    const float s = sigmoid(z);
    return s * (1.0f + z * (1.0f - s));
  }
  if (act == TFG_ACT_GELU) {
    float e;
    const float c = one_plus_erf(z, &e);
    return __builtin_fmaf(z * 0.39894228040143267794f, e, 0.5f * c);
  }
  return 1.0f;
}

// First n in [0, Nb] with gi[n] >= g (b) and >= g + 1 (e), each by 64 probes at a
// time (three rounds for 262,144 nodes), the two searches' loads together. Any
// graph_index ends it with 0 <= b, e <= Nb.
template <typename IdxT>
__device__ __forceinline__ void graph_rows(const IdxT* __restrict__ gi, int Nb, int g, int* b, int* e) {
  int lo[2] = {0, 0}, hi[2] = {Nb, Nb};
  while (hi[0] > lo[0] || hi[1] > lo[1]) {
    int step[2], cnt[2];
    bool lt[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      step[w] = (hi[w] - lo[w] + kWave - 1) / kWave;
      const int at = lo[w] + lane_id() * step[w];
      lt[w] = at < hi[w] && (int64_t)gi[at] < (int64_t)g + w;
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      cnt[w] = __popcll(__ballot(lt[w]));
      const int l = lo[w];
      hi[w] = uniform(cnt[w] == 0 ? l : min(l + cnt[w] * step[w], hi[w]));
      lo[w] = uniform(cnt[w] == 0 ? l : min(l + (cnt[w] - 1) * step[w] + 1, hi[w]));
    }
  }
  *b = lo[0];
  *e = max(lo[1], lo[0]);
}

// What a lane's V channels need of their graph: mean and rstd, and in the
// backward's last pass the two means.
template <typename T, int V>
struct Channels {
  float gamma[V], beta[V];
  int k[V];
  __device__ __forceinline__ void load(const NormArgs& p, int c) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      k[v] = (c + v) / p.C;
      gamma[v] = p.gamma ? (float)static_cast<const T*>(p.gamma)[c + v] : 1.0f;
      beta[v] = p.beta ? (float)static_cast<const T*>(p.beta)[c + v] : 0.0f;
    }
  }
};

// The two terms of rows b, b + rp, .. < e at V channels from c.
template <typename T, int V, bool BWD>
__device__ __forceinline__ void add_rows(const NormArgs& p, const Channels<T, V>& ch, int c, int b,
                                         int e, const float (&mean)[V], const float (&rstd)[V],
                                         double (&s0)[V], double (&s1)[V]) {
  for (int n0 = b; n0 < e; n0 += kU * p.rp) {
    float x[kU][V], d[kU][V];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int64_t n = min(n0 + u * p.rp, e - 1);
      load_cols<T, V>(static_cast<const T*>(p.x) + n * p.ldx + c, x[u]);
      if constexpr (BWD) load_cols<T, V>(static_cast<const T*>(p.dout) + n * p.F + c, d[u]);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (n0 + u * p.rp < e) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if constexpr (BWD) {
            const float xh = (x[u][v] - mean[v]) * rstd[v];
            const float dz = d[u][v] * act_slope(xh * ch.gamma[v] + ch.beta[v], p.act);
            s0[v] += (double)dz;
            s1[v] += (double)dz * (double)xh;
          } else {
            const double xd = (double)x[u][v];
            s0[v] += xd;
            s1[v] += xd * xd;
          }
        }
      }
  }
}

// One row's V channels of the output (or of dx).
template <typename T, int V, bool BWD>
__device__ __forceinline__ void apply_cols(const NormArgs& p, const Channels<T, V>& ch, int c,
                                           int64_t n, const float (&x)[V], const float (&d)[V],
                                           const float (&mean)[V], const float (&rstd)[V],
                                           const float (&ca)[V], const float (&cb)[V]) {
  float y[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float xh = (x[v] - mean[v]) * rstd[v];
    const float z = xh * ch.gamma[v] + ch.beta[v];
    if constexpr (BWD) {
      const float dh = d[v] * act_slope(z, p.act) * ch.gamma[v];
      y[v] = (dh - ca[v] - xh * cb[v]) * rstd[v];
    } else {
      y[v] = act_value(z, p.act);
    }
  }
  store_cols<T, V>(static_cast<T*>(BWD ? p.dx : p.out) + n * p.F + c, y);
}

template <typename T, int V, bool BWD>
__device__ __forceinline__ void apply_rows(const NormArgs& p, const Channels<T, V>& ch, int c, int64_t b,
                                           int64_t e, const float (&mean)[V], const float (&rstd)[V],
                                           const float (&ca)[V], const float (&cb)[V]) {
  for (int64_t n0 = b; n0 < e; n0 += kU * p.rp) {
    float x[kU][V], d[kU][V];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int64_t n = min(n0 + u * p.rp, e - 1);
      load_cols<T, V>(static_cast<const T*>(p.x) + n * p.ldx + c, x[u]);
      if constexpr (BWD) load_cols<T, V>(static_cast<const T*>(p.dout) + n * p.F + c, d[u]);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (n0 + u * p.rp < e)
        apply_cols<T, V, BWD>(p, ch, c, n0 + u * p.rp, x[u], d[u], mean, rstd, ca, cb);
  }
}

// One wavefront a graph (graphs wid, + waves, ..), all three steps; F <= 64 V. Its part of
// LDS: the lanes' sums ([term][column of the lane][lane]), the channels' totals, and the
// groups' statistics.
template <int V> struct WaveLds {
  double red[2][V][kWave];
  double tot[2][V * kWave];
  float st[2][V * kWave];  // per group: mean, rstd or the two means
};
template <typename T, int V, bool BWD, typename IdxT>
__global__ __launch_bounds__(kThreads) void norm_waves(NormArgs p, int waves) {
  __shared__ WaveLds<V> lds[kThreads / kWave];
  const int lane = lane_id(), wave = uniform((int)threadIdx.x / kWave);
  const int wid = blockIdx.x * (kThreads / kWave) + wave;
  if (wid >= waves) return;
  WaveLds<V>& w = lds[wave];
  const int lpr = p.lpr, rp = p.rp, r = lane / lpr, sub = lane - r * lpr, c = sub * V;
  const bool on = r < rp;
  Channels<T, V> ch;
  if (on) ch.load(p, c);
  // lanes of a group in the small step: a power of two, at most 64 / K
  int parts = kWave;
  while (parts > 1 && parts * p.K > kWave) parts >>= 1;
  double g0[V], g1[V];  // (backward: the first row's lanes' channels of dbeta, dgamma)
#pragma unroll
  for (int v = 0; v < V; ++v) g0[v] = g1[v] = 0.0;
  for (int g = wid; g < p.G; g += waves) {
    int b, e;
    graph_rows(static_cast<const IdxT*>(p.gi), p.Nb, g, &b, &e);
    if (b == e) {  // a graph without nodes
      if (!BWD)
        for (int k = lane; k < p.K; k += kWave)
          p.mean[(int64_t)g * p.K + k] = p.rstd[(int64_t)g * p.K + k] = 0.0f;
      continue;
    }
    float mean[V], rstd[V], ca[V], cb[V];
    double s0[V], s1[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      s0[v] = s1[v] = 0.0;
      mean[v] = rstd[v] = ca[v] = cb[v] = 0.0f;
      if (BWD && on) {
        mean[v] = p.mean[(int64_t)g * p.K + ch.k[v]];
        rstd[v] = p.rstd[(int64_t)g * p.K + ch.k[v]];
      }
    }
    if (on && b + r < e) add_rows<T, V, BWD>(p, ch, c, b + r, e, mean, rstd, s0, s1);
    wave_sync();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      w.red[0][v][lane] = s0[v];
      w.red[1][v][lane] = s1[v];
    }
    wave_sync();
    // the rows' lanes added up, (term, column) by (term, column)
    for (int i = lane; i < 2 * V * lpr; i += kWave) {
      const int tv = i / lpr, q = i - tv * lpr;
      const double* at = &w.red[0][0][0] + tv * kWave + q;
      double t = *at;
      for (int j = 1; j < rp; ++j) t += at[j * lpr];
      w.tot[tv / V][q * V + tv % V] = t;
    }
    wave_sync();
    const double cnt = (double)(e - b) * p.C;
    for (int k0 = 0; k0 < p.K; k0 += kWave / parts) {
      const int k = k0 + lane / parts;
      double t0 = 0.0, t1 = 0.0;
      if (k < p.K)
        for (int i = k * p.C + lane % parts; i < (k + 1) * p.C; i += parts) {
          const double f = BWD && p.gamma ? (double)(float)static_cast<const T*>(p.gamma)[i] : 1.0;
          t0 += f * w.tot[0][i];
          t1 += f * w.tot[1][i];
        }
      for (int o = 1; o < parts; o <<= 1) {
        t0 += __shfl_xor(t0, o);
        t1 += __shfl_xor(t1, o);
      }
      if (k >= p.K || lane % parts != 0) continue;
      if constexpr (BWD) {
        w.st[0][k] = (float)(t0 / cnt);
        w.st[1][k] = (float)(t1 / cnt);
      } else {
        const double m = t0 / cnt, var = fmax(t1 / cnt - m * m, 0.0);
        w.st[0][k] = p.mean[(int64_t)g * p.K + k] = (float)m;
        w.st[1][k] = p.rstd[(int64_t)g * p.K + k] = (float)(1.0 / sqrt(var + (double)p.eps));
      }
    }
    if (BWD && r == 0) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        g0[v] += w.tot[0][c + v];
        g1[v] += w.tot[1][c + v];
      }
    }
    wave_sync();
    if (on) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if constexpr (BWD) {
          ca[v] = w.st[0][ch.k[v]];
          cb[v] = w.st[1][ch.k[v]];
        } else {
          mean[v] = w.st[0][ch.k[v]];
          rstd[v] = w.st[1][ch.k[v]];
        }
      }
      apply_rows<T, V, BWD>(p, ch, c, b + r, e, mean, rstd, ca, cb);
    }
  }
  if (BWD && r == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      p.sums[((int64_t)wid * p.F + c + v) * 2] = g0[v];
      p.sums[((int64_t)wid * p.F + c + v) * 2 + 1] = g1[v];
    }
  }
}

// Sums of a block's rows per channel: [2][rp][lpr * V] doubles of LDS, the totals
// left in the first row of each half. Ends with a barrier.
template <int V>
__device__ __forceinline__ void reduce_rows(double* red, int lpr, int rp, int r, int sub,
                                            const double (&s0)[V], const double (&s1)[V]) {
  const int W = lpr * V;
  if (r < rp) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      red[r * W + v * lpr + sub] = s0[v];
      red[(rp + r) * W + v * lpr + sub] = s1[v];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * W; i += kThreads) {
    double* at = red + (i < W ? i : rp * W + i - W);
    double t = *at;
    for (int j = 1; j < rp; ++j) t += at[j * W];
    *at = t;
  }
  __syncthreads();
}

// Per-channel sums of one tile of rows (slots over the graphs, see spans.h).
template <typename T, int V, bool BWD>
__global__ __launch_bounds__(kThreads) void norm_sums(NormArgs p) {
  __shared__ double red[2 * kThreads * V];
  const int lpr = p.lpr, rp = p.rp, r = threadIdx.x / lpr, sub = threadIdx.x - r * lpr;
  const int c0 = blockIdx.y * lpr * V, c = c0 + sub * V;
  const bool on = r < rp && c < p.F;
  const Run t = find_run<kNormTile>(p.goff, p.G, p.Nb, 1, blockIdx.x);
  double s0[V], s1[V];
#pragma unroll
  for (int v = 0; v < V; ++v) s0[v] = s1[v] = 0.0;
  if (t.g >= 0 && on) {
    const int64_t b = clamp_off(p.goff[t.g], p.Nb) + (int64_t)t.tile * kNormTile;
    const int64_t e = min(b + kNormTile, (int64_t)clamp_off(p.goff[t.g + 1], p.Nb));
    Channels<T, V> ch;
    ch.load(p, c);
    float mean[V], rstd[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      mean[v] = BWD ? p.mean[(int64_t)t.g * p.K + ch.k[v]] : 0.0f;
      rstd[v] = BWD ? p.rstd[(int64_t)t.g * p.K + ch.k[v]] : 0.0f;
    }
    if (b + r < e) add_rows<T, V, BWD>(p, ch, c, (int)b + r, (int)e, mean, rstd, s0, s1);
  }
  reduce_rows<V>(red, lpr, rp, r, sub, s0, s1);
  // channel c0 + i lies at place (i % V) * lpr + i / V
  const int W = min(lpr * V, p.F - c0);
  const auto total = [&](int i, int term) { return red[term * rp * lpr * V + (i % V) * lpr + i / V]; };
  if (p.sums != nullptr)
    for (int i = threadIdx.x; i < W; i += kThreads) {
      double* at = p.sums + ((int64_t)blockIdx.x * p.F + c0 + i) * 2;
      at[0] = total(i, 0);
      at[1] = total(i, 1);
    }
  // groups that begin in this slab, or the slab's part of a wider one
  const int k0 = c0 / p.C, k1 = (c0 + W - 1) / p.C;
  for (int k = k0 + threadIdx.x; k <= k1; k += kThreads) {
    double t0 = 0.0, t1 = 0.0;
    for (int i = max(k * p.C - c0, 0); i < min((k + 1) * p.C - c0, W); ++i) {
      const double f = BWD && p.gamma ? (double)(float)static_cast<const T*>(p.gamma)[c0 + i] : 1.0;
      t0 += f * total(i, 0);
      t1 += f * total(i, 1);
    }
    double* at = p.groups + ((int64_t)blockIdx.x * (p.K + p.slabs) + k + blockIdx.y) * 2;
    at[0] = t0;
    at[1] = t1;
  }
}

// The tiles' sums of one (graph, group) joined: mean and rstd, or the backward's two means.
template <bool BWD>
__global__ __launch_bounds__(kThreads) void norm_stats(NormArgs p) {
  __shared__ double part[2][kThreads];
  const int g = blockIdx.x / p.K, k = blockIdx.x % p.K;
  const int b = clamp_off(p.goff[g], p.Nb), n = max(clamp_off(p.goff[g + 1], p.Nb) - b, 0);
  const int64_t first = first_slot<kNormTile>(p.goff, g, p.Nb, 1);
  // slabs whose columns hold a part of the group
  const int s0 = k * p.C / p.slab, s1 = ((k + 1) * p.C - 1) / p.slab + 1, ns = s1 - s0;
  const int items = (n + kNormTile - 1) / kNormTile * ns;
  double t0 = 0.0, t1 = 0.0;
  for (int i = threadIdx.x; i < items; i += kThreads) {
    const int tile = ns == 1 ? i : i / ns;
    const double* at = p.groups + ((first + tile) * (p.K + p.slabs) + k + s0 + (i - tile * ns)) * 2;
    t0 += at[0];
    t1 += at[1];
  }
  part[0][threadIdx.x] = t0;
  part[1][threadIdx.x] = t1;
  for (int h = kThreads / 2; h > 0; h >>= 1) {
    __syncthreads();
    if ((int)threadIdx.x < h) {
      part[0][threadIdx.x] += part[0][threadIdx.x + h];
      part[1][threadIdx.x] += part[1][threadIdx.x + h];
    }
  }
  if (threadIdx.x != 0) return;
  const double cnt = (double)n * p.C;
  const int64_t at = (int64_t)g * p.K + k;
  if constexpr (BWD) {
    p.coef[2 * at] = n > 0 ? (float)(part[0][0] / cnt) : 0.0f;
    p.coef[2 * at + 1] = n > 0 ? (float)(part[1][0] / cnt) : 0.0f;
  } else {
    const double m = n > 0 ? part[0][0] / cnt : 0.0;
    const double var = n > 0 ? fmax(part[1][0] / cnt - m * m, 0.0) : 0.0;
    p.mean[at] = (float)m;
    p.rstd[at] = n > 0 ? (float)(1.0 / sqrt(var + (double)p.eps)) : 0.0f;
  }
}

// The last pass over tiles: every row by its graph.
template <typename T, int V, bool BWD>
__global__ __launch_bounds__(kThreads) void norm_apply(NormArgs p) {
  const int lpr = p.lpr, rp = p.rp, r = threadIdx.x / lpr, sub = threadIdx.x - r * lpr;
  const int c = blockIdx.y * lpr * V + sub * V;
  const Run t = find_run<kNormTile>(p.goff, p.G, p.Nb, 1, blockIdx.x);
  if (t.g < 0 || r >= rp || c >= p.F) return;
  const int64_t b = clamp_off(p.goff[t.g], p.Nb) + (int64_t)t.tile * kNormTile;
  const int64_t e = min(b + kNormTile, (int64_t)clamp_off(p.goff[t.g + 1], p.Nb));
  Channels<T, V> ch;
  ch.load(p, c);
  float mean[V], rstd[V], ca[V], cb[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t at = (int64_t)t.g * p.K + ch.k[v];
    mean[v] = p.mean[at];
    rstd[v] = p.rstd[at];
    ca[v] = BWD ? p.coef[2 * at] : 0.0f;
    cb[v] = BWD ? p.coef[2 * at + 1] : 0.0f;
  }
  apply_rows<T, V, BWD>(p, ch, c, b + r, e, mean, rstd, ca, cb);
}

// dbeta and dgamma: the first sums' groups [groups][F][2] added in order, rounded once.
template <typename T>
__global__ __launch_bounds__(kWave) void norm_params(const double* __restrict__ sums, int groups, int F,
                                                     T* __restrict__ dgamma, T* __restrict__ dbeta) {
  const int i = blockIdx.x * kWave + threadIdx.x, c = i / 2;
  if (c >= F) return;
  double acc[16] = {};
  for (int r = 0; r < groups; r += 16) {
    double x[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) x[u] = sums[((int64_t)min(r + u, groups - 1) * F + c) * 2 + i % 2];
#pragma unroll
    for (int u = 0; u < 16; ++u) acc[u] += r + u < groups ? x[u] : 0.0;
  }
  T* to = i % 2 ? dgamma : dbeta;
#pragma unroll
  for (int h = 8; h > 0; h >>= 1)
#pragma unroll
    for (int u = 0; u < h; ++u) acc[u] += acc[u + h];
  if (to != nullptr) to[c] = (T)acc[0];
}

constexpr int kNormWaves = 4096;  // wavefronts over graphs: sixteen a CU
constexpr int kRowsOfGraph = 128;

// Columns a lane of norm_waves takes (0: not by graph): graphs are small on average, and
// a row fits a wavefront.
int by_graph(int64_t Nb, int64_t F, int64_t G, bool vectors) {
  if (Nb > kRowsOfGraph * G) return 0;
  if (vectors && F <= 4 * kWave) return 4;
  return F <= kWave ? 1 : 0;
}

struct NormLayout {
  size_t goff, err, sums, groups, coef, cols, total;
  int64_t rows;  // of sums, at most
};
// For any way that the width may take.
NormLayout norm_layout(int64_t Nb, int64_t F, int64_t G, int64_t K, bool bwd) {
  NormLayout L;
  const int64_t tiles = Nb / kNormTile + G, waves = std::min<int64_t>(G, kNormWaves);
  const bool only_graphs = by_graph(Nb, F, G, false) == 1;
  const int64_t slabs = (F + kThreads - 1) / kThreads;  // at one column a lane
  L.rows = only_graphs ? waves : std::max(tiles, waves);
  L.goff = 0;
  L.err = align_up(sizeof(int) * (size_t)(G + 1), 256);
  L.sums = L.err + 256;
  L.groups = L.sums + (bwd ? align_up(2 * sizeof(double) * (size_t)(L.rows * F), 256) : 0);
  L.coef = L.groups + (only_graphs ? 0 : align_up(2 * sizeof(double) * (size_t)(tiles * (K + slabs)), 256));
  L.cols = L.coef + (bwd && !only_graphs ? align_up(2 * sizeof(float) * (size_t)(G * K), 256) : 0);
  L.total = L.cols + (bwd ? align_up(column_sums_bytes(L.rows, 2 * F), 256) : 0);
  return L;
}

// Launches both ways; *rows: rows of partial parameter sums.
template <typename T, int V, bool BWD>
int launch_norm_cols(NormArgs& p, int index_type, int64_t* rows, hipStream_t s) {
  const int lanes = p.F / V;
  if (V <= 4 && by_graph(p.Nb, p.F, p.G, V == 4) == V) {
    const int waves = std::min(p.G, kNormWaves);
    const unsigned nb = (unsigned)((waves + 3) / 4);
    p.lpr = lanes;
    p.rp = kWave / lanes;
    *rows = waves;
    constexpr int W = V == 8 ? 4 : V;  // (never launched with eight columns)
    if (index_type == TFG_I64) norm_waves<T, W, BWD, int64_t><<<nb, kThreads, 0, s>>>(p, waves);
    else norm_waves<T, W, BWD, int32_t><<<nb, kThreads, 0, s>>>(p, waves);
    TFG_LAUNCHED("norm_waves");
    return TFG_OK;
  }
  p.lpr = std::min(lanes, kThreads);
  p.rp = kThreads / p.lpr;
  p.slab = p.lpr * V;
  p.slabs = (lanes + p.lpr - 1) / p.lpr;
  const int64_t tiles = p.Nb / kNormTile + p.G;
  *rows = tiles;
  const dim3 grid((unsigned)tiles, (unsigned)p.slabs);
  norm_sums<T, V, BWD><<<grid, kThreads, 0, s>>>(p);
  norm_stats<BWD><<<(unsigned)(p.G * p.K), kThreads, 0, s>>>(p);
  norm_apply<T, V, BWD><<<grid, kThreads, 0, s>>>(p);
  TFG_LAUNCHED("norm_apply");
  return TFG_OK;
}

template <typename T, bool BWD>
int launch_norm_type(NormArgs& p, const GroupNorm& n, int* goff, int* err, int64_t* rows, hipStream_t s) {
  const bool four = p.F % 4 == 0;
  const int way = by_graph(p.Nb, p.F, p.G, four);
  if (way == 0 || err != nullptr)
    if (int rc = launch_segment_bounds(n.graph_index, n.index_type, n.Nb, n.G, goff, err, s)) return rc;
  if constexpr (sizeof(T) == 2)
    if (way == 0 && p.F % 8 == 0) return launch_norm_cols<T, 8, BWD>(p, n.index_type, rows, s);
  if (four) return launch_norm_cols<T, 4, BWD>(p, n.index_type, rows, s);
  return launch_norm_cols<T, 1, BWD>(p, n.index_type, rows, s);
}

template <typename T>
int launch_param_grads(const NormArgs& p, int64_t rows, double* ws, void* dgamma, void* dbeta, hipStream_t s) {
  const int64_t groups = column_groups(rows), per = (rows + groups - 1) / groups;
  const int n = 2 * p.F;
  const unsigned nb = (unsigned)((n + kWave - 1) / kWave);
  column_sums<double, double><<<dim3(nb, (unsigned)groups), kWave * kSumLanes, 0, s>>>(p.sums, rows, n, per, ws);
  norm_params<T><<<nb, kWave, 0, s>>>(ws, (int)groups, p.F, static_cast<T*>(dgamma), static_cast<T*>(dbeta));
  TFG_LAUNCHED("norm_params");
  return TFG_OK;
}

}  // namespace

size_t group_norm_ws_bytes(int64_t Nb, int64_t F, int64_t G, int64_t K, bool bwd) {
  return norm_layout(Nb, F, G, K, bwd).total;
}

int* group_norm_flag(int64_t G, void* ws) {
  return reinterpret_cast<int*>(static_cast<char*>(ws) + align_up(sizeof(int) * (size_t)(G + 1), 256));
}

int launch_group_norm(const GroupNorm& n, bool bwd, void* ws, int* err, hipStream_t s) {
  const NormLayout L = norm_layout(n.Nb, n.F, n.G, n.K, bwd);
  char* w = static_cast<char*>(ws);
  int* goff = reinterpret_cast<int*>(w + L.goff);
  if (err != nullptr) {
    if (int rc = launch_zero_flag(err, s)) return rc;
  }
  NormArgs p{};
  p.x = n.x;
  p.gi = n.graph_index;
  p.gamma = n.gamma;
  p.beta = n.beta;
  p.dout = n.dout;
  p.out = n.out;
  p.dx = n.dx;
  p.mean = n.mean;
  p.rstd = n.rstd;
  p.goff = goff;
  p.ldx = n.ldx;
  p.Nb = (int)n.Nb;
  p.G = (int)n.G;
  p.F = (int)n.F;
  p.K = (int)n.K;
  p.C = (int)(n.F / n.K);
  p.act = n.act;
  p.eps = n.eps;
  p.sums = bwd ? reinterpret_cast<double*>(w + L.sums) : nullptr;
  p.groups = reinterpret_cast<double*>(w + L.groups);
  p.coef = reinterpret_cast<float*>(w + L.coef);
  int64_t rows = 0;
  if (n.G > 0) {
    int rc;
    if (n.float_type == TFG_BF16)
      rc = bwd ? launch_norm_type<__bf16, true>(p, n, goff, err, &rows, s)
               : launch_norm_type<__bf16, false>(p, n, goff, err, &rows, s);
    else
      rc = bwd ? launch_norm_type<float, true>(p, n, goff, err, &rows, s)
               : launch_norm_type<float, false>(p, n, goff, err, &rows, s);
    if (rc) return rc;
  }
  if (!bwd || (n.dgamma == nullptr && n.dbeta == nullptr)) return TFG_OK;
  double* cols = reinterpret_cast<double*>(w + L.cols);
  return n.float_type == TFG_BF16 ? launch_param_grads<__bf16>(p, rows, cols, n.dgamma, n.dbeta, s)
                                  : launch_param_grads<float>(p, rows, cols, n.dgamma, n.dbeta, s);
}

}  // namespace tfg
