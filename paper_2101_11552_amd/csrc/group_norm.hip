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
// Small graphs take one block each for all three steps (their rows are read again
// from the caches); larger ones are cut into tiles of rows.
#include "columns.h"
#include "rows.h"
#include "spans.h"

namespace tfg {

namespace {

constexpr int kThreads = 256;
constexpr int kNormTile = 128;  // rows of a tile
constexpr int kU = 4;           // rows in flight per thread

struct NormArgs {
  const void *x, *gi, *gamma, *beta, *dout;
  void *out, *dx;
  float *mean, *rstd;   // [G, K]
  const int* goff;      // [G + 1] (tiles)
  double* sums;         // [slots or blocks][F][2]
  float* coef;          // [G, K][2] (backward, tiles)
  int64_t ldx;
  int Nb, G, F, K, C, act;
  int lpr, rp;          // lanes a row, rows a block and step
  float eps;
};

// act(z) and act'(z).
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == TFG_ACT_RELU) return z > 0.0f ? z : (z == z ? 0.0f : z);
  if (act == TFG_ACT_SILU) return z / (1.0f + expf(-z));
  if (act == TFG_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752440f));
  return z;
}
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == TFG_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
  if (act == TFG_ACT_SILU) {
    const float s = 1.0f / (1.0f + expf(-z));
    return s * (1.0f + z * (1.0f - s));
  }
  if (act == TFG_ACT_GELU)
    return 0.5f * (1.0f + erff(z * 0.70710678118654752440f)) +
           z * expf(-0.5f * z * z) * 0.39894228040143267794f;
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

// Sums of a block's rows per channel: [2][rp][lpr * V] doubles of LDS, the totals
// left in the first row of each half. Ends with a barrier.
template <int V>
__device__ __forceinline__ void reduce_rows(double* red, int lpr, int rp, int r, int sub,
                                            const double (&s0)[V], const double (&s1)[V]) {
  const int W = lpr * V;
  if (r < rp) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      red[r * W + sub * V + v] = s0[v];
      red[(rp + r) * W + sub * V + v] = s1[v];
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

// One block a graph (graphs blockIdx.x, + gridDim.x, ..): all three steps.
template <typename T, int V, bool BWD, typename IdxT>
__global__ __launch_bounds__(kThreads) void norm_graph(NormArgs p) {
  __shared__ double red[2 * kThreads * V];
  __shared__ float st[2][kThreads];  // per group (K <= F <= kThreads): mean, rstd or the two means
  const int lpr = p.lpr, rp = p.rp, r = threadIdx.x / lpr, sub = threadIdx.x - r * lpr;
  const int c = sub * V;
  const bool on = r < rp;
  const int W = lpr * V;
  Channels<T, V> ch;
  if (on) ch.load(p, c);
  double g0[V], g1[V];  // (backward: this thread's channels of dbeta, dgamma)
#pragma unroll
  for (int v = 0; v < V; ++v) g0[v] = g1[v] = 0.0;
  for (int g = blockIdx.x; g < p.G; g += gridDim.x) {
    int b, e;
    graph_rows(static_cast<const IdxT*>(p.gi), p.Nb, g, &b, &e);
    if (b == e) {  // a graph without nodes
      if (!BWD)
        for (int k = threadIdx.x; k < p.K; k += kThreads)
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
    if (on) add_rows<T, V, BWD>(p, ch, c, b + r, e, mean, rstd, s0, s1);
    reduce_rows<V>(red, lpr, rp, r, sub, s0, s1);
    const double cnt = (double)(e - b) * p.C;
    for (int k = threadIdx.x; k < p.K; k += kThreads) {
      double t0 = 0.0, t1 = 0.0;
      for (int i = k * p.C; i < (k + 1) * p.C; ++i) {
        const double w = BWD && p.gamma ? (double)(float)static_cast<const T*>(p.gamma)[i] : 1.0;
        t0 += w * red[i];
        t1 += w * red[rp * W + i];
      }
      if constexpr (BWD) {
        st[0][k] = (float)(t0 / cnt);
        st[1][k] = (float)(t1 / cnt);
      } else {
        const double m = t0 / cnt, var = fmax(t1 / cnt - m * m, 0.0);
        const float mf = (float)m, rf = (float)(1.0 / sqrt(var + (double)p.eps));
        st[0][k] = p.mean[(int64_t)g * p.K + k] = mf;
        st[1][k] = p.rstd[(int64_t)g * p.K + k] = rf;
      }
    }
    if (BWD && r == 0) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        g0[v] += red[c + v];
        g1[v] += red[rp * W + c + v];
      }
    }
    __syncthreads();
    if (on) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if constexpr (BWD) {
          ca[v] = st[0][ch.k[v]];
          cb[v] = st[1][ch.k[v]];
        } else {
          mean[v] = st[0][ch.k[v]];
          rstd[v] = st[1][ch.k[v]];
        }
      }
      for (int n0 = b + r; n0 < e; n0 += kU * rp) {
        float x[kU][V], d[kU][V];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int64_t n = min(n0 + u * rp, e - 1);
          load_cols<T, V>(static_cast<const T*>(p.x) + n * p.ldx + c, x[u]);
          if constexpr (BWD) load_cols<T, V>(static_cast<const T*>(p.dout) + n * p.F + c, d[u]);
        }
#pragma unroll
        for (int u = 0; u < kU; ++u)
          if (n0 + u * rp < e)
            apply_cols<T, V, BWD>(p, ch, c, n0 + u * rp, x[u], d[u], mean, rstd, ca, cb);
      }
    }
    __syncthreads();  // st and red are written again
  }
  if (BWD && p.sums != nullptr && r == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      p.sums[((int64_t)blockIdx.x * p.F + c + v) * 2] = g0[v];
      p.sums[((int64_t)blockIdx.x * p.F + c + v) * 2 + 1] = g1[v];
    }
  }
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
  const int W = lpr * V;
  for (int i = threadIdx.x; i < W && c0 + i < p.F; i += kThreads) {
    double* at = p.sums + ((int64_t)blockIdx.x * p.F + c0 + i) * 2;
    at[0] = red[i];
    at[1] = red[rp * W + i];
  }
}

// The tiles' sums of one (graph, group) joined: mean and rstd, or the backward's two means.
template <typename T, bool BWD>
__global__ __launch_bounds__(kThreads) void norm_stats(NormArgs p) {
  __shared__ double part[2][kThreads];
  const int g = blockIdx.x / p.K, k = blockIdx.x % p.K;
  const int b = clamp_off(p.goff[g], p.Nb), n = max(clamp_off(p.goff[g + 1], p.Nb) - b, 0);
  const int64_t first = first_slot<kNormTile>(p.goff, g, p.Nb, 1);
  const int64_t items = (int64_t)((n + kNormTile - 1) / kNormTile) * p.C;
  double t0 = 0.0, t1 = 0.0;
  for (int64_t i = threadIdx.x; i < items; i += kThreads) {
    const int64_t tile = i / p.C;
    const int c = k * p.C + (int)(i - tile * p.C);
    const double* at = p.sums + ((first + tile) * p.F + c) * 2;
    const double w = BWD && p.gamma ? (double)(float)static_cast<const T*>(p.gamma)[c] : 1.0;
    t0 += w * at[0];
    t1 += w * at[1];
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
  for (int64_t n0 = b + r; n0 < e; n0 += kU * rp) {
    float x[kU][V], d[kU][V];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int64_t n = min(n0 + u * rp, e - 1);
      load_cols<T, V>(static_cast<const T*>(p.x) + n * p.ldx + c, x[u]);
      if constexpr (BWD) load_cols<T, V>(static_cast<const T*>(p.dout) + n * p.F + c, d[u]);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (n0 + u * rp < e)
        apply_cols<T, V, BWD>(p, ch, c, n0 + u * rp, x[u], d[u], mean, rstd, ca, cb);
  }
}

// dbeta and dgamma: [F][2] doubles rounded once.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_params(const double* __restrict__ sums, int F,
                                                        T* __restrict__ dgamma, T* __restrict__ dbeta) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= F) return;
  if (dbeta) dbeta[c] = (T)sums[2 * c];
  if (dgamma) dgamma[c] = (T)sums[2 * c + 1];
}

constexpr int kGraphBlocks = 2048;  // blocks over graphs: eight a CU

// One block a graph where graphs are small and a row fits a block.
bool by_graph(int64_t Nb, int64_t F, int64_t G) {
  return Nb <= 256 * G && F <= kThreads;
}

struct NormLayout {
  size_t goff, err, sums, coef, cols, total;
  int64_t rows;  // of sums
};
NormLayout norm_layout(int64_t Nb, int64_t F, int64_t G, int64_t K, bool bwd) {
  NormLayout L;
  const bool small = by_graph(Nb, F, G);
  L.rows = small ? std::min<int64_t>(G, kGraphBlocks) : Nb / kNormTile + G;
  L.goff = 0;
  L.err = align_up(sizeof(int) * (size_t)(G + 1), 256);
  L.sums = L.err + 256;
  L.coef = L.sums + (bwd || !small ? align_up(2 * sizeof(double) * (size_t)(L.rows * F), 256) : 0);
  L.cols = L.coef + (bwd && !small ? align_up(2 * sizeof(float) * (size_t)(G * K), 256) : 0);
  L.total = L.cols + (bwd ? align_up(column_sums_bytes(L.rows, 2 * F), 256) +
                                align_up(2 * sizeof(double) * (size_t)F, 256) : 0);
  return L;
}

template <typename T, int V, bool BWD>
int launch_norm_cols(NormArgs& p, const NormLayout& L, bool small, int index_type, hipStream_t s) {
  const int lanes = p.F / V;
  p.lpr = std::min(lanes, kThreads);
  p.rp = kThreads / p.lpr;
  if (small) {
    const unsigned nb = (unsigned)std::min(p.G, kGraphBlocks);
    if (index_type == TFG_I64) norm_graph<T, V, BWD, int64_t><<<nb, kThreads, 0, s>>>(p);
    else norm_graph<T, V, BWD, int32_t><<<nb, kThreads, 0, s>>>(p);
    TFG_LAUNCHED("norm_graph");
    return TFG_OK;
  }
  const dim3 grid((unsigned)L.rows, (unsigned)((lanes + p.lpr - 1) / p.lpr));
  if ((int64_t)p.G * p.K >= (int64_t(1) << 31)) return fail(TFG_ERR_TOO_LARGE, "G * groups not below 2^31");
  norm_sums<T, V, BWD><<<grid, kThreads, 0, s>>>(p);
  norm_stats<T, BWD><<<(unsigned)(p.G * p.K), kThreads, 0, s>>>(p);
  norm_apply<T, V, BWD><<<grid, kThreads, 0, s>>>(p);
  TFG_LAUNCHED("norm_apply");
  return TFG_OK;
}

template <typename T, bool BWD>
int launch_norm_type(NormArgs& p, const NormLayout& L, bool small, int index_type, hipStream_t s) {
  const auto fit = [&](int v) {
    return cols_fit<T>(v, p.x, p.ldx, p.F) &&
           (BWD ? cols_fit<T>(v, p.dout, p.F, p.F) && cols_fit<T>(v, p.dx, p.F, p.F)
                : cols_fit<T>(v, p.out, p.F, p.F));
  };
  if constexpr (sizeof(T) == 2)
    if (fit(8)) return launch_norm_cols<T, 8, BWD>(p, L, small, index_type, s);
  if (fit(4)) return launch_norm_cols<T, 4, BWD>(p, L, small, index_type, s);
  return launch_norm_cols<T, 1, BWD>(p, L, small, index_type, s);
}

template <typename T>
int launch_param_grads(const NormArgs& p, const NormLayout& L, char* ws, void* dgamma, void* dbeta,
                       hipStream_t s) {
  double* cols = reinterpret_cast<double*>(ws + L.cols);
  double* fin = reinterpret_cast<double*>(ws + L.cols + align_up(column_sums_bytes(L.rows, 2 * p.F), 256));
  if (int rc = launch_column_sums(p.sums, p.G == 0 ? 0 : L.rows, 2 * p.F, fin, cols, s)) return rc;
  norm_params<T><<<(unsigned)((p.F + kThreads - 1) / kThreads), kThreads, 0, s>>>(
      fin, p.F, static_cast<T*>(dgamma), static_cast<T*>(dbeta));
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
  const bool small = by_graph(n.Nb, n.F, n.G);
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
  const bool params = bwd && (n.dgamma != nullptr || n.dbeta != nullptr);
  if (bwd || !small) p.sums = reinterpret_cast<double*>(w + L.sums);
  if (bwd && !small) p.coef = reinterpret_cast<float*>(w + L.coef);
  int rc = TFG_OK;
  if (n.G > 0) {
    if (!small || err != nullptr)
      rc = launch_segment_bounds(n.graph_index, n.index_type, n.Nb, n.G, goff, err, s);
    if (rc) return rc;
    if (n.float_type == TFG_BF16)
      rc = bwd ? launch_norm_type<__bf16, true>(p, L, small, n.index_type, s)
               : launch_norm_type<__bf16, false>(p, L, small, n.index_type, s);
    else
      rc = bwd ? launch_norm_type<float, true>(p, L, small, n.index_type, s)
               : launch_norm_type<float, false>(p, L, small, n.index_type, s);
    if (rc) return rc;
  }
  if (!params) return TFG_OK;
  return n.float_type == TFG_BF16 ? launch_param_grads<__bf16>(p, L, w, n.dgamma, n.dbeta, s)
                                  : launch_param_grads<float>(p, L, w, n.dgamma, n.dbeta, s);
}

}  // namespace tfg
