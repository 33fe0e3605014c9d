// Gradients of the attention inside each graph of a BatchGraph (gfx950), the
// kernels, compiled per type and width in attention_grad_bf16_narrow.hip and its like.
//
// With p = exp(u - lse) formed again from the forward's log-sum and
// delta[row] = <dout[row], out[row]> (= the sum of p dp over the keys):
//   dv = p^T dout;  dp = dout v^T;  du = p (dp - delta);
//   dbias[head, b] = sum of du over the pairs of bucket b;
//   ds = du (1 - tanh^2) (capped scores);  dq = scale ds k;  dk = scale ds^T q
// Two passes, each of which owns its outputs (no float atomics between lanes, a
// fixed order of every sum): attn_grad_q over tiles of rows (delta, dq and the
// bias), then attn_grad_kv over tiles of keys (dk, dv), over the queries of all
// heads that share the key/value head. Scores and dp are formed in both: seven
// products instead of five, and no partial dq in memory.
//
// delta from a bf16 output carries that output's rounding, which short rows feel
// (a node's weights are large there): up to 128 keys it is summed from p
// and dp in a first sweep instead. The same sweep serves rows whose log-sum is so
// large (a bias of the type's lowest value) that u - lse has lost the sum: it keeps
// the maximum and the sum apart.
//
// What bounds it: the latency of LDS reads, table look-ups and exponentials at two
// wavefronts a SIMD, whose registers hold a tile's rows, sums and prefetched rows; no unit is
// saturated. bf16, two graphs of 3,000 nodes, 8 heads of 128 on 2, capped, with a bias: 405 us
// over rows (the bias's bins some 100 of them), 488 over keys, 170 TFLOP/s (the vector ALUs
// busy for 129 us, the LDS for 141, the matrix cores for 37 of the first). float32, 4 graphs of
// 1,500, 8 heads of 64: 765 us, 84 TFLOP/s of a large product's 153.
#pragma once

#include "attention.h"
#include "columns.h"

namespace tfg {

struct AttnGrad {
  AttnShape a;
  const void *q, *k, *v, *out, *dout;
  const float* lse;
  void *dq, *dk, *dv;
  // per (query, head): p = exp2((u - row_a) * log2(e) + row_c) with a bias, else
  // exp2(u in base 2 - row_a); +inf: a row without unmasked keys
  float *row_a, *row_c, *row_delta;
  float* bias_part;  // [slots][H * B] partial bias gradients, or NULL
  int vec_q, vec_k, vec_v, vec_o, vec_do, vec_dq, vec_dk, vec_dv;
  int copies;        // bias bins a wavefront keeps: one, or one a query tile
  int small;         // graphs of at most so many queries and keys are another launch's
  int heads;         // key/value heads a block takes
  int nsplit;        // > 1: the queries of a key tile in that many parts, joined afterwards
  float* part;       // [nsplit][2][Nk * Hk * D] partial dk (without scale), dv
};

// Beyond this log-sum its rounding (2^-24 of it) is felt in exp(u - lse).
constexpr float kLongLse = 4096.0f;

struct ScoreScale {
  float scale, to_tanh, to_exp, cap;
  float add;   // the score's addend without a bias
  float unit;  // from what score() gives to base 2
};
template <typename T, bool BIAS, bool CAP>
__device__ __forceinline__ ScoreScale score_scale(const AttnShape& a) {
  ScoreScale c;
  c.scale = a.scale;
  c.to_tanh = CAP ? a.scale / a.cap : 0.0f;
  c.to_exp = c.to_tanh * (2.0f * kLog2e);
  c.cap = a.cap;
  c.add = CAP ? cap_offset<T>(a.cap) : 0.0f;
  c.unit = BIAS || CAP ? kLog2e : a.scale * kLog2e;
  return c;
}
// A raw product as a score (natural units with a bias or a cap, the product itself
// without).
template <typename T, bool BIAS, bool CAP>
__device__ __forceinline__ float score(float x, float add, const ScoreScale& c) {
  float u = x;
  if constexpr (CAP) u = capped<T>(x, c.to_tanh, c.to_exp, c.cap, add);
  else if constexpr (BIAS) u = __builtin_fmaf(x, c.scale, add);
  return u;
}
// The cap's derivative 1 - tanh^2 there. bf16: 4 r (1 - r), r = 1 / (1 + exp(2 x)).
template <typename T, bool CAP>
__device__ __forceinline__ float cap_slope(float x, const ScoreScale& c) {
  if constexpr (!CAP) return 1.0f;
  if constexpr (sizeof(T) == 4) {
    const float t = capped<T>(x, c.to_tanh, c.to_exp, 1.0f, 0.0f);
    return __builtin_fmaf(-t, t, 1.0f);
  } else {
    const float r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * c.to_exp));
    return 4.0f * __builtin_fmaf(-r, r, r);
  }
}
template <bool BIAS>
__device__ __forceinline__ float weight(float u, float unit, float ra, float rc) {
  if constexpr (BIAS) return __builtin_amdgcn_exp2f(__builtin_fmaf(u - ra, unit, rc));
  return __builtin_amdgcn_exp2f(__builtin_fmaf(u, unit, -ra));
}

// Four values to a lane's own bins (a column of LDS), in order: all four are read, each is
// added to what the one before it in the same bin has left, and the last write stays.
// (LDS additions of floats, ds_add_f32, take some 150 cycles a wavefront here.)
__device__ __forceinline__ void add_to_bins(float* bin, const unsigned (&b)[4], f32x4 v) {
  float r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = bin[b[i] * kWave];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int j = 0; j < i; ++j) r[i] = b[j] == b[i] ? r[j] : r[i];
    r[i] += v[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) bin[b[i] * kWave] = r[i];
}

// Two wavefronts a SIMD where one tile each leaves registers for them.
template <typename T, int DP, int TILES> constexpr int grad_waves() {
  return TILES == 1 && DP * sizeof(T) <= 256 ? 2 : 1;
}

// Whether the row tiles' chunks change places (see Tile): in wider heads, and for the
// column tiles, the addresses' registers cost more than the conflicts (4 graphs of 1,500, 8
// heads on 4, bf16, no bias: 97 -> 91 us at width 16, 103 -> 99 at 32, but 198 -> 213 at 64;
// column tiles too, width 32 with a bias: 170 -> 218, a wavefront a SIMD less).
template <typename T, int DP> constexpr bool swapped_chunks() { return sizeof(T) == 2 && DP <= 32; }

// bf16 heads of up to 32 columns: ds as two operands, its rounding and what that left over.
// A row's ds add up to zero, so its dq is what few terms leave of larger ones: with ds
// rounded once and delta from the rounded output, dq of width 8 was off by 2.7e-3 of its
// norm (of wide heads 2.4e-3, of its own rounding alone 1.7e-3). One product more: 160 ->
// 164 us with a bias, 4 graphs of 1,500, 8 heads on 4.
template <typename T, int DP> constexpr bool splits_ds() { return sizeof(T) == 2 && DP <= 32; }

// Operands in registers: the last products' column operands are read from LDS one step
// ahead in bf16, where the compiler would wait for each pair (4 graphs of 1,500, 8 heads on
// 4 of width 64, capped: 220 -> 174 us; of 128 with a bias 496 -> 486). float32's products
// take longer than a read, and its operands twice the registers.
template <typename T> constexpr int operands_ahead() { return sizeof(T) == 2 ? 2 : 1; }

template <typename T, int DP, int WAVES, int QT, int VEC, bool BIAS, bool CAP, bool REST>
__global__ __launch_bounds__(WAVES * kWave, (grad_waves<T, DP, QT>())) void attn_grad_q(AttnGrad p) {
  // keys of a tile: as many as leave LDS for two blocks a CU beside the bias's bins
  // (width 128, two graphs of 3,000 nodes, 8 heads on 2: 408 us with tiles of 32 keys, 493
  // with 64; without a bias or a cap the whole gradient takes 566 us with 64, 652 with 32)
  constexpr int BM = WAVES * QT * 16, BN = sizeof(T) == 2 && !(BIAS && DP == 128) ? 64 : 32;
  constexpr int THREADS = WAVES * kWave;
  constexpr int NB = operands_ahead<T>();
  constexpr bool SPLIT = splits_ds<T, DP>();
  using Rows = Tile<T, DP, swapped_chunks<T, DP>()>;
  using Columns = Tile<T, BN, false>;
  constexpr int KC = Frag<T, DP>::KC, DT = DP / 16, KT = BN / 16;
  using U = Units<BN, DP>;
  // staging units of a thread: four rows of eight columns (K), rows of eight (V)
  constexpr int KU = (BN / 4 * (DP / 8) + THREADS - 1) / THREADS;
  constexpr int VU = (BN * (DP / 8) + THREADS - 1) / THREADS;
  constexpr bool AHEAD = VEC == 8 && (KU * 32 + VU * 8) * sizeof(T) / 4 <= 48;
  __shared__ T Ks[BN * Rows::LD];
  __shared__ T Vs[BN * Rows::LD];
  __shared__ T Kt[DP * Columns::LD];
  extern __shared__ float tab[];
  const AttnShape& a = p.a;
  const int grp = a.H / a.Hk, D = a.D;
  const int per_slot = (a.Hk + p.heads - 1) / p.heads;
  const int slot = (int)(blockIdx.x / per_slot);
  const int kvh0 = (int)(blockIdx.x % per_slot) * p.heads;
  const int kvh1 = min(kvh0 + p.heads, a.Hk);
  const bool want_bias = BIAS && p.bias_part != nullptr;
  float* bins = tab + grp * (a.B + 1);  // [WAVES][copies][B + 1][64], one column a lane
  float* bpart = want_bias ? p.bias_part + (int64_t)slot * a.H * a.B : nullptr;
  const auto no_bias = [&]() {
    for (int i = threadIdx.x; i < (kvh1 - kvh0) * grp * a.B; i += THREADS) bpart[kvh0 * grp * a.B + i] = 0.0f;
  };
  RestScan scan;
  if (REST) {
    if (want_bias) no_bias();  // (the rest's tiles add to their block's row)
    if (!any_rest(a, p.small)) return;
  }
  for (int index = slot;; index += kRestBlocks) {
    const Span s = REST ? next_span<BM, false>(a, grp, p.small, index, scan)
                        : find_span<BM>(a, a.qoff, a.Nq, grp, slot);
    const int64_t M = (int64_t)s.nq * grp;
    const int64_t r0 = (int64_t)s.tile * BM;
    if (s.g < 0 || r0 >= M) {
      if (!REST && want_bias) no_bias();
      return;
  }
  const int lane = lane_id(), col = lane & 15, g = lane >> 4;
  const int wave = uniform((int)threadIdx.x / kWave);
  const uint8_t* dist = BIAS ? dist_block(a, s) : nullptr;
  const int tiles = (s.nk + BN - 1) / BN;
  const ScoreScale sx = score_scale<T, BIAS, CAP>(a);
  int qi[QT], hg[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int64_t r = r0 + (wave * QT + t) * 16 + col;
    qi[t] = r < M ? (int)(r / grp) : -1;
    hg[t] = r < M ? (int)(r - (int64_t)qi[t] * grp) : 0;
  }
  const bool idle = r0 + wave * (QT * 16) >= M;  // a wavefront without rows only stages

  for (int kvh = kvh0; kvh < kvh1; ++kvh) {
    if (BIAS) {
      __syncthreads();
      load_bias<T>(a, kvh, grp, sx.add, tab, THREADS, threadIdx.x);
      if (want_bias)
        for (int i = threadIdx.x; i < WAVES * p.copies * (a.B + 1) * kWave; i += THREADS) bins[i] = 0.0f;
    }
    float ra[QT], rc[QT], delta[QT];
    frag_t<T, DP> qf[QT][KC], df[QT][KC];
    bool again = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int64_t node = s.q0 + max(qi[t], 0);
      const int head = kvh * grp + hg[t];
      const T* qrow = static_cast<const T*>(p.q) + node * a.ldq + (int64_t)head * D;
      const int64_t at = (node * a.H + head) * D;
      float dsum = 0.0f;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        qf[t][c] = df[t][c] = zero_frag<T, DP>();
        if (qi[t] >= 0) {
          qf[t][c] = load_frag<T, DP>(qrow, c, g, D, p.vec_q);
          df[t][c] = load_frag<T, DP>(static_cast<const T*>(p.dout) + at, c, g, D, p.vec_do);
          const frag_t<T, DP> of = load_frag<T, DP>(static_cast<const T*>(p.out) + at, c, g, D, p.vec_o);
#pragma unroll
          for (int e = 0; e < Frag<T, DP>::N; ++e) dsum += (float)df[t][c][e] * (float)of[e];
        }
      }
      dsum += __shfl_xor(dsum, 16);
      dsum += __shfl_xor(dsum, 32);
      delta[t] = dsum;
      ra[t] = INFINITY;  // p = 0
      rc[t] = 0.0f;
      if (qi[t] >= 0) {
        const float ls = p.lse[node * a.H + head];
        if (ls != -INFINITY) ra[t] = BIAS ? ls : ls * kLog2e;
        again = again || (BIAS && ls != -INFINITY && fabsf(ls) > kLongLse);
      }
    }
    again = (sizeof(T) == 2 && s.nk <= 128) || (BIAS && __syncthreads_or(again));

    x8_t<T> kr[KU][4], vr[VU];
    unsigned bk[QT][KT];
    const auto fetch = [&](int kt) {  // past the last key, its own row (p = 0 there)
      const int j0 = kt * BN, last = min(BN, s.nk - j0) - 1;
      const T* kp = static_cast<const T*>(p.k) + (int64_t)(s.k0 + j0) * a.ldk + (int64_t)kvh * D;
      const T* vp = static_cast<const T*>(p.v) + (int64_t)(s.k0 + j0) * a.ldv + (int64_t)kvh * D;
      const unsigned ldk = (unsigned)a.ldk, ldv = (unsigned)a.ldv;
      with_vector<T, VEC>(D, [&](auto vec) {
#pragma unroll
        for (int u = 0; u < KU; ++u) {
          const int c = u * THREADS + threadIdx.x;
          if (U::quad_col(c) >= DP) continue;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            kr[u][i] = load8_within<T, decltype(vec)::value>(kp, min(U::quad(c) * 4 + i, last) * ldk, U::quad_col(c), D);
        }
#pragma unroll
        for (int u = 0; u < VU; ++u) {
          const int c = u * THREADS + threadIdx.x;
          if (U::row8(c) < BN)
            vr[u] = load8_within<T, decltype(vec)::value>(vp, min(U::row8(c), last) * ldv, U::col8(c), D);
        }
      });
    };
    const auto place_tile = [&]() {  // the fetched rows to LDS
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        const int c = u * THREADS + threadIdx.x;
        if (U::quad_col(c) < DP) {
#pragma unroll
          for (int i = 0; i < 4; ++i) Rows::put8(Ks, U::quad(c) * 4 + i, U::quad_col(c), kr[u][i]);
          Columns::put_columns(Kt, U::quad(c), U::quad_col(c), kr[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < VU; ++u) {
        const int c = u * THREADS + threadIdx.x;
        if (U::row8(c) < BN) Rows::put8(Vs, U::row8(c), U::col8(c), vr[u]);
      }
    };
    const auto fetch_buckets = [&](int kt) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const uint8_t* row = dist + (int64_t)max(qi[t], 0) * s.nk;
#pragma unroll
        for (int x = 0; x < KT; ++x)
          bk[t][x] = dist == nullptr ? 0xFFFFFFFFu : load_buckets(row, kt * BN + x * 16 + g * 4, s.nk);
      }
    };
    // raw products and dp of key tile x
    const auto products = [&](int x, f32x4 (&sc)[QT], f32x4 (&dp)[QT]) {
#pragma unroll
      for (int t = 0; t < QT; ++t) sc[t] = dp[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const frag_t<T, DP> kf = Rows::frag(Ks, x * 16 + col, c, g);
        const frag_t<T, DP> vf = Rows::frag(Vs, x * 16 + col, c, g);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          sc[t] = mma(kf, qf[t][c], sc[t]);
          dp[t] = mma(vf, df[t][c], dp[t]);
        }
      }
    };

    if (again) {
      // first sweep: maximum, sum of exp and sum of exp * dp of every row
      float m[QT], l[QT], w[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        m[t] = -INFINITY;
        l[t] = w[t] = 0.0f;
      }
      for (int kt = 0; kt < tiles; ++kt) {
        const int n = min(BN, s.nk - kt * BN);
        fetch(kt);
        if (BIAS) fetch_buckets(kt);
        __syncthreads();
        place_tile();
        __syncthreads();
        if (idle) continue;
        for (int x = 0; x < KT && x * 16 < n; ++x) {
          f32x4 sc[QT], dp[QT];
          products(x, sc, dp);
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            unsigned b4 = bk[t][0];
#pragma unroll
            for (int y = 1; y < KT; ++y) b4 = x == y ? bk[t][y] : b4;
            float mx = m[t];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const unsigned b = min((b4 >> (8 * i)) & 0xFFu, (unsigned)a.B);
              const float add = BIAS ? tab[hg[t] * (a.B + 1) + b] : sx.add;
              float u = score<T, BIAS, CAP>(sc[t][i], add, sx);
              if (BIAS) u = add == -INFINITY ? -INFINITY : u;
              else u = x * 16 + g * 4 + i < n ? u * sx.unit : -INFINITY;
              sc[t][i] = u;
              mx = fmaxf(mx, u);
            }
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float base = mx == -INFINITY ? 0.0f : mx;
            const float unit = BIAS ? kLog2e : 1.0f;
            const float alpha = __builtin_amdgcn_exp2f((m[t] - base) * unit);
            l[t] *= alpha;
            w[t] *= alpha;
            m[t] = mx;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float e = __builtin_amdgcn_exp2f((sc[t][i] - base) * unit);
              l[t] += e;
              if (sc[t][i] != -INFINITY) w[t] += e * dp[t][i];
            }
          }
        }
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        l[t] += __shfl_xor(l[t], 16);
        l[t] += __shfl_xor(l[t], 32);
        w[t] += __shfl_xor(w[t], 16);
        w[t] += __shfl_xor(w[t], 32);
        if (l[t] == 0.0f) continue;  // (no rows, or none unmasked: p = 0 already)
        delta[t] = w[t] / l[t];
        if (BIAS) {
          ra[t] = m[t];
          rc[t] = -log2f(l[t]);
        } else {
          ra[t] = m[t] + log2f(l[t]);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t)
      if (qi[t] >= 0 && g == 0) {
        const int64_t at = (int64_t)(s.q0 + qi[t]) * a.H + kvh * grp + hg[t];
        p.row_a[at] = ra[t];
        if (BIAS) p.row_c[at] = rc[t];
        p.row_delta[at] = delta[t];
      }

    f32x4 o[QT][DT];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (tiles > 0) {
      if (AHEAD) fetch(0);
      if (BIAS) fetch_buckets(0);
    }
    for (int kt = 0; kt < tiles; ++kt) {
      const int n = min(BN, s.nk - kt * BN);
      if (!AHEAD) fetch(kt);
      __syncthreads();
      place_tile();
      __syncthreads();
      if (AHEAD && kt + 1 < tiles) fetch(kt + 1);
      if (idle) continue;
#pragma unroll
      for (int x2 = 0; x2 < KT / 2; ++x2) {
        if (x2 * 32 >= n) break;
        f32x4 sc[2][QT], dp[2][QT];
        products(2 * x2, sc[0], dp[0]);
        products(2 * x2 + 1, sc[1], dp[1]);
        x8_t<T> sf[QT], lo[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          const float* th = tab + hg[t] * (a.B + 1);
          unsigned b[2][4];
          float add[2][4];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              b[h][i] = BIAS ? min((bk[t][2 * x2 + h] >> (8 * i)) & 0xFFu, (unsigned)a.B) : 0;
              add[h][i] = BIAS ? th[b[h][i]] : sx.add;
            }
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float u = score<T, BIAS, CAP>(sc[h][t][i], add[h][i], sx);
              const float slope = cap_slope<T, CAP>(sc[h][t][i], sx);
              const bool live = BIAS ? add[h][i] != -INFINITY : (2 * x2 + h) * 16 + g * 4 + i < n;
              const float du = weight<BIAS>(u, sx.unit, ra[t], rc[t]) * (dp[h][t][i] - delta[t]);
              dp[h][t][i] = live ? du : 0.0f;
              sc[h][t][i] = dp[h][t][i] * slope;
            }
          if (want_bias) {
            float* bin = bins + (wave * p.copies + (p.copies > 1 ? t : 0)) * (a.B + 1) * kWave + lane;
            add_to_bins(bin, b[0], dp[0][t]);
            add_to_bins(bin, b[1], dp[1][t]);
          }
          sf[t] = as_operand<T>(sc[0][t], sc[1][t]);
          if (SPLIT) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              sc[0][t][i] -= (float)sf[t][i];
              sc[1][t][i] -= (float)sf[t][4 + i];
            }
            lo[t] = as_operand<T>(sc[0][t], sc[1][t]);
          }
        }
        constexpr int AT = NB == 2 && DT >= 2 ? 2 : 1;  // column tiles of a step
        x8_t<T> kf[NB][AT];
        const auto operands = [&](int d) {
#pragma unroll
          for (int e = 0; e < AT; ++e) kf[d % NB][e] = Columns::get8(Kt, (d * AT + e) * 16 + col, x2 * 32 + g * 8);
        };
        if (NB == 2) operands(0);
#pragma unroll
        for (int d = 0; d < DT / AT; ++d) {
          if (d + NB - 1 < DT / AT) operands(d + NB - 1);
          if (NB == 2) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int e = 0; e < AT; ++e)
#pragma unroll
            for (int t = 0; t < QT; ++t) {
              if (SPLIT) o[t][d * AT + e] = mma(kf[d % NB][e], lo[t], o[t][d * AT + e]);
              o[t][d * AT + e] = mma(kf[d % NB][e], sf[t], o[t][d * AT + e]);
            }
          if (NB == 2) __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (BIAS && kt + 1 < tiles) fetch_buckets(kt + 1);
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (qi[t] < 0) continue;
      T* row = static_cast<T*>(p.dq) + ((int64_t)(s.q0 + qi[t]) * a.H + kvh * grp + hg[t]) * D;
#pragma unroll
      for (int d = 0; d < DT; ++d) store4<T>(row, d * 16 + g * 4, D, p.vec_dq, o[t][d] * a.scale);
    }
    if (!want_bias) continue;
    __syncthreads();
    // (head, bucket) sums of the bins
    if (p.copies == 1 && 16 % grp == 0) {
      // one head a lane, col % grp: a wavefront a bucket, the lanes of a head added up
      for (int b = wave; b < a.B; b += WAVES) {
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += bins[(w * (a.B + 1) + b) * kWave + lane];
        for (int o = kWave / 2; o >= grp; o >>= 1) sum += __shfl_xor(sum, o);
        if (lane < grp) {
          float* to = bpart + (kvh * grp + lane) * a.B + b;
          *to = REST ? *to + sum : sum;
        }
      }
      continue;
    }
    for (int i = threadIdx.x; i < grp * a.B; i += THREADS) {
      const int h = i / a.B, b = i % a.B;
      float sum = 0.0f;
      for (int w = 0; w < WAVES * p.copies; ++w) {
        const int base = (int)((r0 + w * 16) % grp);  // the row of column c is w * 16 + c
        for (int e = 0; e < kWave; ++e) {
          const int ln = (e + b) & (kWave - 1);  // (neighbouring buckets: other banks)
          if ((base + (ln & 15)) % grp == h) sum += bins[(w * (a.B + 1) + b) * kWave + ln];
        }
      }
      float* to = bpart + kvh * grp * a.B + i;
      *to = REST ? *to + sum : sum;
    }
  }
  if (!REST) return;
  }
}

// Byte j of four neighbouring lanes' words, for lane j of them: from the rows of a
// 4 x 4 block of buckets, one a lane, to its columns.
__device__ __forceinline__ unsigned transpose_quad(unsigned v, unsigned j) {
  const unsigned r0 = (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x00, 0xF, 0xF, true);
  const unsigned r1 = (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x55, 0xF, 0xF, true);
  const unsigned r2 = (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0xAA, 0xF, 0xF, true);
  const unsigned r3 = (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0xFF, 0xF, 0xF, true);
  const unsigned sel = j | ((4 + j) << 8);
  const unsigned lo = __builtin_amdgcn_perm(r1, r0, sel), hi = __builtin_amdgcn_perm(r3, r2, sel);
  return (lo & 0xFFFFu) | (hi << 16);
}

template <typename T, int DP, int WAVES, int KT, int VEC, bool BIAS, bool CAP, bool REST>
__global__ __launch_bounds__(WAVES * kWave, (grad_waves<T, DP, KT>())) void attn_grad_kv(AttnGrad p) {
  constexpr int BK = WAVES * KT * 16, BR = sizeof(T) == 2 ? 64 : 32;
  constexpr int THREADS = WAVES * kWave;
  constexpr int NB = operands_ahead<T>();
  using Rows = Tile<T, DP, swapped_chunks<T, DP>()>;
  using Columns = Tile<T, BR, false>;
  constexpr int KC = Frag<T, DP>::KC, DT = DP / 16, XT = BR / 16;
  using U = Units<BR, DP>;
  constexpr int RU = (BR / 4 * (DP / 8) + THREADS - 1) / THREADS;  // four rows of eight columns
  constexpr bool AHEAD = VEC == 8 && RU * 64 * sizeof(T) / 4 <= 64;
  __shared__ T Qs[BR * Rows::LD];
  __shared__ T Os[BR * Rows::LD];
  __shared__ T Qt[DP * Columns::LD];
  __shared__ T Ot[DP * Columns::LD];
  __shared__ float rows[3][BR];  // row_a, row_c, delta
  extern __shared__ float tab[];
  const AttnShape& a = p.a;
  const int grp = a.H / a.Hk, D = a.D;
  const int per_slot = (a.Hk + p.heads - 1) / p.heads;
  const int slot = (int)(blockIdx.x / per_slot);
  const int kvh0 = (int)(blockIdx.x % per_slot) * p.heads;
  RestScan scan;
  if (REST && !any_rest(a, p.small)) return;
  for (int index = slot;; index += kRestBlocks) {
    const Span s = REST ? next_span<BK, true>(a, grp, p.small, index, scan)
                        : find_span<BK>(a, a.koff, a.Nk, 1, slot);
    const int64_t kt0 = (int64_t)s.tile * BK;
    if (s.g < 0 || kt0 >= s.nk) return;
    const int lane = lane_id(), col = lane & 15, g = lane >> 4;
    const int wave = uniform((int)threadIdx.x / kWave);
    const uint8_t* dist = BIAS ? dist_block(a, s) : nullptr;
    const ScoreScale sx = score_scale<T, BIAS, CAP>(a);
    const bool idle = kt0 + wave * (KT * 16) >= s.nk;  // a wavefront without keys only stages
    int key[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      const int64_t j = kt0 + (wave * KT + t) * 16 + col;
      key[t] = j < s.nk ? (int)j : -1;
  }
  const int rtiles = (s.nq + BR - 1) / BR;

  for (int kvh = kvh0; kvh < min(kvh0 + p.heads, a.Hk); ++kvh) {
    if (BIAS) {
      __syncthreads();
      load_bias<T>(a, kvh, grp, sx.add, tab, THREADS, threadIdx.x);
    }
    frag_t<T, DP> kf[KT][KC], vf[KT][KC];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      const int64_t node = s.k0 + max(key[t], 0);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        kf[t][c] = vf[t][c] = zero_frag<T, DP>();
        if (key[t] >= 0) {
          kf[t][c] = load_frag<T, DP>(static_cast<const T*>(p.k) + node * a.ldk + (int64_t)kvh * D, c, g, D, p.vec_k);
          vf[t][c] = load_frag<T, DP>(static_cast<const T*>(p.v) + node * a.ldv + (int64_t)kvh * D, c, g, D, p.vec_v);
        }
      }
    }
    f32x4 dk[KT][DT], dv[KT][DT];
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int d = 0; d < DT; ++d) dk[t][d] = dv[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    x8_t<T> qr[RU][4], dr[RU][4];
    float rv[3];
    unsigned bk[KT][XT];
    // tile i of the group's heads, one after the other
    const auto fetch = [&](int i) {
      const int head = kvh * grp + i / rtiles, q0 = (i % rtiles) * BR, n = min(BR, s.nq - q0);
      const T* qp = static_cast<const T*>(p.q) + (int64_t)(s.q0 + q0) * a.ldq + (int64_t)head * D;
      const int64_t ldo = (int64_t)a.H * D;
      const T* dp = static_cast<const T*>(p.dout) + (int64_t)(s.q0 + q0) * ldo + (int64_t)head * D;
      const unsigned ldq = (unsigned)a.ldq, ldd = (unsigned)ldo;
      with_vector<T, VEC>(D, [&](auto vec) {  // past the last query, its own row (p = 0 there)
#pragma unroll
        for (int u = 0; u < RU; ++u) {
          const int c = u * THREADS + threadIdx.x;
          if (U::quad_col(c) >= DP) continue;
#pragma unroll
          for (int e4 = 0; e4 < 4; ++e4) {
            const int r = min(U::quad(c) * 4 + e4, n - 1);
            qr[u][e4] = load8_within<T, decltype(vec)::value>(qp, r * ldq, U::quad_col(c), D);
            dr[u][e4] = load8_within<T, decltype(vec)::value>(dp, r * ldd, U::quad_col(c), D);
          }
        }
      });
      if ((int)threadIdx.x < BR) {
        const int64_t at = (int64_t)(s.q0 + q0 + min((int)threadIdx.x, n - 1)) * a.H + head;
        const bool in = (int)threadIdx.x < n;
        rv[0] = in ? p.row_a[at] : INFINITY;  // p = 0
        rv[1] = BIAS && in ? p.row_c[at] : 0.0f;
        rv[2] = in ? p.row_delta[at] : 0.0f;
      }
    };
    const auto fetch_buckets = [&](int i) {
      const int q0 = (i % rtiles) * BR, n = min(BR, s.nq - q0);
#pragma unroll
      for (int x = 0; x < XT; ++x) {
        const int r = x * 16 + g * 4 + (col & 3);
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          bk[t][x] = 0xFFFFFFFFu;
          const int64_t j = kt0 + (wave * KT + t) * 16 + (col & 12);
          if (dist != nullptr && r < n && j < s.nk)
            bk[t][x] = load_buckets(dist + (int64_t)(q0 + r) * s.nk, (int)j, s.nk);
        }
      }
    };
    const int all = rtiles * grp, per = (all + p.nsplit - 1) / p.nsplit;
    const int first = min((int)blockIdx.y * per, all), total = min(first + per, all);
    if (first < total) {
      if (AHEAD) fetch(first);
      if (BIAS) fetch_buckets(first);
    }
    for (int it = first; it < total; ++it) {
      const int n = min(BR, s.nq - (it % rtiles) * BR);
      if (!AHEAD) fetch(it);
      __syncthreads();
#pragma unroll
      for (int u = 0; u < RU; ++u) {
        const int c = u * THREADS + threadIdx.x;
        if (U::quad_col(c) < DP) {
#pragma unroll
          for (int e4 = 0; e4 < 4; ++e4) {
            Rows::put8(Qs, U::quad(c) * 4 + e4, U::quad_col(c), qr[u][e4]);
            Rows::put8(Os, U::quad(c) * 4 + e4, U::quad_col(c), dr[u][e4]);
          }
          Columns::put_columns(Qt, U::quad(c), U::quad_col(c), qr[u]);
          Columns::put_columns(Ot, U::quad(c), U::quad_col(c), dr[u]);
        }
      }
      if ((int)threadIdx.x < BR) {
        rows[0][threadIdx.x] = rv[0];
        if (BIAS) rows[1][threadIdx.x] = rv[1];
        rows[2][threadIdx.x] = rv[2];
      }
      __syncthreads();
      const float* th = tab + (it / rtiles) * (a.B + 1);
      if (AHEAD && it + 1 < total) fetch(it + 1);
      if (idle) continue;
#pragma unroll
      for (int x2 = 0; x2 < XT / 2; ++x2) {
        if (x2 * 32 >= n) break;
        f32x4 sc[KT][2], dp[KT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int x = 2 * x2 + h;
#pragma unroll
          for (int t = 0; t < KT; ++t) sc[t][h] = dp[t][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int c = 0; c < KC; ++c) {
            const frag_t<T, DP> qf = Rows::frag(Qs, x * 16 + col, c, g);
            const frag_t<T, DP> of = Rows::frag(Os, x * 16 + col, c, g);
#pragma unroll
            for (int t = 0; t < KT; ++t) {
              sc[t][h] = mma(qf, kf[t][c], sc[t][h]);
              dp[t][h] = mma(of, vf[t][c], dp[t][h]);
            }
          }
          const f32x4 ra = *reinterpret_cast<const f32x4*>(&rows[0][x * 16 + g * 4]);
          const f32x4 rc = BIAS ? *reinterpret_cast<const f32x4*>(&rows[1][x * 16 + g * 4]) : ra;
          const f32x4 dl = *reinterpret_cast<const f32x4*>(&rows[2][x * 16 + g * 4]);
#pragma unroll
          for (int t = 0; t < KT; ++t) {
            const unsigned b4 = BIAS ? transpose_quad(bk[t][x], (unsigned)(col & 3)) : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const unsigned b = BIAS ? min((b4 >> (8 * i)) & 0xFFu, (unsigned)a.B) : 0;
              const float add = BIAS ? th[b] : sx.add;
              const float u = score<T, BIAS, CAP>(sc[t][h][i], add, sx);
              const float slope = cap_slope<T, CAP>(sc[t][h][i], sx);
              float e = weight<BIAS>(u, sx.unit, ra[i], rc[i]);
              float ds = e * (dp[t][h][i] - dl[i]) * slope;
              if (BIAS) {  // (columns past the keys: zeros in k, not written)
                e = add == -INFINITY ? 0.0f : e;
                ds = add == -INFINITY ? 0.0f : ds;
              }
              sc[t][h][i] = e;
              dp[t][h][i] = ds;
            }
          }
        }
        x8_t<T> pf[KT], sf[KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          pf[t] = as_operand<T>(sc[t][0], sc[t][1]);
          sf[t] = as_operand<T>(dp[t][0], dp[t][1]);
        }
        x8_t<T> of[NB], qf[NB];
        const auto operands = [&](int d) {
          of[d % NB] = Columns::get8(Ot, d * 16 + col, x2 * 32 + g * 8);
          qf[d % NB] = Columns::get8(Qt, d * 16 + col, x2 * 32 + g * 8);
        };
        if (NB == 2) operands(0);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          if (d + NB - 1 < DT) operands(d + NB - 1);
          if (NB == 2) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int t = 0; t < KT; ++t) {
            dv[t][d] = mma(of[d % NB], pf[t], dv[t][d]);
            dk[t][d] = mma(qf[d % NB], sf[t], dk[t][d]);
          }
          if (NB == 2) __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (BIAS && it + 1 < total) fetch_buckets(it + 1);
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      if (key[t] < 0) continue;
      const int64_t at = ((int64_t)(s.k0 + key[t]) * a.Hk + kvh) * D;
      if (p.nsplit > 1) {
        const int64_t n = (int64_t)a.Nk * a.Hk * D;
        float* to = p.part + 2 * blockIdx.y * n + at;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          store4<float>(to, d * 16 + g * 4, D, D % 4 == 0 ? 4 : 1, dk[t][d]);
          store4<float>(to + n, d * 16 + g * 4, D, D % 4 == 0 && n % 4 == 0 ? 4 : 1, dv[t][d]);
        }
        continue;
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        store4<T>(static_cast<T*>(p.dk) + at, d * 16 + g * 4, D, p.vec_dk, dk[t][d] * a.scale);
        store4<T>(static_cast<T*>(p.dv) + at, d * 16 + g * 4, D, p.vec_dv, dv[t][d]);
      }
    }
  }
  if (!REST) return;
  }
}

// The parts of dk and dv added in order, an element a thread. Keys outside every graph
// are left as they were.
template <typename T>
__global__ __launch_bounds__(kBlock) void attn_grad_join(AttnGrad p) {
  const AttnShape& a = p.a;
  const int64_t n = (int64_t)a.Nk * a.Hk * a.D, i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  const int64_t w = (int64_t)a.Hk * a.D;
  if (i >= n || i < a.koff[0] * w || i >= a.koff[a.G] * w) return;
  float dk = 0.0f, dv = 0.0f;
#pragma unroll 4
  for (int sp = 0; sp < p.nsplit; ++sp) {
    dk += p.part[2 * sp * n + i];
    dv += p.part[(2 * sp + 1) * n + i];
  }
  static_cast<T*>(p.dk)[i] = to_type<T>(dk * a.scale);
  static_cast<T*>(p.dv)[i] = to_type<T>(dv);
}

// Tiles of rows and keys that the two passes take.
struct RowPlan {
  int waves, qt, copies, nsplit;
  int64_t slots;
  int small_waves, small_block;  // of the launch over small graphs (0: none)
  size_t small_lds;              // a wavefront's
};
inline size_t bins_bytes(int waves, int copies, int64_t B) {
  return sizeof(float) * (size_t)waves * copies * (B + 1) * kWave;
}

template <typename T, int DP, int WAVES, int QT, int VEC, bool REST = false>
int launch_grad_q(const AttnGrad& p, int64_t slots, hipStream_t s) {
  const int64_t blocks = slots * ((p.a.Hk + p.heads - 1) / p.heads);
  if (blocks >= (int64_t(1) << 31)) return fail(TFG_ERR_TOO_LARGE, "too many query tiles");
  const size_t lds = bias_table_bytes(p.a) + (p.bias_part != nullptr ? bins_bytes(WAVES, p.copies, p.a.B) : 0);
  const bool cap = p.a.cap > 0.0f;
  const unsigned n = (unsigned)blocks;
  if (p.a.B > 0) {
    if (cap) attn_grad_q<T, DP, WAVES, QT, VEC, true, true, REST><<<n, WAVES * kWave, lds, s>>>(p);
    else attn_grad_q<T, DP, WAVES, QT, VEC, true, false, REST><<<n, WAVES * kWave, lds, s>>>(p);
  } else {
    if (cap) attn_grad_q<T, DP, WAVES, QT, VEC, false, true, REST><<<n, WAVES * kWave, lds, s>>>(p);
    else attn_grad_q<T, DP, WAVES, QT, VEC, false, false, REST><<<n, WAVES * kWave, lds, s>>>(p);
  }
  TFG_LAUNCHED("attn_grad_q");
  return TFG_OK;
}
template <typename T, int DP, int WAVES, int KT, int VEC, bool REST = false>
int launch_grad_kv(const AttnGrad& p, hipStream_t s) {
  const int64_t slots = REST ? kRestBlocks : (int64_t)p.a.Nk / (WAVES * KT * 16) + p.a.G;
  const int64_t blocks = slots * ((p.a.Hk + p.heads - 1) / p.heads);
  if (blocks >= (int64_t(1) << 31)) return fail(TFG_ERR_TOO_LARGE, "too many key tiles");
  const size_t lds = bias_table_bytes(p.a);
  const bool cap = p.a.cap > 0.0f;
  const dim3 n((unsigned)blocks, (unsigned)p.nsplit);
  if (p.a.B > 0) {
    if (cap) attn_grad_kv<T, DP, WAVES, KT, VEC, true, true, REST><<<n, WAVES * kWave, lds, s>>>(p);
    else attn_grad_kv<T, DP, WAVES, KT, VEC, true, false, REST><<<n, WAVES * kWave, lds, s>>>(p);
  } else {
    if (cap) attn_grad_kv<T, DP, WAVES, KT, VEC, false, true, REST><<<n, WAVES * kWave, lds, s>>>(p);
    else attn_grad_kv<T, DP, WAVES, KT, VEC, false, false, REST><<<n, WAVES * kWave, lds, s>>>(p);
  }
  TFG_LAUNCHED("attn_grad_kv");
  if (p.nsplit > 1) {
    const int64_t values = (int64_t)p.a.Nk * p.a.Hk * p.a.D;
    attn_grad_join<T><<<(unsigned)((values + kBlock - 1) / kBlock), kBlock, 0, s>>>(p);
    TFG_LAUNCHED("attn_grad_join");
  }
  return TFG_OK;
}

}  // namespace tfg
