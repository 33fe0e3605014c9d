// Gradients of the attention over many small graphs (gfx950): graphs of at most 64
// queries and 64 keys, a wavefront for one (graph, key/value head) at a time, laid out as
// attn_small. All five products of a graph in one pass:
//   S = Q K^T, dP = dO V^T   with a key in each lane (l % 16), rows in its registers;
//   dV^T += dO^T P, dK^T += Q^T dS   P and dS as they lie, dO and Q as columns in LDS;
//   dQ^T = K^T dS^T          dS through LDS (rounded to the features' type), K as columns
// A row's delta is summed from p and dp in float32 (all of its keys are here), and its
// maximum and sum too where the log-sum has lost them (kLongLse). The bias bins stay in
// LDS for all of a wavefront's graphs.
#pragma once

#include "attention_grad.h"
#include "attention_small.h"

namespace tfg {

// Sum and maximum over the 16 lanes of a row of lanes, in all of them.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float row16_sum(float x) {
  x += dpp<0x128>(x);  // row_ror:8
  x += dpp<0x124>(x);
  x += dpp<0x122>(x);
  x += dpp<0x121>(x);
  return x;
}
__device__ __forceinline__ float row16_max(float x) {
  x = fmaxf(x, dpp<0x128>(x));
  x = fmaxf(x, dpp<0x124>(x));
  x = fmaxf(x, dpp<0x122>(x));
  x = fmaxf(x, dpp<0x121>(x));
  return x;
}

template <typename T>
__device__ __forceinline__ x8_t<T> join4(x4_t<T> a, x4_t<T> b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// LDS of a wavefront: Q and dO of 16 rows as columns, K as columns, dS of 16 rows.
template <typename T, int DP> struct SmallGrad {
  static constexpr int LDR = 16 + lds_pad<T>(), LDK = kSmallGraph + lds_pad<T>();
  static constexpr int elements = 2 * DP * LDR + DP * LDK + 16 * LDK;
};
// A lane's chunks of row (or key) `at` as columns.
template <typename T, int DP, int LD>
__device__ __forceinline__ void put_frag_columns(T* dst, int at, int g, const frag_t<T, DP> (&v)[Frag<T, DP>::KC]) {
#pragma unroll
  for (int c = 0; c < Frag<T, DP>::KC; ++c)
#pragma unroll
    for (int e = 0; e < Frag<T, DP>::N; ++e)
      dst[(c * Frag<T, DP>::W + g * Frag<T, DP>::N + e) * LD + at] = v[c][e];
}
inline int small_table(const AttnShape& a) {  // floats, a multiple of 16 bytes
  return a.B > 0 ? (int)((bias_table_bytes(a) / 4 + 3) / 4 * 4) : 0;
}
inline int small_bins(const AttnShape& a, bool want) {
  return want ? a.H / a.Hk * (a.B + 1) * kWave : 0;
}

// bf16 heads of at most 16 columns: three wavefronts a SIMD, although six registers a lane
// then go to scratch memory with a bias (4,096 graphs, 8 heads: 258 -> 220 us).
template <typename T, int DP, bool BIAS, bool CAP>
__global__ __launch_bounds__(4 * kWave, DP * sizeof(T) > 32 ? 1 : CAP ? 2 : 3) void attn_grad_small(AttnGrad p, int waves) {
  using L = SmallGrad<T, DP>;
  constexpr int LDR = L::LDR, LDK = L::LDK, KC = Frag<T, DP>::KC, DT = DP / 16, KT = kSmallTiles;
  extern __shared__ float dyn[];
  const AttnShape& a = p.a;
  const int grp = a.H / a.Hk, D = a.D;
  const int wave = uniform((int)threadIdx.x / kWave), nw = (int)blockDim.x / kWave;
  const int wid = (int)blockIdx.x * nw + wave;
  if (wid >= waves) return;
  const bool want_bias = BIAS && p.bias_part != nullptr;
  const int tabn = BIAS ? (grp * (a.B + 1) + 3) & ~3 : 0, binn = want_bias ? grp * (a.B + 1) * kWave : 0;
  float* tab = dyn + wave * (tabn + binn + L::elements * (int)sizeof(T) / 4);
  float* bins = tab + tabn;
  T* Qt = reinterpret_cast<T*>(bins + binn);
  T* Ot = Qt + DP * LDR;
  T* Kt = Ot + DP * LDR;
  T* Ds = Kt + DP * LDK;
  const int kvh = wid % a.Hk, lane = lane_id(), col = lane & 15, g = lane >> 4;
  const ScoreScale sx = score_scale<T, BIAS, CAP>(a);
  if (BIAS) load_bias<T>(a, kvh, grp, sx.add, tab, kWave, lane);
  for (int i = lane; i < binn; i += kWave) bins[i] = 0.0f;
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};

  for (int gi = wid / a.Hk; gi < a.G; gi += waves / a.Hk) {
    const Span s = small_span(a, uniform(gi));
    if (s.g < 0) continue;
    const uint8_t* dist = BIAS && s.nk > 0 ? dist_block(a, s) : nullptr;
    const int kts = (s.nk + 15) / 16, last = s.nk - 1;
    frag_t<T, DP> kf[KT][KC], vf[KT][KC];
    f32x4 dk[KT][DT], dv[KT][DT];
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
      for (int d = 0; d < DT; ++d) dk[x][d] = dv[x][d] = zero;
    if (s.nk > 0) {
      const T* kp = static_cast<const T*>(p.k) + (int64_t)s.k0 * a.ldk + (int64_t)kvh * D;
      const T* vp = static_cast<const T*>(p.v) + (int64_t)s.k0 * a.ldv + (int64_t)kvh * D;
#pragma unroll
      for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const unsigned r = min(x * 16 + col, last);
          kf[x][c] = frag_within<T, DP, true>(kp + r * (unsigned)a.ldk, c, g, D);
          vf[x][c] = frag_within<T, DP, true>(vp + r * (unsigned)a.ldv, c, g, D);
        }
      wave_sync();
#pragma unroll
      for (int x = 0; x < KT; ++x) put_frag_columns<T, DP, LDK>(Kt, x * 16 + col, g, kf[x]);
    }
    for (int h = 0; h < grp; ++h) {
      const int head = kvh * grp + h;
      const float* th = tab + h * (a.B + 1);
      for (int r0 = 0; r0 < s.nq; r0 += 16) {
        const int n = min(16, s.nq - r0);
        const int64_t node0 = s.q0 + r0;
        const unsigned r = min(col, n - 1);
        // rows as operands, and as columns in LDS
        frag_t<T, DP> qf[KC], of[KC];
        unsigned bk[KT];
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          qf[c] = frag_within<T, DP, false>(static_cast<const T*>(p.q) + (node0 + r) * a.ldq + (int64_t)head * D, c, g, D);
          of[c] = frag_within<T, DP, false>(static_cast<const T*>(p.dout) + ((node0 + r) * a.H + head) * D, c, g, D);
        }
        if (BIAS) {
          const int br = g * 4 + (col & 3);
#pragma unroll
          for (int y = 0; y < KT; ++y) {
            bk[y] = 0xFFFFFFFFu;
            if (dist != nullptr && br < n && y * 16 + (col & 12) < s.nk)
              bk[y] = load_buckets(dist + (r0 + br) * s.nk, y * 16 + (col & 12), s.nk);
          }
        }
        const float lse = p.lse[(node0 + r) * a.H + head];
        wave_sync();
        put_frag_columns<T, DP, LDR>(Qt, col, g, qf);
        put_frag_columns<T, DP, LDR>(Ot, col, g, of);
        const bool again = BIAS && __ballot(lse != -INFINITY && fabsf(lse) > kLongLse) != 0;
        float ra[4], rc[4], delta[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float ls = __shfl(lse, g * 4 + i);
          ra[i] = g * 4 + i < n && ls != -INFINITY ? (BIAS ? ls : ls * kLog2e) : INFINITY;  // +inf: p = 0
          rc[i] = delta[i] = 0.0f;
        }
        f32x4 sc[KT], dp[KT];
#pragma unroll
        for (int y = 0; y < KT; ++y) {
          if (y >= kts) break;
          sc[y] = dp[y] = zero;
#pragma unroll
          for (int c = 0; c < KC; ++c) {
            sc[y] = mma(qf[c], kf[y][c], sc[y]);
            dp[y] = mma(of[c], vf[y][c], dp[y]);
          }
          if (BIAS) bk[y] = transpose_quad(bk[y], (unsigned)(col & 3));
        }
        if (again) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int y = 0; y < KT; ++y)
              if (y < kts) {
                const float add = th[min((bk[y] >> (8 * i)) & 0xFFu, (unsigned)a.B)];
                m = fmaxf(m, add == -INFINITY ? add : score<T, BIAS, CAP>(sc[y][i], add, sx));
              }
            m = row16_max(m);
#pragma unroll
            for (int y = 0; y < KT; ++y)
              if (y < kts) {
                const float add = th[min((bk[y] >> (8 * i)) & 0xFFu, (unsigned)a.B)];
                const float u = score<T, BIAS, CAP>(sc[y][i], add, sx);
                l += add == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((u - m) * kLog2e);
              }
            l = row16_sum(l);
            if (l != 0.0f) {
              ra[i] = m;
              rc[i] = -log2f(l);
            }
          }
        }
        f32x4 slope[KT];
#pragma unroll
        for (int y = 0; y < KT; ++y) {
          if (y >= kts) break;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float add = BIAS ? th[min((bk[y] >> (8 * i)) & 0xFFu, (unsigned)a.B)] : sx.add;
            const bool live = BIAS ? add != -INFINITY : y * 16 + col < s.nk;
            const float e = weight<BIAS>(score<T, BIAS, CAP>(sc[y][i], add, sx), sx.unit, ra[i], rc[i]);
            slope[y][i] = cap_slope<T, CAP>(sc[y][i], sx);
            sc[y][i] = live ? e : 0.0f;
            dp[y][i] = live ? dp[y][i] : 0.0f;
            delta[i] = __builtin_fmaf(sc[y][i], dp[y][i], delta[i]);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) delta[i] = row16_sum(delta[i]);
        x4_t<T> pf[KT], sf[KT];
#pragma unroll
        for (int y = 0; y < KT; ++y) {
          if (y >= kts) break;
          unsigned b[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            dp[y][i] = sc[y][i] * (dp[y][i] - delta[i]);
            b[i] = BIAS ? min((bk[y] >> (8 * i)) & 0xFFu, (unsigned)a.B) : 0;
          }
          if (want_bias) add_to_bins(bins + h * (a.B + 1) * kWave + lane, b, dp[y]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            pf[y][i] = to_type<T>(sc[y][i]);
            sf[y][i] = to_type<T>(CAP ? dp[y][i] * slope[y][i] : dp[y][i]);
            Ds[(g * 4 + i) * LDK + y * 16 + col] = sf[y][i];
          }
        }
        // the keys from kts * 16 to the next multiple of 32 have no weight
        if (kts & 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) Ds[(g * 4 + i) * LDK + kts * 16 + col] = (T)0.0f;
        }
        wave_sync();
        // dV, dK over these rows
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const x4_t<T> oc = *reinterpret_cast<const x4_t<T>*>(Ot + (d * 16 + col) * LDR + g * 4);
          const x4_t<T> qc = *reinterpret_cast<const x4_t<T>*>(Qt + (d * 16 + col) * LDR + g * 4);
#pragma unroll
          for (int y = 0; y < KT; ++y) {
            if (y >= kts) break;
            dv[y][d] = mma(oc, pf[y], dv[y][d]);
            dk[y][d] = mma(qc, sf[y], dk[y][d]);
          }
        }
        // dQ of these rows
        f32x4 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = zero;
#pragma unroll
        for (int y = 0; y < KT / 2; ++y) {
          if (2 * y >= kts) break;
          const x8_t<T> ds = lds8<T>(Ds + col * LDK + y * 32 + g * 8);
#pragma unroll
          for (int d = 0; d < DT; ++d) o[d] = mma(lds8<T>(Kt + (d * 16 + col) * LDK + y * 32 + g * 8), ds, o[d]);
        }
        if (col < n) {
          T* row = static_cast<T*>(p.dq) + ((node0 + col) * a.H + head) * D;
#pragma unroll
          for (int d = 0; d < DT; ++d) store4<T>(row, d * 16 + g * 4, D, p.vec_dq, o[d] * a.scale);
        }
      }
    }
#pragma unroll
    for (int y = 0; y < KT; ++y) {
      const int key = y * 16 + col;
      if (key >= s.nk) continue;
      const int64_t at = ((int64_t)(s.k0 + key) * a.Hk + kvh) * D;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        store4<T>(static_cast<T*>(p.dk) + at, d * 16 + g * 4, D, p.vec_dk, dk[y][d] * a.scale);
        store4<T>(static_cast<T*>(p.dv) + at, d * 16 + g * 4, D, p.vec_dv, dv[y][d]);
      }
    }
  }
  if (!want_bias) return;
  wave_sync();
  for (int i = 0; i < grp * a.B; ++i) {
    float sum = bins[(i / a.B * (a.B + 1) + i % a.B) * kWave + lane];
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) p.bias_part[((int64_t)(wid / a.Hk) * a.H + (int64_t)kvh * grp) * a.B + i] = sum;
  }
}

// The launch: wavefronts a block by what their LDS allows, wavefronts in all by how many
// blocks the card holds at once; 0: the kernel does not take this shape.
struct SmallPlan {
  int waves, per_block;
  size_t lds;  // a wavefront
};
inline SmallPlan small_grad_plan(int float_type, const AttnShape& a, bool want) {
  SmallPlan r{0, 0, 0};
  const size_t sz = float_type == TFG_BF16 ? 2 : 4;
  const int DP = a.D <= 16 ? 16 : a.D <= 32 ? 32 : 64, per = (int)(16 / sz);
  if (a.D > 64 || (sz == 4 && a.D > 32) || a.D % per != 0 || !small_graphs(a.Nq, a.Nk, a.G, a.Hk)) return r;
  const size_t elements = 2 * DP * (16 + per) + DP * (kSmallGraph + per) + 16 * (kSmallGraph + per);
  r.lds = sizeof(float) * (size_t)(small_table(a) + small_bins(a, want)) + sz * elements;
  if (r.lds > (40u << 10)) return r;
  r.per_block = 4;
  // as many as the card holds at once (4,096 graphs: 212 us with 12 a CU, 224 with 24, 266 with 8)
  const int held = DP * sz > 32 ? 2 : a.cap > 0.0f ? 2 : 3;
  const int blocks = (int)std::min<size_t>((160u << 10) / (4 * r.lds), held);  // a CU
  r.waves = small_waves(a, 4 * blocks);
  return r;
}

template <typename T, int DP>
int launch_grad_small(const AttnGrad& p, const SmallPlan& r, hipStream_t s) {
  const unsigned blocks = (unsigned)((r.waves + r.per_block - 1) / r.per_block);
  const unsigned threads = r.per_block * kWave;
  const size_t lds = r.lds * r.per_block;
  const bool cap = p.a.cap > 0.0f;
  if (p.a.B > 0) {
    if (cap) attn_grad_small<T, DP, true, true><<<blocks, threads, lds, s>>>(p, r.waves);
    else attn_grad_small<T, DP, true, false><<<blocks, threads, lds, s>>>(p, r.waves);
  } else {
    if (cap) attn_grad_small<T, DP, false, true><<<blocks, threads, lds, s>>>(p, r.waves);
    else attn_grad_small<T, DP, false, false><<<blocks, threads, lds, s>>>(p, r.waves);
  }
  TFG_LAUNCHED("attn_grad_small");
  return TFG_OK;
}

}  // namespace tfg
