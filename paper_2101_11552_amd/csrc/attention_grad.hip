// Gradients of the attention inside each graph of a BatchGraph (gfx950).
//
// With p = exp(u - lse) recomputed from the forward's log-sum and
// delta[row] = <dout[row], out[row]> (= sum over the keys of p dp):
//   dv = p^T dout;  dp = dout v^T;  du = p (dp - delta);
//   dbias[head, b] = sum of du over the pairs of bucket b;
//   ds = du (1 - tanh^2) (capped scores);  dq = scale ds k;  dk = scale ds^T q
// Two passes, each of which owns its outputs (no atomics between blocks, a fixed
// order of every sum): attn_grad_q over tiles of rows (delta, dq and the bias),
// then attn_grad_kv over tiles of keys (dk, dv), whose rows are the queries of
// all heads that share the key/value head. Scores and dp are formed in both:
// seven products instead of five, in exchange for no float atomics on dq.
#include "attention.h"
#include "columns.h"

namespace tfg {
namespace {

struct AttnGrad {
  AttnShape a;
  const void *q, *k, *v, *out, *dout;
  const float* lse;
  void *dq, *dk, *dv;
  float* delta;      // [Nq, H]
  float* bias_part;  // [slots][H * B] partial bias gradients, or NULL
  int vec_q, vec_k, vec_v, vec_o, vec_do, vec_dq, vec_dk, vec_dv;
  int copies;        // bias bins a wavefront keeps: one, or one a query tile
};

// Scores of one tile in base 2 from the raw products, and the derivative of the
// cap at them.
template <typename T>
__device__ __forceinline__ float capped(float s, float inv_cap, float cap2, float scale2,
                                        bool cap, float* slope) {
  if (!cap) {
    *slope = 1.0f;
    return s * scale2;
  }
  const float t = cap_tanh<T>(s * inv_cap);
  *slope = 1.0f - t * t;
  return cap2 * t;
}

template <typename T, int DP, int WAVES, int QT>
__global__ __launch_bounds__(WAVES * kWave) void attn_grad_q(AttnGrad p) {
  constexpr int BM = WAVES * QT * 16, BN = sizeof(T) == 2 ? 64 : 32;
  constexpr int THREADS = WAVES * kWave, LDK = DP + lds_pad<T>(), LDT = BN + lds_pad<T>();
  constexpr int KC = DP / 32, DT = DP / 16, KT = BN / 16;
  __shared__ T Ks[BN * LDK];
  __shared__ T Vs[BN * LDK];
  __shared__ T Kt[DP * LDT];
  extern __shared__ float dyn[];
  const AttnShape& a = p.a;
  const int grp = a.H / a.Hk, D = a.D;
  const int64_t slot = blockIdx.x / a.Hk;
  const int kvh = (int)(blockIdx.x % a.Hk);
  float* tab = dyn;
  float* bins = dyn + grp * a.B;  // [WAVES][copies][B][64], one column a lane
  const bool want_bias = p.bias_part != nullptr;
  float* bpart = want_bias ? p.bias_part + (slot * a.H + (int64_t)kvh * grp) * a.B : nullptr;
  const Span s = find_span<BM>(a, a.qoff, a.Nq, grp, slot);
  const int64_t M = (int64_t)s.nq * grp;
  const int64_t r0 = (int64_t)s.tile * BM;
  if (s.g < 0 || r0 >= M) {
    if (want_bias)
      for (int i = threadIdx.x; i < grp * a.B; i += THREADS) bpart[i] = 0.0f;
    return;
  }
  const int lane = lane_id(), col = lane & 15, g = lane >> 4;
  const int wave = uniform((int)threadIdx.x / kWave);
  const uint8_t* dist = a.B > 0 ? dist_block(a, s) : nullptr;
  if (a.B > 0) load_bias<T>(a, kvh, grp, tab, THREADS);
  if (want_bias)
    for (int i = threadIdx.x; i < WAVES * p.copies * a.B * kWave; i += THREADS) bins[i] = 0.0f;

  int qi[QT], hg[QT];
  float lse2[QT], delta[QT];
  x8_t<T> qf[QT][KC], df[QT][KC];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int64_t r = r0 + (wave * QT + t) * 16 + col;
    qi[t] = r < M ? (int)(r / grp) : -1;
    hg[t] = r < M ? (int)(r - (int64_t)qi[t] * grp) : 0;
    const int64_t node = s.q0 + max(qi[t], 0);
    const int head = kvh * grp + hg[t];
    const T* qrow = static_cast<const T*>(p.q) + node * a.ldq + (int64_t)head * D;
    const int64_t at = (node * a.H + head) * D;
    float dsum = 0.0f;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[t][c][e] = df[t][c][e] = (T)0.0f;
      if (qi[t] >= 0) {
        qf[t][c] = load8<T>(qrow, c * 32 + g * 8, D, p.vec_q);
        df[t][c] = load8<T>(static_cast<const T*>(p.dout) + at, c * 32 + g * 8, D, p.vec_do);
        const x8_t<T> of = load8<T>(static_cast<const T*>(p.out) + at, c * 32 + g * 8, D, p.vec_o);
#pragma unroll
        for (int e = 0; e < 8; ++e) dsum += (float)df[t][c][e] * (float)of[e];
      }
    }
    dsum += __shfl_xor(dsum, 16);
    dsum += __shfl_xor(dsum, 32);
    delta[t] = dsum;
    lse2[t] = INFINITY;  // p = 0
    if (qi[t] >= 0) {
      const float ls = p.lse[node * a.H + head];
      if (ls != -INFINITY) lse2[t] = ls * kLog2e;
      if (g == 0) p.delta[node * a.H + head] = dsum;
    }
  }
  f32x4 o[QT][DT];
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int tiles = (s.nk + BN - 1) / BN;
  const float scale2 = a.scale * kLog2e, inv_cap = a.cap > 0.0f ? a.scale / a.cap : 0.0f;
  const float cap2 = a.cap * kLog2e;
  const bool cap = a.cap > 0.0f;

  for (int kt = 0; kt < tiles; ++kt) {
    const int j0 = kt * BN, n = min(BN, s.nk - j0);
    const T* kp = static_cast<const T*>(p.k) + (int64_t)(s.k0 + j0) * a.ldk + (int64_t)kvh * D;
    const T* vp = static_cast<const T*>(p.v) + (int64_t)(s.k0 + j0) * a.ldv + (int64_t)kvh * D;
    __syncthreads();
    stage_columns<T, BN, DP, LDT, LDK, THREADS>(Kt, Ks, n, D, p.vec_k,
                                                [&](int r) { return kp + r * a.ldk; });
    stage_rows<T, BN, DP, LDK, THREADS>(Vs, n, D, p.vec_v, [&](int r) { return vp + r * a.ldv; });
    __syncthreads();
#pragma unroll
    for (int x2 = 0; x2 < KT / 2; ++x2) {
      f32x4 sc[QT][2], dp[QT][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int x = 2 * x2 + h;
#pragma unroll
        for (int t = 0; t < QT; ++t) sc[t][h] = dp[t][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const x8_t<T> kf = lds8<T>(Ks + (x * 16 + col) * LDK + c * 32 + g * 8);
          const x8_t<T> vf = lds8<T>(Vs + (x * 16 + col) * LDK + c * 32 + g * 8);
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            sc[t][h] = mma(kf, qf[t][c], sc[t][h]);
            dp[t][h] = mma(vf, df[t][c], dp[t][h]);
          }
        }
      }
      x8_t<T> sf[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const uint8_t* drow = dist != nullptr && qi[t] >= 0 ? dist + (int64_t)qi[t] * s.nk : nullptr;
        float* bin = bins + (int64_t)(wave * p.copies + (p.copies > 1 ? t : 0)) * a.B * kWave + lane;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int j = j0 + (2 * x2 + h) * 16 + g * 4;
          unsigned bk = 0xFFFFFFFFu;
          if (a.B > 0 && drow != nullptr) bk = load_buckets(drow, j, s.nk);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float slope;
            float u = capped<T>(sc[t][h][i], inv_cap, cap2, scale2, cap, &slope);
            bool live = j + i < s.nk;
            int b = 0;
            if (a.B > 0) {
              b = (int)((bk >> (8 * i)) & 0xFFu);
              live = live && b < a.B;
              u += tab[hg[t] * a.B + (b < a.B ? b : 0)];
            }
            const float du = live ? __builtin_amdgcn_exp2f(u - lse2[t]) * (dp[t][h][i] - delta[t]) : 0.0f;
            // (one lane adds to a bin: the order of its additions is the program's)
            if (want_bias && live)
              __hip_atomic_fetch_add(bin + b * kWave, du, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            sc[t][h][i] = du * slope;
          }
        }
        sf[t] = as_operand<T>(sc[t][0], sc[t][1]);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const x8_t<T> kf = lds8<T>(Kt + (d * 16 + col) * LDT + x2 * 32 + g * 8);
#pragma unroll
        for (int t = 0; t < QT; ++t) o[t][d] = mma(kf, sf[t], o[t][d]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    if (qi[t] < 0) continue;
    T* row = static_cast<T*>(p.dq) + ((int64_t)(s.q0 + qi[t]) * a.H + kvh * grp + hg[t]) * D;
#pragma unroll
    for (int d = 0; d < DT; ++d) store4<T>(row, d * 16 + g * 4, D, p.vec_dq, o[t][d] * a.scale);
  }
  if (!want_bias) return;
  __syncthreads();
  // (head, bucket) sums of the bins; neighbouring buckets start at other lanes, so
  // that they read other banks
  for (int i = threadIdx.x; i < grp * a.B; i += THREADS) {
    const int h = i / a.B, b = i % a.B;
    float sum = 0.0f;
    for (int w = 0; w < WAVES * p.copies; ++w) {
      // the row of column c in this bin: (w * 16 + c) past the tile's first, up to
      // a multiple of the group where one bin serves every query tile
      const int first = p.copies > 1 || QT == 1 ? w * 16 : 0;
      const int base = (int)((r0 + first) % grp);
      for (int e = 0; e < kWave; ++e) {
        const int ln = (e + b) & (kWave - 1);
        if ((base + (ln & 15)) % grp == h) sum += bins[((int64_t)w * a.B + b) * kWave + ln];
      }
    }
    bpart[i] = sum;
  }
}

template <typename T, int DP, int WAVES, int KT>
__global__ __launch_bounds__(WAVES * kWave) void attn_grad_kv(AttnGrad p) {
  constexpr int BK = WAVES * KT * 16, BR = sizeof(T) == 2 ? 64 : 32;
  constexpr int THREADS = WAVES * kWave, LDK = DP + lds_pad<T>(), LDT = BR + lds_pad<T>();
  constexpr int KC = DP / 32, DT = DP / 16;
  __shared__ T Qs[BR * LDK];
  __shared__ T Os[BR * LDK];
  __shared__ T Qt[DP * LDT];
  __shared__ T Ot[DP * LDT];
  __shared__ float row_lse[BR], row_delta[BR];
  __shared__ int row_q[BR], row_h[BR];
  extern __shared__ float tab[];
  const AttnShape& a = p.a;
  const int grp = a.H / a.Hk, D = a.D;
  const int64_t slot = blockIdx.x / a.Hk;
  const int kvh = (int)(blockIdx.x % a.Hk);
  const Span s = find_span<BK>(a, a.koff, a.Nk, 1, slot);
  const int64_t M = (int64_t)s.nq * grp;
  const int64_t kt0 = (int64_t)s.tile * BK;
  if (s.g < 0 || kt0 >= s.nk) return;
  const int lane = lane_id(), col = lane & 15, g = lane >> 4;
  const int wave = uniform((int)threadIdx.x / kWave);
  const uint8_t* dist = a.B > 0 ? dist_block(a, s) : nullptr;
  if (a.B > 0) load_bias<T>(a, kvh, grp, tab, THREADS);

  int key[KT];
  x8_t<T> kf[KT][KC], vf[KT][KC];
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    const int64_t j = kt0 + (wave * KT + t) * 16 + col;
    key[t] = j < s.nk ? (int)j : -1;
    const int64_t node = s.k0 + max(key[t], 0);
#pragma unroll
    for (int c = 0; c < KC; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) kf[t][c][e] = vf[t][c][e] = (T)0.0f;
      if (key[t] >= 0) {
        kf[t][c] = load8<T>(static_cast<const T*>(p.k) + node * a.ldk + (int64_t)kvh * D,
                            c * 32 + g * 8, D, p.vec_k);
        vf[t][c] = load8<T>(static_cast<const T*>(p.v) + node * a.ldv + (int64_t)kvh * D,
                            c * 32 + g * 8, D, p.vec_v);
      }
    }
  }
  f32x4 dk[KT][DT], dv[KT][DT];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[t][d] = dv[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const float scale2 = a.scale * kLog2e, inv_cap = a.cap > 0.0f ? a.scale / a.cap : 0.0f;
  const float cap2 = a.cap * kLog2e;
  const bool cap = a.cap > 0.0f;

  for (int64_t rt = 0; rt < M; rt += BR) {
    const int n = (int)min<int64_t>(BR, M - rt);
    __syncthreads();
    for (int r = threadIdx.x; r < BR; r += THREADS) {
      const int64_t rr = min(rt + r, M - 1);
      const int qq = (int)(rr / grp), h = (int)(rr - (int64_t)qq * grp);
      const int64_t at = (int64_t)(s.q0 + qq) * a.H + kvh * grp + h;
      const float ls = p.lse[at];
      row_lse[r] = r < n && ls != -INFINITY ? ls * kLog2e : INFINITY;  // p = 0
      row_delta[r] = p.delta[at];
      row_q[r] = qq;
      row_h[r] = h * a.B;
    }
    const auto head_row = [&](int r, int64_t ld) -> int64_t {
      const int64_t rr = rt + r;
      const int64_t qq = rr / grp;
      return (s.q0 + qq) * ld + (kvh * grp + (rr - qq * grp)) * D;
    };
    stage_columns<T, BR, DP, LDT, LDK, THREADS>(
        Qt, Qs, n, D, p.vec_q, [&](int r) { return static_cast<const T*>(p.q) + head_row(r, a.ldq); });
    stage_columns<T, BR, DP, LDT, LDK, THREADS>(Ot, Os, n, D, p.vec_do, [&](int r) {
      return static_cast<const T*>(p.dout) + head_row(r, (int64_t)a.H * D);
    });
    __syncthreads();
#pragma unroll
    for (int x2 = 0; x2 < BR / 32; ++x2) {
      f32x4 sc[KT][2], dp[KT][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int x = 2 * x2 + h;
#pragma unroll
        for (int t = 0; t < KT; ++t) sc[t][h] = dp[t][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const x8_t<T> qf = lds8<T>(Qs + (x * 16 + col) * LDK + c * 32 + g * 8);
          const x8_t<T> of = lds8<T>(Os + (x * 16 + col) * LDK + c * 32 + g * 8);
#pragma unroll
          for (int t = 0; t < KT; ++t) {
            sc[t][h] = mma(qf, kf[t][c], sc[t][h]);
            dp[t][h] = mma(of, vf[t][c], dp[t][h]);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = x * 16 + g * 4 + i;
          const float ls = row_lse[r], dl = row_delta[r];
#pragma unroll
          for (int t = 0; t < KT; ++t) {
            float slope;
            float u = capped<T>(sc[t][h][i], inv_cap, cap2, scale2, cap, &slope);
            bool live = key[t] >= 0 && r < n;
            if (a.B > 0) {
              int b = 255;
              if (live && dist != nullptr) b = dist[(int64_t)row_q[r] * s.nk + key[t]];
              live = live && b < a.B;
              u += tab[row_h[r] + (b < a.B ? b : 0)];
            }
            const float e = live ? __builtin_amdgcn_exp2f(u - ls) : 0.0f;
            sc[t][h][i] = e;
            dp[t][h][i] = live ? e * (dp[t][h][i] - dl) * slope : 0.0f;
          }
        }
      }
      x8_t<T> pf[KT], sf[KT];
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        pf[t] = as_operand<T>(sc[t][0], sc[t][1]);
        sf[t] = as_operand<T>(dp[t][0], dp[t][1]);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const x8_t<T> of = lds8<T>(Ot + (d * 16 + col) * LDT + x2 * 32 + g * 8);
        const x8_t<T> qf = lds8<T>(Qt + (d * 16 + col) * LDT + x2 * 32 + g * 8);
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          dv[t][d] = mma(of, pf[t], dv[t][d]);
          dk[t][d] = mma(qf, sf[t], dk[t][d]);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    if (key[t] < 0) continue;
    const int64_t at = ((int64_t)(s.k0 + key[t]) * a.Hk + kvh) * D;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      store4<T>(static_cast<T*>(p.dk) + at, d * 16 + g * 4, D, p.vec_dk, dk[t][d] * a.scale);
      store4<T>(static_cast<T*>(p.dv) + at, d * 16 + g * 4, D, p.vec_dv, dv[t][d]);
    }
  }
}

constexpr size_t kMaxLds = 160 << 10;

// Tiles of rows the first pass takes.
struct RowPlan {
  int waves, qt, copies;
  int64_t slots;
};
size_t bins_bytes(int waves, int copies, int64_t B) {
  return sizeof(float) * (size_t)waves * copies * B * kWave;
}
RowPlan row_plan(int64_t Nq, int64_t G, int64_t H, int64_t Hk, int64_t D, int64_t B) {
  const int64_t grp = H / Hk, rows = Nq * grp / std::max<int64_t>(G, 1);
  RowPlan r{1, 1, 1, 0};
  if (rows > 96) r = {4, 2, 1, 0};
  else if (rows > 16) r = {1, 2, 1, 0};
  if (16 % grp != 0) r.copies = r.qt;
  // the LDS of the tiles (three of BN x DP), the bias table and the bins
  const int64_t DP = D <= 32 ? 32 : D <= 64 ? 64 : 128;
  const size_t tiles = 3 * 2 * 64 * (size_t)(DP + 16) + 2 * 8 * (size_t)DP;
  if (tiles + sizeof(float) * (size_t)(grp * B) + bins_bytes(r.waves, r.copies, B) > kMaxLds) r = {1, 1, 1, 0};
  r.slots = Nq * grp / (r.waves * r.qt * 16) + G;
  return r;
}

template <typename T, int DP, int WAVES, int QT>
int launch_grad_q(const AttnGrad& p, int64_t slots, hipStream_t s) {
  const int64_t blocks = slots * p.a.Hk;
  if (blocks >= (int64_t(1) << 31)) return fail(TFG_ERR_TOO_LARGE, "too many query tiles");
  size_t lds = sizeof(float) * (size_t)(p.a.H / p.a.Hk * p.a.B);
  if (p.bias_part != nullptr) lds += bins_bytes(WAVES, p.copies, p.a.B);
  attn_grad_q<T, DP, WAVES, QT><<<(unsigned)blocks, WAVES * kWave, lds, s>>>(p);
  TFG_LAUNCHED("attn_grad_q");
  return TFG_OK;
}
template <typename T, int DP, int WAVES, int KT>
int launch_grad_kv(const AttnGrad& p, hipStream_t s) {
  const int64_t blocks = ((int64_t)p.a.Nk / (WAVES * KT * 16) + p.a.G) * p.a.Hk;
  if (blocks >= (int64_t(1) << 31)) return fail(TFG_ERR_TOO_LARGE, "too many key tiles");
  attn_grad_kv<T, DP, WAVES, KT><<<(unsigned)blocks, WAVES * kWave,
                                   sizeof(float) * (size_t)(p.a.H / p.a.Hk * p.a.B), s>>>(p);
  TFG_LAUNCHED("attn_grad_kv");
  return TFG_OK;
}

template <typename T, int DP>
int launch_grad_width(const AttnGrad& p, const RowPlan& r, hipStream_t s) {
  if (p.a.Nq > 0) {
    int rc;
    if (r.waves == 4) rc = launch_grad_q<T, DP, 4, 2>(p, r.slots, s);
    else if (r.qt == 2) rc = launch_grad_q<T, DP, 1, 2>(p, r.slots, s);
    else rc = launch_grad_q<T, DP, 1, 1>(p, r.slots, s);
    if (rc) return rc;
  }
  if (p.a.Nk == 0) return TFG_OK;
  if (p.a.Nk / p.a.G <= 96) return launch_grad_kv<T, DP, 1, 2>(p, s);
  constexpr int KT = DP == 128 || sizeof(T) == 4 ? 1 : 2;
  return launch_grad_kv<T, DP, 4, KT>(p, s);
}

template <typename T>
int launch_grad_type(AttnGrad& p, const RowPlan& r, void* dbias, double* sums, hipStream_t s) {
  const int D = p.a.D;
  const int64_t ldo = (int64_t)p.a.H * D, ldk = (int64_t)p.a.Hk * D;
  p.vec_q = row_vector<T>(p.q, p.a.ldq, D);
  p.vec_k = row_vector<T>(p.k, p.a.ldk, D);
  p.vec_v = row_vector<T>(p.v, p.a.ldv, D);
  p.vec_o = row_vector<T>(p.out, ldo, D);
  p.vec_do = row_vector<T>(p.dout, ldo, D);
  p.vec_dq = row_vector<T>(p.dq, ldo, D);
  p.vec_dk = row_vector<T>(p.dk, ldk, D);
  p.vec_dv = row_vector<T>(p.dv, ldk, D);
  int rc;
  if (D <= 32) rc = launch_grad_width<T, 32>(p, r, s);
  else if (D <= 64) rc = launch_grad_width<T, 64>(p, r, s);
  else rc = launch_grad_width<T, 128>(p, r, s);
  if (rc || dbias == nullptr) return rc;
  const int n = p.a.H * p.a.B;
  // (no queries: no rows to add, zeros)
  return launch_column_sums(p.bias_part, p.a.Nq == 0 ? 0 : r.slots, n, static_cast<T*>(dbias), sums, s);
}

struct GradLayout {
  size_t delta, part, sums, total;
};
GradLayout grad_layout(int64_t Nq, int64_t H, int64_t B, const RowPlan& r) {
  GradLayout L;
  L.delta = 0;
  L.part = align_up(sizeof(float) * (size_t)(Nq * H), 256);
  L.sums = L.part + align_up(sizeof(float) * (size_t)(B > 0 ? r.slots * H * B : 0), 256);
  L.total = L.sums + align_up(B > 0 ? column_sums_bytes(r.slots, H * B) : 0, 256) + 256;
  return L;
}

}  // namespace

size_t attention_backward_ws_bytes(int64_t Nq, int64_t G, int64_t H, int64_t Hk, int64_t D, int64_t B) {
  return grad_layout(Nq, H, B, row_plan(Nq, G, H, Hk, D, B)).total;
}

int launch_attention_backward(const AttnShape& a, int float_type, const void* q, const void* k,
                              const void* v, const void* out, const float* lse, const void* dout,
                              void* dq, void* dk, void* dv, void* dbias, void* ws, hipStream_t s) {
  if (a.G == 0 && dbias == nullptr) return TFG_OK;
  const RowPlan r = row_plan(a.Nq, a.G, a.H, a.Hk, a.D, a.B);
  const GradLayout L = grad_layout(a.Nq, a.H, a.B, r);
  char* w = static_cast<char*>(ws);
  AttnGrad p{};
  p.a = a;
  if (a.G == 0) p.a.Nq = p.a.Nk = 0;
  p.q = q;
  p.k = k;
  p.v = v;
  p.out = out;
  p.dout = dout;
  p.lse = lse;
  p.dq = dq;
  p.dk = dk;
  p.dv = dv;
  p.delta = reinterpret_cast<float*>(w + L.delta);
  p.bias_part = dbias != nullptr ? reinterpret_cast<float*>(w + L.part) : nullptr;
  p.copies = r.copies;
  double* sums = reinterpret_cast<double*>(w + L.sums);
  if (float_type == TFG_BF16) return launch_grad_type<__bf16>(p, r, dbias, sums, s);
  return launch_grad_type<float>(p, r, dbias, sums, s);
}

}  // namespace tfg
