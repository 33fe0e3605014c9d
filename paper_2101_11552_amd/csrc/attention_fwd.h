// Attention inside each graph of a BatchGraph (gfx950), the forward kernels, compiled per
// type and width in attention_bf16_narrow.hip and its like.
//
//   s = scale * <q, k>;  u = cap * tanh(s / cap) (cap > 0) + bias[head, dist];
//   out = sum over the graph's unmasked keys of softmax(u) * v
//
// One pass over the keys with the running maximum m and sum l of the softmax:
// a wavefront holds 16 * QT rows; for a tile of keys it forms S^T = K Q^T (a
// row's scores in the four lanes l % 16 = row, in registers), rescales l and the
// output by exp(m_old - m_new) where the maximum grew, and adds V^T P^T, whose
// right operand is P^T as it lies in the registers (tiles.h). Keys pass through
// LDS, row-major for the first product and as columns for the second; the next
// tile's rows are on their way to registers meanwhile. Capped scores without a
// bias are bounded by the cap, so that no maximum is kept for them.
// Scores, maximum, sum and output are float32; P is rounded to the features'
// type for its product (bf16: half a step, 2^-9 of each weight at most, as the
// output's own rounding).
//
// What bounds it (bf16): three graphs of 4,000 to 9,000 nodes, 8 heads of 64, capped: 514 us,
// 500 TFLOP/s; the matrix products alone would take 216 us at a large product's 1,190
// TFLOP/s, a score's exponential, reciprocal and exponential (16 cycles a wavefront each)
// some 305. float32: 4 graphs of 1,500, 8 heads of 64: 185 us, 100 TFLOP/s of a large
// product's 153. One query for a few very long graphs: reading k and v, 3.3 TB/s.
#pragma once

#include <type_traits>

#include "attention.h"

namespace tfg {

struct AttnFwd {
  AttnShape a;
  const void *q, *k, *v;
  void* out;
  float* lse;
  int vec_q, vec_o;
  int nsplit;      // > 1: the keys of a graph in that many parts, joined afterwards
  float* part;     // [nsplit][Nq * H][D] unnormalised partial outputs
  float* part_ml;  // [nsplit][Nq * H][2] their maximum and sum
  int small;       // graphs of at most so many queries and keys are another launch's
  int heads;       // key/value heads a block takes
};

// CAP: 0 none, 1 capped scores, 2 bounded ones (capped at kBoundedCap at most, no bias).
// Heads of 16 columns: four wavefronts a SIMD (float32, 96 graphs of 100 to 500, capped with
// a bias: 159 us, three 174).
template <typename T, int DP, int WAVES, int QT, int VEC, bool BIAS, int CAP, bool REST>
__global__ __launch_bounds__(WAVES * kWave, (DP == 16 && VEC == 8 && !REST ? 4 : 1)) void attn_fwd(AttnFwd p) {
  constexpr int BM = WAVES * QT * 16, BN = sizeof(T) == 2 ? 64 : 32;
  constexpr int THREADS = WAVES * kWave;
  using KTile = Tile<T, DP>;
  using VTile = Tile<T, BN>;
  constexpr int KC = Frag<T, DP>::KC, DT = DP / 16, KT = BN / 16;
  using U = Units<BN, DP>;
  // staging units of a thread: rows of eight columns (K), four rows of eight (V)
  constexpr int KU = (BN * DP / 8 + THREADS - 1) / THREADS;
  constexpr int VU = (BN / 4 * (DP / 8) + THREADS - 1) / THREADS;
  // the next tile waits in registers where it takes at most 48 of them
  constexpr bool AHEAD = VEC == 8 && (KU * 8 + VU * 32) * sizeof(T) / 4 <= 48;
  __shared__ T Ks[BN * KTile::LD];
  __shared__ T Vt[DP * VTile::LD];
  extern __shared__ float tab[];
  const AttnShape& a = p.a;
  const int grp = a.H / a.Hk, D = a.D;
  const int per_slot = (a.Hk + p.heads - 1) / p.heads;
  const int slot = (int)(blockIdx.x / per_slot);
  const int kvh0 = (int)(blockIdx.x % per_slot) * p.heads;
  RestScan scan;
  if (REST && !any_rest(a, p.small)) return;
  for (int index = slot;; index += kRestBlocks) {
    const Span s = REST ? next_span<BM, false>(a, grp, p.small, index, scan)
                        : find_span<BM>(a, a.qoff, a.Nq, grp, slot);
    const int64_t M = (int64_t)s.nq * grp;
    const int64_t r0 = (int64_t)s.tile * BM;
    if (s.g < 0 || r0 >= M) return;
    const int lane = lane_id(), col = lane & 15, g = lane >> 4;
    const int wave = uniform((int)threadIdx.x / kWave);
    const uint8_t* dist = BIAS ? dist_block(a, s) : nullptr;
    const int tiles = (s.nk + BN - 1) / BN;
    const int per = (tiles + p.nsplit - 1) / p.nsplit;
    const int t0 = min((int)blockIdx.y * per, tiles), t1 = min(t0 + per, tiles);
    const bool flip = a.scale < 0.0f;  // the maximum is taken over raw products: q changes sign
    const float scale = fabsf(a.scale), scale2 = scale * kLog2e;
    constexpr bool bounded = CAP == 2;
    const float to_tanh = CAP ? scale / a.cap : 0.0f, to_exp = to_tanh * (2.0f * kLog2e);
    const float cap = bounded ? a.cap * kLog2e : a.cap, cap_add = cap_offset<T>(cap);

    // this lane's rows (one a query tile)
    int qi[QT], hg[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int64_t r = r0 + (wave * QT + t) * 16 + col;
      qi[t] = r < M ? (int)(r / grp) : -1;
      hg[t] = r < M ? (int)(r - (int64_t)qi[t] * grp) : 0;
  }
  const bool idle = r0 + wave * (QT * 16) >= M;  // a wavefront without rows only stages

  for (int kvh = kvh0; kvh < min(kvh0 + p.heads, a.Hk); ++kvh) {
    if (BIAS) {
      __syncthreads();
      load_bias<T>(a, kvh, grp, CAP ? cap_add : 0.0f, tab, THREADS, threadIdx.x);
    }
    frag_t<T, DP> qf[QT][KC];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const T* row = static_cast<const T*>(p.q) + (int64_t)(s.q0 + max(qi[t], 0)) * a.ldq +
                     (int64_t)(kvh * grp + hg[t]) * D;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        qf[t][c] = zero_frag<T, DP>();
        if (qi[t] >= 0) qf[t][c] = load_frag<T, DP>(row, c, g, D, p.vec_q);
        if (flip) qf[t][c] = -qf[t][c];
      }
    }
    float m[QT], l[QT];
    f32x4 o[QT][DT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      m[t] = bounded ? 0.0f : -INFINITY;
      l[t] = 0.0f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    x8_t<T> kr[KU], vr[VU][4];
    unsigned bk[QT][KT];
    const auto fetch = [&](int kt) {  // the rows of tile kt to registers; past the last key, its own
      const int j0 = kt * BN, last = min(BN, s.nk - j0) - 1;
      const T* kp = static_cast<const T*>(p.k) + (int64_t)(s.k0 + j0) * a.ldk + (int64_t)kvh * D;
      const T* vp = static_cast<const T*>(p.v) + (int64_t)(s.k0 + j0) * a.ldv + (int64_t)kvh * D;
      const unsigned ldk = (unsigned)a.ldk, ldv = (unsigned)a.ldv;
      with_vector<T, VEC>(D, [&](auto vec) {
#pragma unroll
        for (int u = 0; u < KU; ++u) {
          const int c = u * THREADS + threadIdx.x;
          if (U::row8(c) < BN)
            kr[u] = load8_within<T, decltype(vec)::value>(kp, min(U::row8(c), last) * ldk, U::col8(c), D);
        }
#pragma unroll
        for (int u = 0; u < VU; ++u) {
          const int c = u * THREADS + threadIdx.x;
          if (U::quad_col(c) >= DP) continue;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            vr[u][i] = load8_within<T, decltype(vec)::value>(vp, min(U::quad(c) * 4 + i, last) * ldv, U::quad_col(c), D);
        }
      });
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
    if (t0 < t1) {
      if (AHEAD) fetch(t0);
      if (BIAS) fetch_buckets(t0);
    }
    for (int kt = t0; kt < t1; ++kt) {
      const int n = min(BN, s.nk - kt * BN);
      if (!AHEAD) fetch(kt);
      __syncthreads();  // the last tile has been used
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        const int c = u * THREADS + threadIdx.x;
        if (U::row8(c) < BN) KTile::put8(Ks, U::row8(c), U::col8(c), kr[u]);
      }
#pragma unroll
      for (int u = 0; u < VU; ++u) {
        const int c = u * THREADS + threadIdx.x;
        if (U::quad_col(c) < DP) VTile::put_columns(Vt, U::quad(c), U::quad_col(c), vr[u]);
      }
      __syncthreads();
      if (AHEAD && kt + 1 < t1) fetch(kt + 1);
      if (idle) continue;
      f32x4 sc[QT][KT];
#pragma unroll
      for (int x = 0; x < KT; ++x) {
#pragma unroll
        for (int t = 0; t < QT; ++t) sc[t][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const frag_t<T, DP> kf = KTile::frag(Ks, x * 16 + col, c, g);
#pragma unroll
          for (int t = 0; t < QT; ++t) sc[t][x] = mma(kf, qf[t][c], sc[t][x]);
        }
      }
      // the tile's weights, in place of its products (tail: keys from n on are masked; with a
      // bias their buckets are)
      const auto soften = [&](auto tail) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          // scores: natural units with a bias, raw products without one, base 2 where bounded
          if constexpr (BIAS) {
            const float* th = tab + hg[t] * (a.B + 1);
#pragma unroll
            for (int x = 0; x < KT; ++x)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const unsigned b = min((bk[t][x] >> (8 * i)) & 0xFFu, (unsigned)a.B);
                const float add = th[b];
                // (a select: whatever a masked pair's product is, NaN too, it is masked)
                const float u = CAP ? capped<T>(sc[t][x][i], to_tanh, to_exp, cap, add)
                                    : __builtin_fmaf(sc[t][x][i], scale, add);
                sc[t][x][i] = add == -INFINITY ? -INFINITY : u;
              }
          } else {
            if constexpr (CAP) {
#pragma unroll
              for (int x = 0; x < KT; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[t][x][i] = capped<T>(sc[t][x][i], to_tanh, to_exp, cap, cap_add);
            }
            if constexpr (decltype(tail)::value) {
#pragma unroll
              for (int x = 0; x < KT; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  if (x * 16 + g * 4 + i >= n) sc[t][x][i] = -INFINITY;
            }
          }
          float sum = 0.0f;
          if (bounded) {
#pragma unroll
            for (int x = 0; x < KT; ++x)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                sc[t][x][i] = __builtin_amdgcn_exp2f(sc[t][x][i]);
                sum += sc[t][x][i];
              }
            l[t] += sum;
            continue;
          }
          const float unit = BIAS || CAP ? kLog2e : scale2;  // one unit of a score in base 2
          float mx = -INFINITY;
#pragma unroll
          for (int x = 0; x < KT; ++x)
            mx = fmaxf(fmaxf(fmaxf(mx, sc[t][x][0]), fmaxf(sc[t][x][1], sc[t][x][2])), sc[t][x][3]);
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          const float mn = fmaxf(m[t], mx);
          float base = mn == -INFINITY ? 0.0f : mn;  // (nothing unmasked so far)
          if (__ballot(mn > m[t]) != 0) {
            const float alpha = __builtin_amdgcn_exp2f((m[t] - base) * unit);
            l[t] *= alpha;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[t][d] *= alpha;
            m[t] = mn;
          }
          if (BIAS && __ballot(fabsf(base) > kHugeScore) != 0) {
            // a bias of the type's lowest value: base * log2(e) would overflow
#pragma unroll
            for (int x = 0; x < KT; ++x)
#pragma unroll
              for (int i = 0; i < 4; ++i) sc[t][x][i] -= base;
            base = 0.0f;
          }
          const float off = -base * unit;
#pragma unroll
          for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              sc[t][x][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][x][i], unit, off));
              sum += sc[t][x][i];
            }
          l[t] += sum;
        }
      };
      if (!BIAS && n < BN) soften(std::true_type{});
      else soften(std::false_type{});
      if (BIAS && kt + 1 < t1) fetch_buckets(kt + 1);
#pragma unroll
      for (int x = 0; x < KT / 2; ++x) {
        x8_t<T> pf[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) pf[t] = as_operand<T>(sc[t][2 * x], sc[t][2 * x + 1]);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const x8_t<T> vf = VTile::get8(Vt, d * 16 + col, x * 32 + g * 8);
#pragma unroll
          for (int t = 0; t < QT; ++t) o[t][d] = mma(vf, pf[t], o[t][d]);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      l[t] += __shfl_xor(l[t], 16);
      l[t] += __shfl_xor(l[t], 32);
      if (qi[t] < 0) continue;
      const int64_t row = (int64_t)(s.q0 + qi[t]) * a.H + kvh * grp + hg[t];
      // the maximum in natural units
      const float mu = BIAS || CAP || m[t] == -INFINITY ? m[t] : m[t] * scale;
      if (p.nsplit > 1) {
        const int64_t at = (int64_t)blockIdx.y * a.Nq * a.H + row;
#pragma unroll
        for (int d = 0; d < DT; ++d)
          store4<float>(p.part + at * D, d * 16 + g * 4, D, D % 4 == 0 ? 4 : 1, o[t][d]);
        if (g == 0) {
          p.part_ml[2 * at] = mu;
          p.part_ml[2 * at + 1] = l[t];
        }
        continue;
      }
      // a row without unmasked keys: zeros, and -inf as its log-sum
      const float inv = l[t] == 0.0f ? 0.0f : 1.0f / l[t];
      T* orow = static_cast<T*>(p.out) + row * D;
#pragma unroll
      for (int d = 0; d < DT; ++d) store4<T>(orow, d * 16 + g * 4, D, p.vec_o, o[t][d] * inv);
      if (p.lse != nullptr && g == 0)
        p.lse[row] = l[t] == 0.0f ? -INFINITY : mu + log2f(l[t]) * kLn2;
    }
  }
  if (!REST) return;
  }
}

// Joins the parts of each (query, head): W wavefronts a row, lane i of each with part i's
// maximum and sum; wavefront w of the row adds the outputs of the parts w, w + W, .., two
// columns a lane. Rows outside every graph are left as they were.
constexpr int kKeyParts = 64;  // at most
constexpr int kFewParts = 4;   // one wavefront a row up to these, else four
template <typename T, int W>
__global__ __launch_bounds__(kBlock) void attn_join(AttnFwd p) {
  constexpr int C = kMaxHeadDim / kWave, R = kBlock / kWave / W, N = W == 1 ? kFewParts : kKeyParts / W;
  __shared__ float part[W][kMaxHeadDim];
  const AttnShape& a = p.a;
  const int lane = lane_id(), wave = uniform((int)threadIdx.x / kWave);
  const int64_t rows = (int64_t)a.Nq * a.H, row = (int64_t)blockIdx.x * R + (W == 1 ? wave : 0);
  if (row >= rows) return;
  const int q = (int)(row / a.H), w0 = W == 1 ? 0 : wave;
  if (q < a.qoff[0] || q >= a.qoff[a.G]) return;
  float ml = 0.0f, mm = -INFINITY;  // (a part without keys, or none unmasked: l = 0)
  if (lane < p.nsplit) {
    ml = p.part_ml[2 * (lane * rows + row) + 1];
    mm = ml != 0.0f ? p.part_ml[2 * (lane * rows + row)] : -INFINITY;
  }
  float x[N][C];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int sp = min(w0 + i * W, p.nsplit - 1);
#pragma unroll
    for (int c = 0; c < C; ++c)
      x[i][c] = p.part[(sp * rows + row) * a.D + min(c * kWave + lane, a.D - 1)];
  }
  float m = mm;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float w = ml != 0.0f ? __builtin_amdgcn_exp2f((mm - m) * kLog2e) : 0.0f;
  float l = w * ml, acc[C] = {};
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) l += __shfl_xor(l, o);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float ws = w0 + i * W < p.nsplit ? __shfl(w, (w0 + i * W) & (kWave - 1)) : 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] += ws != 0.0f ? ws * x[i][c] : 0.0f;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (p.lse != nullptr && lane == 0 && w0 == 0)
    p.lse[row] = l == 0.0f ? -INFINITY : m + log2f(l) * kLn2;
  T* out = static_cast<T*>(p.out) + row * a.D;
  if constexpr (W == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (c * kWave + lane < a.D) out[c * kWave + lane] = to_type<T>(acc[c] * inv);
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c) part[wave][c * kWave + lane] = acc[c];
    __syncthreads();
    const int d = threadIdx.x;
    if (d < a.D) {
      float t = part[0][d];
#pragma unroll
      for (int j = 1; j < W; ++j) t += part[j][d];
      out[d] = to_type<T>(t * inv);
    }
  }
}

template <typename T, int DP, int WAVES, int QT, int VEC, bool REST = false>
int launch_fwd(AttnFwd& p, hipStream_t s) {
  constexpr int BM = WAVES * QT * 16;
  const int grp = p.a.H / p.a.Hk;
  const int64_t slots = REST ? kRestBlocks : (int64_t)p.a.Nq * grp / BM + p.a.G;
  if ((int64_t)p.a.Nq * grp / BM + p.a.G >= (int64_t(1) << 31)) return fail(TFG_ERR_TOO_LARGE, "too many query tiles");
  const int64_t blocks = slots * ((p.a.Hk + p.heads - 1) / p.heads);
  if (blocks >= (int64_t(1) << 31)) return fail(TFG_ERR_TOO_LARGE, "too many query tiles");
  const dim3 grid((unsigned)blocks, (unsigned)p.nsplit);
  const size_t lds = bias_table_bytes(p.a);
  const int cap = p.a.cap <= 0.0f ? 0 : p.a.B > 0 || p.a.cap > kBoundedCap ? 1 : 2;
  if (p.a.B > 0) {
    if (cap) attn_fwd<T, DP, WAVES, QT, VEC, true, 1, REST><<<grid, WAVES * kWave, lds, s>>>(p);
    else attn_fwd<T, DP, WAVES, QT, VEC, true, 0, REST><<<grid, WAVES * kWave, lds, s>>>(p);
  } else {
    if (cap == 2) attn_fwd<T, DP, WAVES, QT, VEC, false, 2, REST><<<grid, WAVES * kWave, lds, s>>>(p);
    else if (cap) attn_fwd<T, DP, WAVES, QT, VEC, false, 1, REST><<<grid, WAVES * kWave, lds, s>>>(p);
    else attn_fwd<T, DP, WAVES, QT, VEC, false, 0, REST><<<grid, WAVES * kWave, lds, s>>>(p);
  }
  TFG_LAUNCHED("attn_fwd");
  if (p.nsplit > 1) {
    const int64_t rows = (int64_t)p.a.Nq * p.a.H;
    if (p.nsplit <= kFewParts) attn_join<T, 1><<<(unsigned)((rows + 3) / 4), kBlock, 0, s>>>(p);
    else attn_join<T, 4><<<(unsigned)rows, kBlock, 0, s>>>(p);
    TFG_LAUNCHED("attn_join");
  }
  return TFG_OK;
}

}  // namespace tfg
