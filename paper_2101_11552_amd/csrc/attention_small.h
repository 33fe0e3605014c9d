// Attention over many small graphs (gfx950): graphs of at most 64 queries and 64 keys,
// a wavefront for one (graph, key/value head) at a time, with all of the graph's keys in
// its registers. No block barriers: a wavefront keeps its own part of LDS, takes one head
// for good and the graphs wid / Hk, + waves / Hk, .., so that neighbouring wavefronts read
// neighbouring columns of the same rows. Tiles of 16 rows or keys past a graph's end are
// skipped: at 35 nodes 9 of the 16 tiles of a 64 x 64 block are left.
// Larger graphs are left to the kernels of attention_fwd.h and attention_grad.h.
#pragma once

#include "attention_fwd.h"

namespace tfg {

constexpr int kSmallGraph = 64;
constexpr int kSmallTiles = kSmallGraph / 16;

// The graph's rows, or g < 0 where another launch has it.
__device__ __forceinline__ Span small_span(const AttnShape& a, int g) {
  Span s;
  s.g = g;
  s.tile = 0;
  s.q0 = clamp_off(a.qoff[g], a.Nq);
  s.nq = max(clamp_off(a.qoff[g + 1], a.Nq) - s.q0, 0);
  s.k0 = clamp_off(a.koff[g], a.Nk);
  s.nk = max(clamp_off(a.koff[g + 1], a.Nk) - s.k0, 0);
  if (s.nq > kSmallGraph || s.nk > kSmallGraph) s.g = -1;
  return s;
}

// Chunk c of group g of a row whose width is whole vectors; columns past D as load8_within,
// or zero.
template <typename T, int DP, bool ZERO>
__device__ __forceinline__ frag_t<T, DP> frag_within(const T* row, int c, int g, int D) {
  frag_t<T, DP> v;
  const int d0 = c * Frag<T, DP>::W + g * Frag<T, DP>::N;
  if constexpr (DP == 16) {
    typedef frag_t<T, DP> any4 __attribute__((aligned(sizeof(T))));
    v = *reinterpret_cast<const any4*>(row + min(d0, D - 4));
  } else {
    v = load8_within<T, 8>(row, 0u, d0, D);
  }
  if constexpr (ZERO) {
    if constexpr (sizeof(T) == 4 && DP > 16) {  // (eight columns may hold half a vector)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = d0 + (e & 4) < D ? v[e] : (T)0.0f;
    } else {
      if (d0 >= D) v = zero_frag<T, DP>();
    }
  }
  return v;
}

template <typename T, int DP> constexpr int small_fwd_lds() {  // elements a wavefront, without the table
  return DP * Tile<T, kSmallGraph>::LD;
}

template <typename T, int DP, bool BIAS, int CAP>
__global__ __launch_bounds__(4 * kWave) void attn_small(AttnFwd p, int waves) {
  constexpr int KC = Frag<T, DP>::KC, DT = DP / 16, KT = kSmallTiles;
  constexpr int VU = (kSmallGraph / 4 * (DP / 8) + kWave - 1) / kWave;
  using U = Units<kSmallGraph, DP>;
  using VTile = Tile<T, kSmallGraph>;
  extern __shared__ float dyn[];
  const AttnShape& a = p.a;
  const int grp = a.H / a.Hk, D = a.D;
  const int wave = uniform((int)threadIdx.x / kWave), nw = (int)blockDim.x / kWave;
  const int wid = (int)blockIdx.x * nw + wave;
  if (wid >= waves) return;
  const int tabn = BIAS ? (grp * (a.B + 1) + 3) & ~3 : 0;
  float* tab = dyn + wave * (tabn + small_fwd_lds<T, DP>() * (int)sizeof(T) / 4);
  T* Vt = reinterpret_cast<T*>(tab + tabn);
  const int kvh = wid % a.Hk, lane = lane_id(), col = lane & 15, g = lane >> 4;
  constexpr bool bounded = CAP == 2;
  const bool flip = a.scale < 0.0f;
  const float scale = fabsf(a.scale), scale2 = scale * kLog2e;
  const float to_tanh = CAP ? scale / a.cap : 0.0f, to_exp = to_tanh * (2.0f * kLog2e);
  const float cap = bounded ? a.cap * kLog2e : a.cap, cap_add = cap_offset<T>(cap);
  const float unit = bounded ? 1.0f : BIAS || CAP ? kLog2e : scale2;
  if (BIAS) load_bias<T>(a, kvh, grp, CAP ? cap_add : 0.0f, tab, kWave, lane);

  for (int gi = wid / a.Hk; gi < a.G; gi += waves / a.Hk) {
    const Span s = small_span(a, uniform(gi));
    if (s.g < 0 || s.nq == 0) continue;
    const uint8_t* dist = BIAS && s.nk > 0 ? dist_block(a, s) : nullptr;
    const int last = s.nk - 1;
    const int kts = (s.nk + 15) / 16;
    const T* kp = static_cast<const T*>(p.k) + (int64_t)s.k0 * a.ldk + (int64_t)kvh * D;
    const T* vp = static_cast<const T*>(p.v) + (int64_t)s.k0 * a.ldv + (int64_t)kvh * D;
    frag_t<T, DP> kf[KT][KC];
    x8_t<T> vr[VU][4];
    if (s.nk > 0) {
#pragma unroll
      for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int c = 0; c < KC; ++c)
          kf[x][c] = frag_within<T, DP, false>(kp + min(x * 16 + col, last) * (unsigned)a.ldk, c, g, D);
#pragma unroll
      for (int u = 0; u < VU; ++u) {
        const int c = u * kWave + lane;
        if (U::quad_col(c) >= DP) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          vr[u][i] = load8_within<T, 8>(vp, min(U::quad(c) * 4 + i, last) * (unsigned)a.ldv, U::quad_col(c), D);
      }
      wave_sync();
#pragma unroll
      for (int u = 0; u < VU; ++u) {
        const int c = u * kWave + lane;
        if (U::quad_col(c) < DP) VTile::put_columns(Vt, U::quad(c), U::quad_col(c), vr[u]);
      }
      wave_sync();
    }
    for (int h = 0; h < grp; ++h) {
      const int head = kvh * grp + h;
      const float* th = tab + h * (a.B + 1);
      for (int r0 = 0; r0 < s.nq; r0 += 16) {
        const int r = r0 + col, rc = min(r, s.nq - 1);
        const int64_t node = s.q0 + rc;
        frag_t<T, DP> qf[KC];
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          qf[c] = frag_within<T, DP, true>(static_cast<const T*>(p.q) + node * a.ldq + (int64_t)head * D, c, g, D);
          if (flip) qf[c] = -qf[c];
        }
        unsigned bk[KT];
        if (BIAS) {
#pragma unroll
          for (int x = 0; x < KT; ++x)
            bk[x] = dist == nullptr ? 0xFFFFFFFFu : load_buckets(dist + rc * s.nk, x * 16 + g * 4, s.nk);
        }
        f32x4 sc[KT];
        float mx = -INFINITY;
#pragma unroll
        for (int x = 0; x < KT; ++x) {
          if (x >= kts) break;
          sc[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int c = 0; c < KC; ++c) sc[x] = mma(kf[x][c], qf[c], sc[x]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float u = sc[x][i];
            if constexpr (BIAS) {
              const float add = th[min((bk[x] >> (8 * i)) & 0xFFu, (unsigned)a.B)];
              u = CAP ? capped<T>(u, to_tanh, to_exp, cap, add) : __builtin_fmaf(u, scale, add);
              u = add == -INFINITY ? -INFINITY : u;
            } else {
              if constexpr (CAP != 0) u = capped<T>(u, to_tanh, to_exp, cap, cap_add);
              u = x * 16 + g * 4 + i < s.nk ? u : -INFINITY;
            }
            sc[x][i] = u;
            if (!bounded) mx = fmaxf(mx, u);
          }
        }
        float base = 0.0f;
        if (!bounded) {
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          base = mx == -INFINITY ? 0.0f : mx;  // (nothing unmasked)
        }
        float l = 0.0f;
#pragma unroll
        for (int x = 0; x < KT; ++x) {
          if (x >= kts) break;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            // (a difference first: a bias of the type's lowest value does not overflow)
            sc[x][i] = __builtin_amdgcn_exp2f((sc[x][i] - base) * unit);
            l += sc[x][i];
          }
        }
        f32x4 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int x = 0; x < KT / 2; ++x) {
          if (2 * x >= kts) break;
          const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
          const x8_t<T> pf = as_operand<T>(sc[2 * x], 2 * x + 1 < kts ? sc[2 * x + 1] : zero);
#pragma unroll
          for (int d = 0; d < DT; ++d)
            o[d] = mma(VTile::get8(Vt, d * 16 + col, x * 32 + g * 8), pf, o[d]);
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (r >= s.nq) continue;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        T* orow = static_cast<T*>(p.out) + (node * a.H + head) * D;
#pragma unroll
        for (int d = 0; d < DT; ++d) store4<T>(orow, d * 16 + g * 4, D, p.vec_o, o[d] * inv);
        if (p.lse != nullptr && g == 0) {
          const float mu = bounded ? 0.0f : BIAS || CAP ? base : base * scale;
          p.lse[node * a.H + head] = l == 0.0f ? -INFINITY : mu + log2f(l) * kLn2;
        }
      }
    }
  }
}

// Whether graphs are small on average and many enough for a wavefront each.
inline bool small_graphs(int64_t Nq, int64_t Nk, int64_t G, int64_t Hk) {
  return G * Hk >= 512 && Nq <= kSmallGraph * G && Nk <= kSmallGraph * G;
}

// Wavefronts of a launch: whole multiples of the heads, `per_cu` a CU at most.
inline int small_waves(const AttnShape& a, int per_cu) {
  const int64_t most = std::max<int64_t>(256 * per_cu / a.Hk, 1);
  return (int)(std::min<int64_t>(a.G, most) * a.Hk);
}

// Bytes of LDS a wavefront takes; a block of four has to fit a CU.
template <typename T, int DP> size_t small_lds_bytes(const AttnShape& a) {
  return (bias_table_bytes(a) + 15) / 16 * 16 + sizeof(T) * small_fwd_lds<T, DP>();
}
template <typename T, int DP> bool small_fits(const AttnShape& a) {
  return 4 * small_lds_bytes<T, DP>(a) <= size_t(160) << 10;
}

template <typename T, int DP>
int launch_small(const AttnFwd& p, hipStream_t s) {
  const size_t lds = small_lds_bytes<T, DP>(p.a);
  const int waves = small_waves(p.a, 16);
  const unsigned blocks = (unsigned)((waves + 3) / 4);
  const int cap = p.a.cap <= 0.0f ? 0 : p.a.B > 0 || p.a.cap > kBoundedCap ? 1 : 2;
  if (p.a.B > 0) {
    if (cap) attn_small<T, DP, true, 1><<<blocks, 4 * kWave, 4 * lds, s>>>(p, waves);
    else attn_small<T, DP, true, 0><<<blocks, 4 * kWave, 4 * lds, s>>>(p, waves);
  } else {
    if (cap == 2) attn_small<T, DP, false, 2><<<blocks, 4 * kWave, 4 * lds, s>>>(p, waves);
    else if (cap) attn_small<T, DP, false, 1><<<blocks, 4 * kWave, 4 * lds, s>>>(p, waves);
    else attn_small<T, DP, false, 0><<<blocks, 4 * kWave, 4 * lds, s>>>(p, waves);
  }
  TFG_LAUNCHED("attn_small");
  return TFG_OK;
}

}  // namespace tfg
