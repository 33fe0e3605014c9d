// Attention inside each graph of a BatchGraph (gfx950), forward.
//
//   s = scale * <q, k>;  u = cap * tanh(s / cap) (cap > 0) + bias[head, dist];
//   out = sum over the graph's unmasked keys of softmax(u) * v
//
// One pass over the keys with the running maximum m and sum l of the softmax:
// a wavefront holds 16 * QT rows; for a tile of keys it forms S^T = K Q^T (a
// row's scores in the four lanes l % 16 = row, in registers), rescales l and the
// output by exp(m_old - m_new), and adds V^T P^T, whose right operand is P^T as
// it lies in the registers (tiles.h). Keys pass through LDS, row-major for the
// first product and as columns for the second. Scores, maximum, sum and output
// are float32; P is rounded to the features' type for its product (bf16: half a
// step, 2^-9 of each weight, like the output's own rounding).
#include "attention.h"

namespace tfg {
namespace {

struct AttnFwd {
  AttnShape a;
  const void *q, *k, *v;
  void* out;
  float* lse;
  int vec_q, vec_k, vec_v, vec_o;
  int64_t slots;
  int nsplit;      // > 1: the keys of a graph in that many parts, joined afterwards
  float* part;     // [nsplit][Nq * H][D] unnormalised partial outputs
  float* part_ml;  // [nsplit][Nq * H][2] their maximum (base 2) and sum
};

template <typename T, int DP, int WAVES, int QT>
__global__ __launch_bounds__(WAVES * kWave) void attn_fwd(AttnFwd p) {
  constexpr int BM = WAVES * QT * 16, BN = sizeof(T) == 2 ? 64 : 32;
  constexpr int THREADS = WAVES * kWave, LDK = DP + lds_pad<T>(), LDV = BN + lds_pad<T>();
  constexpr int KC = DP >= 32 ? DP / 32 : 1, DT = DP / 16, KT = BN / 16;
  __shared__ T Ks[BN * LDK];
  __shared__ T Vt[DP * LDV];
  extern __shared__ float tab[];
  const AttnShape& a = p.a;
  const int grp = a.H / a.Hk, D = a.D;
  const int64_t work = blockIdx.x;
  const int64_t slot = work / a.Hk;
  const int kvh = (int)(work % a.Hk);
  const Span s = find_span<BM>(a, a.qoff, a.Nq, grp, slot);
  const int64_t M = (int64_t)s.nq * grp;
  const int64_t r0 = (int64_t)s.tile * BM;
  if (s.g < 0 || r0 >= M) return;
  const int lane = lane_id(), col = lane & 15, g = lane >> 4;
  const int wave = uniform((int)threadIdx.x / kWave);
  const uint8_t* dist = a.B > 0 ? dist_block(a, s) : nullptr;
  if (a.B > 0) load_bias<T>(a, kvh, grp, tab, THREADS);

  // this lane's rows (one a query tile)
  int qi[QT], hg[QT];
  x8_t<T> qf[QT][KC];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int64_t r = r0 + (wave * QT + t) * 16 + col;
    qi[t] = r < M ? (int)(r / grp) : -1;
    hg[t] = r < M ? (int)(r - (int64_t)qi[t] * grp) : 0;
    const T* row = static_cast<const T*>(p.q) + (int64_t)(s.q0 + max(qi[t], 0)) * a.ldq +
                   (int64_t)(kvh * grp + hg[t]) * D;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[t][c][e] = (T)0.0f;
      if (qi[t] >= 0) qf[t][c] = load8<T>(row, c * 32 + g * 8, D, p.vec_q);
    }
  }
  float m[QT], l[QT];
  f32x4 o[QT][DT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // this part's tiles of keys
  const int tiles = (s.nk + BN - 1) / BN;
  const int per = (tiles + p.nsplit - 1) / p.nsplit;
  const int t0 = min((int)blockIdx.y * per, tiles), t1 = min(t0 + per, tiles);
  const float scale2 = a.scale * kLog2e, inv_cap = a.cap > 0.0f ? a.scale / a.cap : 0.0f;
  const float cap2 = a.cap * kLog2e;

  for (int kt = t0; kt < t1; ++kt) {
    const int j0 = kt * BN, n = min(BN, s.nk - j0);
    const T* kp = static_cast<const T*>(p.k) + (int64_t)(s.k0 + j0) * a.ldk + (int64_t)kvh * D;
    const T* vp = static_cast<const T*>(p.v) + (int64_t)(s.k0 + j0) * a.ldv + (int64_t)kvh * D;
    __syncthreads();
    stage_rows<T, BN, DP, LDK, THREADS>(Ks, n, D, p.vec_k, [&](int r) { return kp + r * a.ldk; });
    stage_columns<T, BN, DP, LDV, 0, THREADS>(Vt, nullptr, n, D, p.vec_v,
                                              [&](int r) { return vp + r * a.ldv; });
    __syncthreads();
    f32x4 sc[QT][KT];
#pragma unroll
    for (int x = 0; x < KT; ++x) {
#pragma unroll
      for (int t = 0; t < QT; ++t) sc[t][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const x8_t<T> kf = lds8<T>(Ks + (x * 16 + col) * LDK + c * 32 + g * 8);
#pragma unroll
        for (int t = 0; t < QT; ++t) sc[t][x] = mma(kf, qf[t][c], sc[t][x]);
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const uint8_t* drow = dist != nullptr && qi[t] >= 0 ? dist + (int64_t)qi[t] * s.nk : nullptr;
      float mx = -INFINITY;
#pragma unroll
      for (int x = 0; x < KT; ++x) {
        const int j = j0 + x * 16 + g * 4;
        unsigned bk = 0xFFFFFFFFu;
        if (a.B > 0 && drow != nullptr) bk = load_buckets(drow, j, s.nk);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float u = a.cap > 0.0f ? cap2 * cap_tanh<T>(sc[t][x][i] * inv_cap) : sc[t][x][i] * scale2;
          bool live = j + i < s.nk;
          if (a.B > 0) {
            const int b = (int)((bk >> (8 * i)) & 0xFFu);
            live = live && b < a.B;
            u += tab[hg[t] * a.B + (b < a.B ? b : 0)];
          }
          u = live ? u : -INFINITY;
          sc[t][x][i] = u;
          mx = fmaxf(mx, u);
        }
      }
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m[t], mx);
      const float base = mn == -INFINITY ? 0.0f : mn;  // (nothing unmasked so far)
      const float alpha = __builtin_amdgcn_exp2f(m[t] - base);
      m[t] = mn;
      float sum = 0.0f;
#pragma unroll
      for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f(sc[t][x][i] - base);
          sc[t][x][i] = e;
          sum += e;
        }
      l[t] = l[t] * alpha + sum;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[t][d] *= alpha;
    }
#pragma unroll
    for (int x = 0; x < KT / 2; ++x) {
      x8_t<T> pf[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) pf[t] = as_operand<T>(sc[t][2 * x], sc[t][2 * x + 1]);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const x8_t<T> vf = lds8<T>(Vt + (d * 16 + col) * LDV + x * 32 + g * 8);
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
    if (p.nsplit > 1) {
      const int64_t at = (int64_t)blockIdx.y * a.Nq * a.H + row;
#pragma unroll
      for (int d = 0; d < DT; ++d) store4<float>(p.part + at * D, d * 16 + g * 4, D, D % 4 == 0 ? 4 : 1, o[t][d]);
      if (g == 0) {
        p.part_ml[2 * at] = m[t];
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
      p.lse[row] = l[t] == 0.0f ? -INFINITY : (m[t] + log2f(l[t])) * kLn2;
  }
}

// Joins the parts of each (query, head): one wavefront a row, lanes over the
// columns. Rows outside every graph are left as they were.
template <typename T>
__global__ __launch_bounds__(kBlock) void attn_join(AttnFwd p) {
  const AttnShape& a = p.a;
  const int64_t rows = (int64_t)a.Nq * a.H;
  const int64_t row = (int64_t)blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave;
  const int q = (int)(row / a.H);
  if (row >= rows || q < a.qoff[0] || q >= a.qoff[a.G]) return;
  const int lane = lane_id();
  float m = -INFINITY;
  for (int sp = 0; sp < p.nsplit; ++sp) m = fmaxf(m, p.part_ml[2 * (sp * rows + row)]);
  const float base = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, acc[kMaxHeadDim / kWave] = {};
  for (int sp = 0; sp < p.nsplit; ++sp) {
    const float w = __builtin_amdgcn_exp2f(p.part_ml[2 * (sp * rows + row)] - base);
    l += w * p.part_ml[2 * (sp * rows + row) + 1];
#pragma unroll
    for (int c = 0; c < kMaxHeadDim / kWave; ++c)
      if (c * kWave + lane < a.D) acc[c] += w * p.part[(sp * rows + row) * a.D + c * kWave + lane];
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int c = 0; c < kMaxHeadDim / kWave; ++c)
    if (c * kWave + lane < a.D)
      static_cast<T*>(p.out)[row * a.D + c * kWave + lane] = to_type<T>(acc[c] * inv);
  if (p.lse != nullptr && lane == 0)
    p.lse[row] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <typename T, int DP, int WAVES, int QT>
int launch_fwd(AttnFwd& p, hipStream_t s) {
  constexpr int BM = WAVES * QT * 16;
  const int grp = p.a.H / p.a.Hk;
  p.slots = (int64_t)p.a.Nq * grp / BM + p.a.G;
  const int64_t blocks = p.slots * p.a.Hk;
  if (blocks >= (int64_t(1) << 31)) return fail(TFG_ERR_TOO_LARGE, "too many query tiles");
  attn_fwd<T, DP, WAVES, QT><<<dim3((unsigned)blocks, (unsigned)p.nsplit), WAVES * kWave,
                               sizeof(float) * (size_t)(grp * p.a.B), s>>>(p);
  TFG_LAUNCHED("attn_fwd");
  if (p.nsplit > 1) {
    const int64_t rows = (int64_t)p.a.Nq * p.a.H;
    attn_join<T><<<(unsigned)((rows + 3) / 4), kBlock, 0, s>>>(p);
    TFG_LAUNCHED("attn_join");
  }
  return TFG_OK;
}

template <typename T, int DP>
int launch_fwd_rows(AttnFwd& p, hipStream_t s) {
  const int64_t rows = (int64_t)p.a.Nq * (p.a.H / p.a.Hk) / std::max(p.a.G, 1);
  if (rows <= 16) return launch_fwd<T, DP, 1, 1>(p, s);
  if (rows <= 96) return launch_fwd<T, DP, 1, 2>(p, s);
  return launch_fwd<T, DP, 4, 2>(p, s);
}

template <typename T>
int launch_fwd_type(AttnFwd& p, hipStream_t s) {
  if (p.a.D <= 32) return launch_fwd_rows<T, 32>(p, s);
  if (p.a.D <= 64) return launch_fwd_rows<T, 64>(p, s);
  return launch_fwd_rows<T, 128>(p, s);
}

// Parts of the keys of each graph: more than one where the rows alone leave most
// of the card idle and graphs have many keys.
int key_parts(int64_t Nq, int64_t Nk, int64_t G, int64_t H, int64_t Hk) {
  if (G < 1 || Nq < 1) return 1;
  const int64_t grp = H / Hk, rows = Nq * grp / G;
  const int64_t tile = rows <= 16 ? 16 : rows <= 96 ? 32 : 128;
  const int64_t blocks = G * ((rows + tile - 1) / tile) * Hk;
  const int64_t keys = Nk / G;
  return (int)std::max<int64_t>(std::min<int64_t>({1024 / std::max<int64_t>(blocks, 1), keys / 256, 64}), 1);
}

}  // namespace

size_t attention_ws_bytes(int64_t Nq, int64_t Nk, int64_t G, int64_t H, int64_t Hk, int64_t D) {
  const int n = key_parts(Nq, Nk, G, H, Hk);
  return n > 1 ? sizeof(float) * (size_t)n * (size_t)(Nq * H) * (size_t)(D + 2) + 512 : 256;
}

int launch_attention(const AttnShape& a, int float_type, const void* q, const void* k,
                     const void* v, void* out, float* lse, void* ws, hipStream_t s) {
  if (a.G == 0 || a.Nq == 0) return TFG_OK;
  AttnFwd p{};
  p.a = a;
  p.q = q;
  p.k = k;
  p.v = v;
  p.out = out;
  p.lse = lse;
  p.nsplit = key_parts(a.Nq, a.Nk, a.G, a.H, a.Hk);
  if (p.nsplit > 1) {
    p.part = static_cast<float*>(ws);
    p.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) +
                                         align_up(sizeof(float) * (size_t)p.nsplit * a.Nq * a.H * a.D, 256));
  }
  const int64_t ldo = (int64_t)a.H * a.D;
  if (float_type == TFG_BF16) {
    p.vec_q = row_vector<__bf16>(q, a.ldq, a.D);
    p.vec_k = row_vector<__bf16>(k, a.ldk, a.D);
    p.vec_v = row_vector<__bf16>(v, a.ldv, a.D);
    p.vec_o = row_vector<__bf16>(out, ldo, a.D);
    return launch_fwd_type<__bf16>(p, s);
  }
  p.vec_q = row_vector<float>(q, a.ldq, a.D);
  p.vec_k = row_vector<float>(k, a.ldk, a.D);
  p.vec_v = row_vector<float>(v, a.ldv, a.D);
  p.vec_o = row_vector<float>(out, ldo, a.D);
  return launch_fwd_type<float>(p, s);
}

namespace {
__global__ __launch_bounds__(kBlock) void attn_check(AttnShape a, int* __restrict__ err) {
  const int g = blockIdx.x * kBlock + threadIdx.x;
  if (g > a.G) return;
  int bad = 0;
  const int q = a.qoff[g], k = a.koff[g];
  if (q < 0 || q > a.Nq || k < 0 || k > a.Nk) bad |= kErrIndex;
  if (g < a.G) {
    const int64_t nq = (int64_t)a.qoff[g + 1] - q, nk = (int64_t)a.koff[g + 1] - k;
    if (nq < 0 || nk < 0) bad |= kErrUnsorted;
    if (a.B > 0 && nq > 0 && nk > 0) {
      const int64_t o = a.doff[g];
      if (o < 0 || o > a.dist_bytes || nq * nk > a.dist_bytes - o) bad |= kErrIndex;
    }
  }
  if (bad != 0) atomicOr(err, bad);
}
}  // namespace

int launch_attention_check(const AttnShape& a, int* err, hipStream_t s) {
  if (int rc = launch_zero_flag(err, s)) return rc;
  attn_check<<<(unsigned)(a.G / kBlock + 1), kBlock, 0, s>>>(a, err);
  TFG_LAUNCHED("attn_check");
  return TFG_OK;
}

int max_attention_width() { return kMaxHeadDim; }
int max_attention_bias_entries() { return kMaxBiasEntries; }

}  // namespace tfg
