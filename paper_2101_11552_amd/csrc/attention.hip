// Attention inside each graph of a BatchGraph (gfx950): the choice of kernels and the
// check of offsets. The kernels are in attention_fwd.h and
// attention_small.h.
#include <limits>

#include "attention_launch.h"

namespace tfg {
namespace {

// Parts of the keys of each graph: more than one where the rows alone leave most
// of the card idle and graphs have many keys.
int key_parts(int64_t Nq, int64_t Nk, int64_t G, int64_t H, int64_t Hk) {
  if (G < 1 || Nq < 1 || small_graphs(Nq, Nk, G, Hk)) return 1;
  const int64_t grp = H / Hk, rows = Nq * grp / G;
  const int64_t tile = rows <= 16 ? 16 : 64;
  const int64_t blocks = G * ((rows + tile - 1) / tile) * Hk;
  const int64_t keys = Nk / G;
  return (int)std::max<int64_t>(std::min<int64_t>({1024 / std::max<int64_t>(blocks, 1), keys / 256, kKeyParts}), 1);
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
  // masked scores are raw products of -inf, which a scale of zero would make NaN
  if (a.scale == 0.0f) p.a.scale = std::numeric_limits<float>::denorm_min();
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
  const bool narrow = a.D <= 32;
  if (float_type == TFG_BF16) return narrow ? launch_fwd_bf16_narrow(p, s) : launch_fwd_bf16_wide(p, s);
  return narrow ? launch_fwd_f32_narrow(p, s) : launch_fwd_f32_wide(p, s);
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
