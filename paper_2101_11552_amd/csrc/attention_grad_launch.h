// The choice among the attention's gradient kernels (gfx950).
#pragma once

#include "attention_grad_small.h"

namespace tfg {

template <typename T, int DP>
int launch_grad_width(AttnGrad& p, const RowPlan& r, hipStream_t s) {
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
  p.heads = 1;
  p.small = 0;
  if constexpr (DP * sizeof(T) <= 128) {
    if (r.small_waves > 0) {
      AttnGrad q = p;
      q.bias_part = p.bias_part != nullptr ? p.bias_part + r.slots * p.a.H * p.a.B : nullptr;
      if (int rc = launch_grad_small<T, DP>(q, SmallPlan{r.small_waves, r.small_block, r.small_lds}, s)) return rc;
      p.small = kSmallGraph;  // the rest: graphs with more nodes, few if any
      p.heads = p.a.Hk;
      if (r.waves == 1) {
        if (int rc = launch_grad_q<T, DP, 1, 1, 0, true>(p, r.slots, s)) return rc;
      } else if (int rc = launch_grad_q<T, DP, 4, 1, 8, true>(p, r.slots, s)) {
        return rc;
      }
      return launch_grad_kv<T, DP, 4, 1, 8, true>(p, s);
    }
  }
  const bool whole = whole_vectors<T>(D);
  if (p.a.Nq > 0) {
    int rc;
    constexpr int QT = (sizeof(T) == 2 ? DP == 64 : DP == 16) ? 2 : 1;  // (the plan's widths)
    if (r.waves == 1) rc = launch_grad_q<T, DP, 1, 1, 0>(p, r.slots, s);
    else if (!whole) rc = launch_grad_q<T, DP, 4, 1, 0>(p, r.slots, s);
    else if (r.qt == 2) rc = launch_grad_q<T, DP, 4, QT, 8>(p, r.slots, s);
    else rc = launch_grad_q<T, DP, 4, 1, 8>(p, r.slots, s);
    if (rc) return rc;
  }
  if (p.a.Nk == 0) return TFG_OK;
  if (!whole) return launch_grad_kv<T, DP, 4, 1, 0>(p, s);
  return launch_grad_kv<T, DP, 4, 1, 8>(p, s);
}

// Heads of at most 32 columns, and wider ones (translation units of their own).
template <typename T>
int launch_grad_narrow(AttnGrad& p, const RowPlan& r, hipStream_t s) {
  return p.a.D <= 16 ? launch_grad_width<T, 16>(p, r, s) : launch_grad_width<T, 32>(p, r, s);
}
template <typename T>
int launch_grad_wide(AttnGrad& p, const RowPlan& r, hipStream_t s) {
  return p.a.D <= 64 ? launch_grad_width<T, 64>(p, r, s) : launch_grad_width<T, 128>(p, r, s);
}
#define TFG_ATTN_GRAD(name) int launch_grad_##name(AttnGrad& p, const RowPlan& r, hipStream_t s)
TFG_ATTN_GRAD(bf16_narrow);
TFG_ATTN_GRAD(bf16_wide);
TFG_ATTN_GRAD(f32_narrow);
TFG_ATTN_GRAD(f32_wide);

}  // namespace tfg
