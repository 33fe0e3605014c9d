// The choice among the forward attention kernels (gfx950).
#pragma once

#include "attention_small.h"

namespace tfg {

// Tiles of 64 rows, or of 16 for a few queries each. Of 128, two row tiles a wavefront, for
// bf16 heads of 33 to 64 columns and graphs of a thousand rows and more: two wavefronts a
// SIMD either way there (three graphs of 4,000 to 9,000 nodes, 8 heads of 64, 556 -> 526 us;
// 96 graphs of 100 to 500: 120 -> 129; other widths lose a wavefront: 16 columns 377 -> 383,
// 128 905 -> 1,020).
template <typename T, int DP>
int launch_fwd_rows(AttnFwd& p, hipStream_t s) {
  const int64_t rows = (int64_t)p.a.Nq * (p.a.H / p.a.Hk) / std::max(p.a.G, 1);
  const int D = p.a.D;
  p.vec_q = row_vector<T>(p.q, p.a.ldq, D);
  p.vec_o = row_vector<T>(p.out, (int64_t)p.a.H * D, D);
  p.heads = 1;
  p.small = 0;
  const bool whole = whole_vectors<T>(D);
  if (p.nsplit == 1 && whole && small_graphs(p.a.Nq, p.a.Nk, p.a.G, p.a.Hk) && small_fits<T, DP>(p.a)) {
    if (int rc = launch_small<T, DP>(p, s)) return rc;
    p.small = kSmallGraph;  // the rest: graphs with more nodes, few if any
    p.heads = p.a.Hk;
    return launch_fwd<T, DP, 4, 1, 8, true>(p, s);
  }
  if (!whole) return rows <= 16 ? launch_fwd<T, DP, 1, 1, 0>(p, s) : launch_fwd<T, DP, 4, 1, 0>(p, s);
  if (rows <= 16) return launch_fwd<T, DP, 1, 1, 8>(p, s);
  if constexpr (DP == 64 && sizeof(T) == 2)
    if (rows >= 1024 && rows / 128 * p.a.G * p.a.Hk >= 768) return launch_fwd<T, DP, 4, 2, 8>(p, s);
  return launch_fwd<T, DP, 4, 1, 8>(p, s);
}

// Heads of at most 32 columns, and wider ones (translation units of their own).
template <typename T>
int launch_fwd_narrow(AttnFwd& p, hipStream_t s) {
  return p.a.D <= 16 ? launch_fwd_rows<T, 16>(p, s) : launch_fwd_rows<T, 32>(p, s);
}
template <typename T>
int launch_fwd_wide(AttnFwd& p, hipStream_t s) {
  return p.a.D <= 64 ? launch_fwd_rows<T, 64>(p, s) : launch_fwd_rows<T, 128>(p, s);
}
#define TFG_ATTN_FWD(name) int launch_fwd_##name(AttnFwd& p, hipStream_t s)
TFG_ATTN_FWD(bf16_narrow);
TFG_ATTN_FWD(bf16_wide);
TFG_ATTN_FWD(f32_narrow);
TFG_ATTN_FWD(f32_wide);

}  // namespace tfg
