// Tiles of rows over graphs of any sizes, without a list and without the sizes on
// the host (gfx950).
//
// off[G + 1] are the graphs' first rows (of `mul` rows each). Graph g owns the
// slots from s(g) = floor(off[g] * mul / TILE) + g on: floor(a + n) - floor(a) + 1 is
// at least the ceil(rows / TILE) tiles that it needs, so that a grid of
// floor(rows / TILE) + G slots covers every batch, with at most one slot a graph
// idle, and a slot finds its graph by searching the offsets.
#pragma once

#include "wave.h"

namespace tfg {

struct Run {
  int g, tile;  // graph (< 0: none) and tile of it
};

__device__ __forceinline__ int clamp_off(int v, int n) { return v < 0 ? 0 : (v > n ? n : v); }

template <int TILE>
__device__ __forceinline__ int64_t first_slot(const int* off, int g, int n_off, int mul) {
  return (int64_t)clamp_off(off[g], n_off) * mul / TILE + g;
}

// The graph of a slot: 64 lanes probe 64 graphs at a time (two rounds of loads for
// 4,096 graphs). Every lane of the wavefront calls it with the same arguments.
// Offsets that decrease give some graph in [0, G).
template <int TILE>
__device__ __forceinline__ Run find_run(const int* off, int G, int n_off, int mul, int64_t slot) {
  int lo = 0, hi = G;
  while (true) {
    const int step = (hi - lo + kWave - 1) / kWave;
    const int at = lo + lane_id() * step;
    const bool le = at < hi && first_slot<TILE>(off, at, n_off, mul) <= slot;
    const int cnt = __popcll(__ballot(le));
    if (cnt == 0) return Run{-1, 0};  // (the first graph starts behind this slot)
    lo = uniform(lo + (cnt - 1) * step);
    hi = uniform(min(lo + step, hi));
    if (step == 1) break;
  }
  const int64_t tile = slot - first_slot<TILE>(off, lo, n_off, mul);
  if (tile < 0) return Run{-1, 0};  // (only where the offsets decrease)
  return Run{lo, (int)tile};
}

}  // namespace tfg
