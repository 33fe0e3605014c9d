// Column sums of a tall matrix in a fixed order, in double (gfx950): the rows'
// partial results of gradients that belong to no row.
#pragma once

#include "wave.h"

namespace tfg {

constexpr int kSumLanes = 4;  // row lanes of a block, 64 columns each

// out[group][c] = sum of the group's rows of in[rows][n]: lane y takes the rows
// y, y + 4, .. of the group, the four lanes' sums are added in order.
template <typename In, typename Out>
__global__ __launch_bounds__(kWave* kSumLanes) void column_sums(const In* __restrict__ in,
                                                               int64_t rows, int n, int64_t per,
                                                               Out* __restrict__ out) {
  __shared__ double part[kSumLanes][kWave];
  const int x = threadIdx.x & (kWave - 1), y = threadIdx.x / kWave;
  const int c = blockIdx.x * kWave + x;
  const int64_t r0 = blockIdx.y * per, r1 = min(r0 + per, rows);
  double acc[4] = {};
  if (c < n)
    for (int64_t r = r0 + y; r < r1; r += 8 * kSumLanes) {
      In x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = in[min(r + u * kSumLanes, r1 - 1) * n + c];
#pragma unroll
      for (int u = 0; u < 8; ++u) acc[u % 4] += r + u * kSumLanes < r1 ? (double)x[u] : 0.0;
    }
  part[y][x] = (acc[0] + acc[1]) + (acc[2] + acc[3]);
  __syncthreads();
  if (y == 0 && c < n)
    out[(int64_t)blockIdx.y * n + c] = (Out)((part[0][x] + part[1][x]) + (part[2][x] + part[3][x]));
}

// Groups of rows of the first of the two sums, and the bytes of its results.
inline int64_t column_groups(int64_t rows) {
  return std::max<int64_t>(std::min<int64_t>((rows + 63) / 64, 64), 1);
}
inline size_t column_sums_bytes(int64_t rows, int64_t n) {
  return sizeof(double) * (size_t)(column_groups(rows) * n);
}

// out[c] = sum of in[rows][n] over the rows; ws: column_sums_bytes(rows, n).
template <typename In, typename Out>
int launch_column_sums(const In* in, int64_t rows, int n, Out* out, double* ws, hipStream_t s) {
  if (n == 0) return TFG_OK;
  const unsigned nb = (unsigned)((n + kWave - 1) / kWave);
  const int64_t groups = column_groups(rows), per = (rows + groups - 1) / groups;
  column_sums<In, double><<<dim3(nb, (unsigned)groups), kWave * kSumLanes, 0, s>>>(in, rows, n, per, ws);
  column_sums<double, Out><<<dim3(nb, 1), kWave * kSumLanes, 0, s>>>(ws, groups, n, groups, out);
  TFG_LAUNCHED("column_sums");
  return TFG_OK;
}

}  // namespace tfg
