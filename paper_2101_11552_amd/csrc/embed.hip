// Rows of a table by id, and the table's gradient by sorted ids (gfx950).
//
// Forward: out[n] = scale * table[ids[n]], a row copy: bound by memory. A lane takes 16
// bytes of a row of any width; where the width is no multiple of that, the row's last
// lane steps back to end at its last column (and writes some again, the same).
//
// Gradient: dtable[v] = scale * sum of dout[n] over the n with ids[n] = v. The ids
// are sorted (stable, csr.hip), so that every row's terms are a run of sorted
// positions. The positions are cut into tiles of kEmbedTile, whatever the ids'
// distribution: a group of lanes adds the rows of its tile in order and writes
// every run that lies inside it; a run that crosses a tile's edge leaves float32
// partial rows, which a second kernel joins in tile order. Rows without ids get
// zeros. No atomics: the order of every sum is fixed by the ids.
//
// What bounds it: memory. 500,000 rows of 300 bf16 columns from 100,003, ids by Zipf's law:
// lookup 94 us (6.4 TB/s), sums by sorted ids 79, joins 23, the sort's three passes 72;
// 143,360 rows of 128 float32 columns from 119: 19, 17, 5 and 25.
#include "rows.h"

namespace tfg {

namespace {

constexpr int kEmbThreads = 256;
constexpr int kEmbRows = 4;     // rows in flight per thread (forward)
constexpr int kEmbedTile = 64;  // sorted positions of a tile
constexpr int kEmbU = 8;        // rows in flight per thread (gradient)
constexpr int kJoinU = 8;

template <typename T, int V, typename IdxT>
__global__ __launch_bounds__(kEmbThreads) void embed_rows(
    const T* __restrict__ table, int64_t ldt, int64_t rows, int F, const IdxT* __restrict__ ids,
    int64_t N, float scale, int64_t pad, T* __restrict__ out, int lpr, int rp, int* __restrict__ err) {
  const int r = threadIdx.x / lpr, sub = threadIdx.x - r * lpr;
  const int64_t n0 = (int64_t)blockIdx.x * (rp * kEmbRows) + r;
  if (r >= rp) return;
  int64_t id[kEmbRows];
  bool bad = false;
#pragma unroll
  for (int u = 0; u < kEmbRows; ++u) {
    const int64_t n = n0 + u * rp;
    id[u] = n < N ? (int64_t)ids[n] : 0;
  }
#pragma unroll
  for (int u = 0; u < kEmbRows; ++u) {
    const bool off = id[u] < 0 || id[u] >= rows;
    bad = bad || off;
    id[u] = off ? 0 : id[u] == pad ? -1 : id[u];  // (pad lies in the table, or is negative)
  }
  if (bad && err != nullptr && sub == 0 && blockIdx.y == 0) atomicOr(err, kErrIndex);
  const int cw = (blockIdx.y * lpr + sub) * V, c = min(cw, F - V);
  if (cw >= F) return;
  float x[kEmbRows][V];
#pragma unroll
  for (int u = 0; u < kEmbRows; ++u) {
#pragma unroll
    for (int v = 0; v < V; ++v) x[u][v] = 0.0f;
    if (id[u] >= 0 && n0 + u * rp < N) load_cols<T, V>(table + id[u] * ldt + c, x[u]);
  }
#pragma unroll
  for (int u = 0; u < kEmbRows; ++u)
    if (n0 + u * rp < N) {
#pragma unroll
      for (int v = 0; v < V; ++v) x[u][v] = id[u] >= 0 ? x[u][v] * scale : 0.0f;
      store_cols<T, V>(out + (n0 + u * rp) * F + c, x[u]);
    }
}

struct EmbedGrad {
  const void* dout;
  const int *key, *perm, *rowptr;
  int64_t N, rows, pad;
  int F, lpr, rp;
  float scale;
  float *head, *tail;  // [tiles][F]
  void* dtable;
};

// Tiles of sorted positions; see the top of the file. A run that began before the
// tile goes to head[tile] (also where it goes on behind it), one that begins in it
// and goes on behind it to tail[tile].
template <typename T, int V>
__global__ __launch_bounds__(kEmbThreads) void embed_grad_tiles(EmbedGrad p) {
  const int r = threadIdx.x / p.lpr, sub = threadIdx.x - r * p.lpr;
  const int64_t tile = (int64_t)blockIdx.x * p.rp + r;
  const int64_t b = tile * kEmbedTile;
  const int cw = (blockIdx.y * p.lpr + sub) * V, c = min(cw, p.F - V);
  if (r >= p.rp || b >= p.N || cw >= p.F) return;
  const int64_t e = min(b + kEmbedTile, p.N);
  const T* dout = static_cast<const T*>(p.dout);
  T* dtable = static_cast<T*>(p.dtable);
  int cur = p.key[b];
  bool whole = b == 0 || p.key[b - 1] != cur;  // the run starts here
  const int after = e < p.N ? p.key[e] : -1;
  float acc[V];
#pragma unroll
  for (int v = 0; v < V; ++v) acc[v] = 0.0f;
  const auto flush = [&](bool ends) {
    if (whole && ends) {
      if (cur == p.pad) return;
      float y[V];
#pragma unroll
      for (int v = 0; v < V; ++v) y[v] = acc[v] * p.scale;
      store_cols<T, V>(dtable + (int64_t)cur * p.F + c, y);
    } else {
      float* to = (whole ? p.tail : p.head) + tile * p.F + c;
#pragma unroll
      for (int v = 0; v < V; ++v) to[v] = acc[v];
    }
  };
  // the ids and places of the next rows are loaded while these are added
  int kn[kEmbU], an[kEmbU];
#pragma unroll
  for (int u = 0; u < kEmbU; ++u) {
    const int64_t n = min(b + u, e - 1);
    kn[u] = p.key[n];
    an[u] = p.perm[n];
  }
  for (int64_t n0 = b; n0 < e; n0 += kEmbU) {
    int k[kEmbU], at[kEmbU];
    float x[kEmbU][V];
#pragma unroll
    for (int u = 0; u < kEmbU; ++u) {
      k[u] = kn[u];
      at[u] = an[u];
    }
#pragma unroll
    for (int u = 0; u < kEmbU; ++u) load_cols<T, V>(dout + (int64_t)at[u] * p.F + c, x[u]);
    if (n0 + kEmbU < e) {
#pragma unroll
      for (int u = 0; u < kEmbU; ++u) {
        const int64_t n = min(n0 + kEmbU + u, e - 1);
        kn[u] = p.key[n];
        an[u] = p.perm[n];
      }
    }
#pragma unroll
    for (int u = 0; u < kEmbU; ++u)
      if (n0 + u < e) {
        if (k[u] != cur) {
          flush(true);
          cur = k[u];
          whole = true;
#pragma unroll
          for (int v = 0; v < V; ++v) acc[v] = 0.0f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] += x[u][v];
      }
  }
  flush(after != cur);
}

// V floats at any address of one.
template <int V>
__device__ __forceinline__ void load_floats(const float* p, float (&x)[V]) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int h = 0; h < V; h += 4) {
      const f32x4 t = *reinterpret_cast<const any4_t<float>*>(p + h);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[h + i] = t[i];
    }
  } else {
    x[0] = *p;
  }
}

// Runs over several tiles: the block of the tile in which a run starts and that it
// leaves adds tail[tile] and the heads of the tiles behind it, rp groups of lanes
// each every rp-th head, joined in order.
template <typename T, int V>
__global__ __launch_bounds__(kEmbThreads) void embed_grad_join(EmbedGrad p) {
  __shared__ float part[kEmbThreads * V];
  const int64_t tile = blockIdx.x, e = (tile + 1) * kEmbedTile;
  if (e >= p.N) return;
  const int id = p.key[e - 1];
  if (p.key[e] != id || id == p.pad) return;
  const int64_t b = p.rowptr[id], end = p.rowptr[id + 1];
  if (b / kEmbedTile != tile) return;  // it starts in an earlier tile
  const int64_t last = (end - 1) / kEmbedTile;
  const int r = threadIdx.x / p.lpr, sub = threadIdx.x - r * p.lpr;
  const int cw = (blockIdx.y * p.lpr + sub) * V, c = min(cw, p.F - V);
  const bool on = r < p.rp && cw < p.F;
  float acc[kJoinU][V];
#pragma unroll
  for (int u = 0; u < kJoinU; ++u)
#pragma unroll
    for (int v = 0; v < V; ++v) acc[u][v] = 0.0f;
  if (on) {
    for (int64_t t = tile + 1 + r; t <= last; t += kJoinU * p.rp) {
      float x[kJoinU][V];
#pragma unroll
      for (int u = 0; u < kJoinU; ++u) load_floats<V>(p.head + min(t + u * p.rp, last) * p.F + c, x[u]);
#pragma unroll
      for (int u = 0; u < kJoinU; ++u)
#pragma unroll
        for (int v = 0; v < V; ++v) acc[u][v] += t + u * p.rp <= last ? x[u][v] : 0.0f;
    }
#pragma unroll
    for (int h = kJoinU / 2; h > 0; h >>= 1)
#pragma unroll
      for (int u = 0; u < h; ++u)
#pragma unroll
        for (int v = 0; v < V; ++v) acc[u][v] += acc[u + h][v];
#pragma unroll
    for (int v = 0; v < V; ++v) part[(r * p.lpr + sub) * V + v] = acc[0][v];
  }
  __syncthreads();
  if (!on || r != 0) return;
  float y[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float t = p.tail[tile * p.F + c + v];
    for (int j = 0; j < p.rp; ++j) t += part[(j * p.lpr + sub) * V + v];
    y[v] = t * p.scale;
  }
  store_cols<T, V>(static_cast<T*>(p.dtable) + (int64_t)id * p.F + c, y);
}

// Zeros to the rows without ids and to the padding's.
template <typename T, int V>
__global__ __launch_bounds__(kEmbThreads) void embed_grad_zero(EmbedGrad p) {
  const int r = threadIdx.x / p.lpr, sub = threadIdx.x - r * p.lpr;
  const int64_t v0 = ((int64_t)blockIdx.x * p.rp + r) * kEmbRows;
  const int cw = (blockIdx.y * p.lpr + sub) * V, c = min(cw, p.F - V);
  if (r >= p.rp || cw >= p.F) return;
  float zero[V];
#pragma unroll
  for (int v = 0; v < V; ++v) zero[v] = 0.0f;
#pragma unroll
  for (int u = 0; u < kEmbRows; ++u)
    if (v0 + u < p.rows && (p.rowptr[v0 + u] == p.rowptr[v0 + u + 1] || v0 + u == p.pad))
      store_cols<T, V>(static_cast<T*>(p.dtable) + (v0 + u) * p.F + c, zero);
}

// Lanes a row and rows a block for F columns, V a lane.
struct Lanes {
  int lpr, rp;
  unsigned slabs;
};
Lanes lanes_of(int64_t F, int V) {
  Lanes l;
  const int64_t n = (F + V - 1) / V;
  l.lpr = (int)std::min<int64_t>(n, kEmbThreads);
  l.rp = kEmbThreads / l.lpr;
  l.slabs = (unsigned)((n + l.lpr - 1) / l.lpr);
  return l;
}

template <typename T, int V>
int launch_embed_cols(const Embed& a, int* err, hipStream_t s) {
  const Lanes l = lanes_of(a.F, V);
  const int64_t per = (int64_t)l.rp * kEmbRows;
  const dim3 grid((unsigned)((a.N + per - 1) / per), l.slabs);
  if (a.index_type == TFG_I64)
    embed_rows<T, V, int64_t><<<grid, kEmbThreads, 0, s>>>(
        static_cast<const T*>(a.table), a.ldt, a.V, (int)a.F, static_cast<const int64_t*>(a.ids), a.N,
        a.scale, a.pad, static_cast<T*>(a.out), l.lpr, l.rp, err);
  else
    embed_rows<T, V, int32_t><<<grid, kEmbThreads, 0, s>>>(
        static_cast<const T*>(a.table), a.ldt, a.V, (int)a.F, static_cast<const int32_t*>(a.ids), a.N,
        a.scale, a.pad, static_cast<T*>(a.out), l.lpr, l.rp, err);
  TFG_LAUNCHED("embed_rows");
  return TFG_OK;
}

template <typename T>
int launch_embed_type(const Embed& a, int* err, hipStream_t s) {
  return a.F >= vector_cols<T>() ? launch_embed_cols<T, vector_cols<T>()>(a, err, s)
                                 : launch_embed_cols<T, 1>(a, err, s);
}

template <typename T, int V>
int launch_grad_cols(EmbedGrad p, hipStream_t s) {
  const Lanes l = lanes_of(p.F, V);
  p.lpr = l.lpr;
  p.rp = l.rp;
  const int64_t tiles = (p.N + kEmbedTile - 1) / kEmbedTile;
  if (tiles > 0) {
    embed_grad_tiles<T, V><<<dim3((unsigned)((tiles + l.rp - 1) / l.rp), l.slabs), kEmbThreads, 0, s>>>(p);
    embed_grad_join<T, V><<<dim3((unsigned)tiles, l.slabs), kEmbThreads, 0, s>>>(p);
  }
  const int64_t per = (int64_t)l.rp * kEmbRows;
  embed_grad_zero<T, V><<<dim3((unsigned)((p.rows + per - 1) / per), l.slabs), kEmbThreads, 0, s>>>(p);
  TFG_LAUNCHED("embed_grad");
  return TFG_OK;
}

template <typename T>
int launch_grad_type(const EmbedGrad& p, hipStream_t s) {
  return p.F >= vector_cols<T>() ? launch_grad_cols<T, vector_cols<T>()>(p, s) : launch_grad_cols<T, 1>(p, s);
}

struct EmbedLayout {
  size_t err, key, perm, col, rowptr, sort, head, tail, total;
};
EmbedLayout embed_layout(int64_t N, int64_t V, int64_t F) {
  EmbedLayout L;
  size_t off = 256;
  const auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes, 256);
    return at;
  };
  const int64_t tiles = (N + kEmbedTile - 1) / kEmbedTile;
  L.err = 0;
  L.key = take(sizeof(int) * (size_t)N);
  L.perm = take(sizeof(int) * (size_t)N);
  L.col = take(sizeof(int) * (size_t)N);
  L.rowptr = take(sizeof(int) * (size_t)(V + 1));
  L.sort = take(sort_ids_scratch_bytes(N, V));
  L.head = take(sizeof(float) * (size_t)(tiles * F));
  L.tail = take(sizeof(float) * (size_t)(tiles * F));
  L.total = off;
  return L;
}

}  // namespace

size_t embedding_backward_ws_bytes(int64_t N, int64_t V, int64_t F) {
  return embed_layout(N, V, F).total;
}

int launch_embedding(const Embed& a, int* err, hipStream_t s) {
  if (err != nullptr)
    if (int rc = launch_zero_flag(err, s)) return rc;
  if (a.N == 0 || a.F == 0) return TFG_OK;
  return a.float_type == TFG_BF16 ? launch_embed_type<__bf16>(a, err, s)
                                  : launch_embed_type<float>(a, err, s);
}

int launch_embedding_backward(const Embed& a, const void* dout, void* dtable, void* ws, int* err,
                              hipStream_t s) {
  if (err != nullptr)
    if (int rc = launch_zero_flag(err, s)) return rc;
  if (a.V == 0 || a.F == 0) return TFG_OK;
  const EmbedLayout L = embed_layout(a.N, a.V, a.F);
  char* w = static_cast<char*>(ws);
  EmbedGrad p{};
  int* key = reinterpret_cast<int*>(w + L.key);
  int* perm = reinterpret_cast<int*>(w + L.perm);
  int* rowptr = reinterpret_cast<int*>(w + L.rowptr);
  if (int rc = sort_ids(a.ids, a.index_type, a.N, a.V, key, perm, rowptr,
                        reinterpret_cast<int*>(w + L.col), w + L.sort, err, s))
    return rc;
  p.dout = dout;
  p.key = key;
  p.perm = perm;
  p.rowptr = rowptr;
  p.N = a.N;
  p.rows = a.V;
  p.pad = a.pad;
  p.F = (int)a.F;
  p.scale = a.scale;
  p.head = reinterpret_cast<float*>(w + L.head);
  p.tail = reinterpret_cast<float*>(w + L.tail);
  p.dtable = dtable;
  return a.float_type == TFG_BF16 ? launch_grad_type<__bf16>(p, s) : launch_grad_type<float>(p, s);
}

}  // namespace tfg
