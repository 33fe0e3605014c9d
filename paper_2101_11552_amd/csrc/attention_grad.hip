// The attention's gradients inside each graph (gfx950): workspace and launches. The
// kernels are in attention_grad.h and attention_grad_small.h.
#include "attention_grad_launch.h"

namespace tfg {
namespace {

constexpr size_t kMaxLds = 160 << 10;

// A launch that fills the card has some kBlocks blocks.
constexpr int64_t kBlocks = 768;

// Two row tiles a wavefront read each staged tile of keys once for both, where that costs
// no wavefront a SIMD (bf16 heads of 33 to 64 columns: two wavefronts either way, 455 -> 425
// us for 96 graphs of 100 to 500 nodes, 8 heads; float32 of up to 16, 666 -> 609) and the
// blocks still fill the card. Elsewhere it does (bf16 of 17 to 32: three to two, 295 -> 324).
// Two key tiles a wavefront always do, or gain nothing.
bool two_row_tiles(int float_type, int64_t D) {
  return float_type == TFG_BF16 ? D > 32 && D <= 64 : D <= 16;
}

RowPlan row_plan(const AttnShape& a, int float_type, bool want_bias) {
  const int64_t Nq = a.Nq, Nk = a.Nk, G = a.G, H = a.H, Hk = a.Hk, D = a.D, B = a.B;
  const int64_t grp = H / Hk, graphs = std::max<int64_t>(G, 1), rows = Nq * grp / graphs;
  RowPlan r{1, 1, 1, 1, 0, 0, 0, 0};
  const SmallPlan sp = small_grad_plan(float_type, a, want_bias);
  r.small_waves = sp.waves;
  r.small_block = sp.per_block;
  r.small_lds = sp.lds;
  if (rows > 16 || sp.waves > 0) r.waves = 4;
  if (sp.waves == 0 && rows > 192 && two_row_tiles(float_type, D) && D % (float_type == TFG_BF16 ? 8 : 4) == 0 && rows / 128 * graphs * Hk >= kBlocks) r.qt = 2;
  if (16 % grp != 0) r.copies = r.qt;
  // the LDS of the tiles (three of 64 x DP bf16 or 32 x DP float32), the bias table and the bins
  const int64_t DP = D <= 16 ? 16 : D <= 32 ? 32 : D <= 64 ? 64 : 128;
  const size_t tiles = 3 * 2 * 64 * (size_t)(DP + 16) + 2 * 8 * (size_t)DP;
  if (tiles + sizeof(float) * (size_t)(grp * (B + 1)) + bins_bytes(r.waves, r.copies, B) > kMaxLds)
    r.waves = r.qt = r.copies = 1;
  r.slots = sp.waves > 0 ? kRestBlocks : Nq * grp / (r.waves * r.qt * 16) + G;
  const int64_t keys = Nk / graphs;
  // the queries of a key tile in parts of at least four tiles of rows
  const int64_t blocks = std::max<int64_t>(keys / 64, 1) * graphs * Hk;
  const int64_t tiles_of_rows = (Nq / graphs + 63) / 64 * grp;
  if (sp.waves == 0) r.nsplit = (int)std::max<int64_t>(std::min<int64_t>({kBlocks / blocks, tiles_of_rows / 4, 16}), 1);
  return r;
}

struct GradLayout {
  size_t a, c, delta, part, sums, keys, total;
};
// Rows of partial bias gradients: of the tiles of rows, then of the wavefronts over small graphs.
int64_t bias_rows(const RowPlan& r, int64_t Hk) { return r.slots + r.small_waves / Hk; }

GradLayout grad_layout(int64_t Nq, int64_t keys, int64_t H, int64_t Hk, int64_t B, const RowPlan& r) {
  GradLayout L;
  const size_t rows = align_up(sizeof(float) * (size_t)(Nq * H), 256);
  L.a = 0;
  L.c = rows;
  L.delta = 2 * rows;
  L.part = 3 * rows;
  L.sums = L.part + align_up(sizeof(float) * (size_t)(B > 0 ? bias_rows(r, Hk) * H * B : 0), 256);
  L.keys = L.sums + align_up(B > 0 ? column_sums_bytes(bias_rows(r, Hk), H * B) : 0, 256);
  L.total = L.keys + align_up(r.nsplit > 1 ? 2 * sizeof(float) * (size_t)(r.nsplit * keys) : 0, 256) + 256;
  return L;
}

}  // namespace

size_t attention_backward_ws_bytes(int float_type, int64_t Nq, int64_t Nk, int64_t G, int64_t H, int64_t Hk,
                                   int64_t D, int64_t B) {
  AttnShape a{};
  a.Nq = (int)Nq;
  a.Nk = (int)Nk;
  a.G = (int)G;
  a.H = (int)H;
  a.Hk = (int)Hk;
  a.D = (int)D;
  a.B = (int)B;
  // (with or without the bias's gradient the tiles may differ)
  size_t most = 0;
  for (const bool want : {false, true})
    most = std::max(most, grad_layout(Nq, Nk * Hk * D, H, Hk, B, row_plan(a, float_type, want && B > 0)).total);
  return most;
}

int launch_attention_backward(const AttnShape& a, int float_type, const void* q, const void* k,
                              const void* v, const void* out, const float* lse, const void* dout,
                              void* dq, void* dk, void* dv, void* dbias, void* ws, hipStream_t s) {
  if (a.G == 0 && dbias == nullptr) return TFG_OK;
  const RowPlan r = row_plan(a, float_type, dbias != nullptr);
  const GradLayout L = grad_layout(a.Nq, (int64_t)a.Nk * a.Hk * a.D, a.H, a.Hk, a.B, r);
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
  p.row_a = reinterpret_cast<float*>(w + L.a);
  p.row_c = reinterpret_cast<float*>(w + L.c);
  p.row_delta = reinterpret_cast<float*>(w + L.delta);
  p.bias_part = dbias != nullptr ? reinterpret_cast<float*>(w + L.part) : nullptr;
  p.copies = r.copies;
  p.nsplit = r.nsplit;
  p.part = reinterpret_cast<float*>(w + L.keys);
  const bool narrow = a.D <= 32;
  int rc;
  if (float_type == TFG_BF16) rc = narrow ? launch_grad_bf16_narrow(p, r, s) : launch_grad_bf16_wide(p, r, s);
  else rc = narrow ? launch_grad_f32_narrow(p, r, s) : launch_grad_f32_wide(p, r, s);
  if (rc || dbias == nullptr) return rc;
  // (no queries: no rows to add, zeros)
  double* sums = reinterpret_cast<double*>(w + L.sums);
  const int64_t slots = p.a.Nq == 0 ? 0 : bias_rows(r, a.Hk);
  if (float_type == TFG_BF16)
    return launch_column_sums(p.bias_part, slots, a.H * a.B, static_cast<__bf16*>(dbias), sums, s);
  return launch_column_sums(p.bias_part, slots, a.H * a.B, static_cast<float*>(dbias), sums, s);
}

}  // namespace tfg
