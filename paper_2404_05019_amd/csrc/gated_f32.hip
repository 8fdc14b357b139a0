// The gated feed-forward block's products in fp32 (gated_tiles.hpp).
#include "gated_tiles.hpp"

namespace scmoe {

using GatedF = GatedCfg<true, 128, 128, 2, 2, 2>;    // 4 waves of 64 x 64, 64 KiB LDS, two workgroups per CU
using GatedD = GatedCfg<true, 64, 64, 4, 1, 2>;      // the same with 32 KiB, four workgroups per CU: for DW, whose k is a segment's rows
using GatedG = GatedCfg<true, 64, 64, 4, 1, 3>;

// The larger tiles, which read less per product, where they come to eight rounds (of two a compute unit) and more, or to two with a long K;
// else the smaller ones, of which more are under way at a time.  us of a forward call / a gradient, all products on larger | smaller tiles:
// 16384 rows, d = 1024, F = 4096, E = 8 2905 / 5826 | 3020 / 6376; 16384, d = 384, F = 1536 525 / 1166 | 470 / 952; 4096, d = 1024, F = 2048
// 408 / 797 | 381 / 755; 777, d = 1000, F = 1360, E = 5 163 / 336 | 85 / 175; 40, d = 1024, F = 4096, E = 8 382 / 679 | 148 / 319.
int launch_gated_f32(const GatedArgs& a, int mode, int keep, int64_t max_rows, hipStream_t stream) {
  constexpr int B = GatedF::BM, BN = GatedF::BN;
  double tiles = 0;
  for (const GatedJob& j : a.j) {
    if (j.C == nullptr) continue;
    const double across = mode == G_GATE ? (2.0 * j.N + BN - 1) / BN : (j.N + BN - 1) / BN;
    tiles += across * (mode == G_DW ? static_cast<double>((j.M + B - 1) / B) * a.E : static_cast<double>(max_rows) / B + 0.5 * static_cast<double>(a.E < max_rows ? a.E : max_rows));
  }
  const double rounds = tiles / (2.0 * num_cus());
  if (rounds >= 8.0 || (mode != G_DW && rounds >= 2.0 && a.j[0].Kd >= 4096)) return launch_gated_mode<GatedF>(a, mode, keep, max_rows, stream);
  if (mode == G_DW) return launch_gated_cfg<GatedD, G_DW, KEEP_NONE, 0>(a, max_rows, stream);   // (777 rows 165 / 160, 2000, d = 512, F = 1024, E = 16 180 / 175)
  return launch_gated_rows<GatedG>(a, mode, keep, max_rows, stream);
}

// DX and DW in one launch, where DX has up to two tiles of 64 x 64 a compute unit (its own launch has three), and DW up to 24 rounds.  DX's tiles with three
// stages, three workgroups a unit, up to 0.6 tiles a unit, where a tile's time counts; else two stages and four workgroups.  us of a
// gradient, two launches / so with three stages / with two: 100 rows, d = 512, F = 2048, E = 8 125 / 111 / 136; 500, 384, 1536, 8 110 / 95 / 108; 16, 1024, 4096, 8
// 280 / 266 / 310; 777, 1000, 1360, 5 164 / 158 / 152; 1000, 1024, 2048, 8 315 / 287 / 282; 5000, 256, 1024, 4 176 / 163 / 160; 300, 1024, 2048, 16 240 / 264 /
// 242; more tiles: 2000, 1024, 2048, 8 429 / 453 / 432; 16384, 384, 1536, 8 933 / 966 / 946.
int launch_gated_gradients_f32(const GatedArgs& x, const GatedArgs& w, int64_t max_rows, hipStream_t stream) {
  const double cus = num_cus(), tx = likely_tiles(x, G_DX, max_rows, 64, 64);
  if (tx <= 2.0 * cus && likely_tiles(w, G_DW, max_rows, 64, 64) <= 24.0 * 4.0 * cus)
    return tx <= 0.6 * cus ? launch_gated_pair<GatedG, GatedD>(x, w, max_rows, stream) : launch_gated_pair<GatedD, GatedD>(x, w, max_rows, stream);
  const int st = launch_gated_f32(w, G_DW, KEEP_NONE, max_rows, stream);
  return st == SCMOE_OK ? launch_gated_f32(x, G_DX, KEEP_NONE, max_rows, stream) : st;
}

}  // namespace scmoe
