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

}  // namespace scmoe
