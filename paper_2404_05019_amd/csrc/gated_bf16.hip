// The gated feed-forward block's products in bf16 (gated_tiles.hpp).
#include "gated_tiles.hpp"
#include <math.h>

namespace scmoe {

using GatedA = GatedCfg<false, 256, 256, 2, 4, 2>;   // 8 waves of 128 x 64, 128 KiB LDS, one workgroup per CU
using GatedU = GatedCfg<false, 128, 128, 2, 2, 2>;   // 4 waves of 64 x 64, 64 KiB LDS, two workgroups per CU

// Which tiles: by rounds of workgroups, an expert's last row tile counted as half full.  A 256 x 256 tile is one workgroup's, alone on its
// compute unit; of the 128 x 128 ones a unit has two, which take 1.5 times as long for their share of the work.  A last, partly filled
// round costs between half a round and a whole one: its workgroups have the caches to themselves.  us, large / small tiles:
//   16384 rows, d = 1024, F = 4096, E = 8      GATE 342 / 371, DH 238 / 271, DX 236 / 305, DW 390 / 491, DOWN 120 / 149
//   8192 rows, d = 384, F = 1536, E = 8        DH 40.6 / 39.2, DX 71 / 37, DW 63 / 42
//   5003 rows, d = 1000, F = 2728, E = 32      GATE 127 / 141, DOWN 92 / 85
//   2000 rows, d = 768, F = 2048, E = 64       GATE 144 / 129, DH 70 / 55, DX 113 / 97, DW 142 / 174, DOWN 70 / 63
static bool large_tiles(const GatedArgs& a, int mode, int64_t max_rows) {
  const int64_t cus = num_cus();
  double tiles[2] = {0, 0};
  for (int q = 0; q < 2; ++q) {
    const int B = q == 0 ? 256 : 128, BN = mode == G_GATE ? B / 2 : B;
    for (const GatedJob& j : a.j) {
      if (j.C == nullptr) continue;
      const double across = (j.N + BN - 1) / BN;
      if (mode == G_DW) tiles[q] += across * ((j.M + B - 1) / B) * a.E;
      else tiles[q] += across * (static_cast<double>(max_rows) / B + 0.5 * static_cast<double>(a.E < max_rows ? a.E : max_rows));
    }
  }
  auto rounds = [](double t) {
    const double whole = floor(t), rest = t - whole;
    return whole < 1.0 ? 1.0 : rest > 0.0 ? whole + 0.5 + 0.5 * rest : whole;
  };
  return 4.0 * rounds(tiles[0] / static_cast<double>(cus)) <= 2.0 * 1.5 * rounds(tiles[1] / (2.0 * static_cast<double>(cus)));
}

int launch_gated_bf16(const GatedArgs& a, int mode, int keep, int64_t max_rows, hipStream_t stream) {
  return large_tiles(a, mode, max_rows) ? launch_gated_mode<GatedA>(a, mode, keep, max_rows, stream) : launch_gated_mode<GatedU>(a, mode, keep, max_rows, stream);
}

}  // namespace scmoe
