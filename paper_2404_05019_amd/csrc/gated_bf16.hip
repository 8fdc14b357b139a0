// The gated feed-forward block's products in bf16 (gated_tiles.hpp).
#include "gated_tiles.hpp"
#include <math.h>

namespace scmoe {

using GatedA = GatedCfg<false, 256, 256, 2, 4, 2>;   // 8 waves of 128 x 64, 128 KiB LDS, one workgroup per CU
using GatedV = GatedCfg<false, 256, 128, 4, 2, 3, 2048>;   // 8 waves of 64 x 64, 160 KiB LDS, one workgroup per CU: DOWN, DX
using GatedU = GatedCfg<false, 128, 128, 2, 2, 2>;   // 4 waves of 64 x 64, 64 KiB LDS, two workgroups per CU

using GatedS = GatedCfg<false, 64, 64, 4, 1, 3>;     // 4 waves of 16 x 64, 64 KiB LDS, two workgroups per CU

// Which tiles: by rounds of workgroups.  A 256 x 256 tile is one workgroup's, alone on its compute unit (its time: 4); of the 128 x 128
// ones a unit has two, which take 1.5 times as long for their share of the work (3; one alone on its unit: 2), and a 256 x 128 one, which
// DOWN and DX have too, takes 2.6.  A last, partly filled round costs between half a round and a whole one: its workgroups have the caches to
// themselves.  us, 256 x 256 / 128 x 128 / 64 x 64 tiles (GATE, DOWN: of a forward call; DH, DX, DW: of a gradient):
//   16384 rows, d = 1024, F = 4096, E = 8      GATE 368 / 397 / 597, DH 794 / 809 / 910, DX 787 / 865 / 1084, DW 799 / 890 / 1187
//   8192 rows, d = 384, F = 1536, E = 8        GATE 56 / 51 / 67, DH 119 / 119 / 127, DX 150 / 119 / 129, DW 138 / 120 / 137
//   5003 rows, d = 1000, F = 2728, E = 32      GATE 273 / 283 / 341, DH 476 / 469 / 508, DX 476 / 476 / 531, DW 476 / 504 / 725
//   2000 rows, d = 768, F = 2048, E = 64       GATE 157 / 145 / 152, DH 334 / 334 / 335, DX 336 / 334 / 329, DW 333 / 366 / 524
//   64 rows, d = 2048, F = 8192, E = 16        GATE 345 / 311 / 319, DH 660 / 665 / 677, DX 797 / 668 / 699, DW 667 / 744 / 1136
// 256 x 128 tiles against those that would be taken else:
//   5003 rows, d = 1000, F = 2728, E = 32      DOWN 186 / 199, DX 446 / 465;   6000, d = 1024, F = 4096, E = 8  DX 374 / 391
//   but 3001, d = 768, F = 2048, E = 12        DX 155 / 139;   8192, d = 384, F = 1536, E = 8  DX 124 / 117
// 64 x 64 tiles where the 128 x 128 ones would leave half of the compute units without work, or are fewer than 1.5 of them with a short K; their rows of an
// operand across k are 128 bytes long, which streams weights worse, and a gradient of weights (all tiles are written, whatever the rows)
// always has tiles enough:
//   1 row, d = 2048, F = 8192, E = 16          GATE 60 / 38 / 33, DH 447 / 426 / 421, DX 581 / 427 / 388
//   30 rows, d = 1000, F = 2728, E = 8         GATE 47 / 41 / 38
//   500 rows, d = 1000, F = 2728, E = 8        GATE 74 / 70 / 71, DH 148 / 134 / 133, DX 198 / 133 / 122
//   2000 rows, d = 512, F = 1024, E = 8        GATE 35 / 29 / 28, DH 72 / 57 / 49, DX 80 / 57 / 49, DW 57 / 57 / 65
enum { TILES_256, TILES_256_128, TILES_128, TILES_64 };
static int tiles_for(const GatedArgs& a, int mode, int64_t max_rows) {
  const double cus = num_cus(), segs = static_cast<double>(a.E < max_rows ? a.E : max_rows);
  // an expert's row tiles of that many rows: its last one half full, unless the average leaves room in one
  auto row_tiles = [&](double rows) {
    const double mean = static_cast<double>(max_rows) / segs;
    return segs * (mean <= 0.75 * rows ? 1.0 : mean / rows + 0.5);
  };
  auto tiles = [&](int rows, int cols) {
    double n = 0;
    for (const GatedJob& j : a.j) {
      if (j.C == nullptr) continue;
      const double across = (j.N + cols - 1) / cols;
      n += across * (mode == G_DW ? static_cast<double>((j.M + rows - 1) / rows) * a.E : row_tiles(rows));
    }
    return n;
  };
  auto rounds = [](double t) {
    const double whole = floor(t), rest = t - whole;
    return whole < 1.0 ? 1.0 : rest > 0.0 ? whole + 0.5 + 0.5 * rest : whole;
  };
  const bool gate = mode == G_GATE;                            // (half as many columns: a tile has those of g and of u)
  const double small = tiles(128, gate ? 64 : 128);
  if (mode != G_DW && small < (a.j[0].Kd < 2048 ? 1.5 : 0.5) * cus) return TILES_64;
  const double t256 = 4.0 * rounds(tiles(256, gate ? 128 : 256) / cus), t128 = small <= cus ? 2.0 : 3.0 * rounds(small / (2.0 * cus));
  if ((mode == G_DOWN || mode == G_DX) && 2.6 * rounds(tiles(256, 128) / cus) < (t256 < t128 ? t256 : t128)) return TILES_256_128;
  return t256 <= t128 ? TILES_256 : TILES_128;
}

int launch_gated_bf16(const GatedArgs& a, int mode, int keep, int64_t max_rows, hipStream_t stream) {
  switch (tiles_for(a, mode, max_rows)) {
    case TILES_256_128: return mode == G_DOWN ? launch_gated_cfg<GatedV, G_DOWN, KEEP_NONE, 0>(a, max_rows, stream) : launch_gated_cfg<GatedV, G_DX, KEEP_NONE, 0>(a, max_rows, stream);
    case TILES_256: return launch_gated_mode<GatedA>(a, mode, keep, max_rows, stream);
    case TILES_128: return launch_gated_mode<GatedU>(a, mode, keep, max_rows, stream);
    default: return launch_gated_rows<GatedS>(a, mode, keep, max_rows, stream);
  }
}

}  // namespace scmoe
