// The gated feed-forward block's products in bf16 (gated_tiles.hpp).
#include "gated_tiles.hpp"
#include <algorithm>
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
// 64 x 64 tiles where the 128 x 128 ones would leave half of the compute units without work, or, with a short K, are fewer than 1.5 of them (GATE 0.6, DH 0.7,
// where the segments are not short as well); their rows of an operand across k are 128 bytes long, which streams weights worse, and a gradient of weights (all tiles are written, whatever the rows)
// always has tiles enough:
//   1 row, d = 2048, F = 8192, E = 16          GATE 60 / 38 / 33, DH 447 / 426 / 421, DX 581 / 427 / 388
//   30 rows, d = 1000, F = 2728, E = 8         GATE 47 / 41 / 38
//   500 rows, d = 1000, F = 2728, E = 8        GATE 74 / 70 / 71, DH 148 / 134 / 133, DX 198 / 133 / 122
//   2000 rows, d = 512, F = 1024, E = 8        GATE 35 / 29 / 28, DH 72 / 57 / 49, DX 80 / 57 / 49, DW 57 / 57 / 65
// 128 x 128 / 64 x 64 with a short K, and their number of the larger tiles:
//   GATE  3000 rows, d = 512, F = 512, E = 12 (235) 21.8 / 25.6; 1500, 768, 1024, 8 (251) 25.5 / 29.2; 1000, 512, 2048, 2 (282) 24.8 / 27.2; 300, 512, 4096, 1
//         (182) 23.8 / 25.0; but 500, 512, 1024, 8 (128) 19.4 / 18.8; short segments: 200, 1024, 4096, 4 (256) 35.8 / 34.6; 30, 1000, 2728, 8 (344) 41 / 38
//   DH    1000, 1024, 2048, 8 (189) 98 / 104; 4096, 128, 1024, 4 (272) 34.7 / 36.6; but 2000, 512, 1024, 8 (157) 36.2 / 33.8; 1200, 1024, 2048, 20 (320) 166 / 160
enum { TILES_256, TILES_256_128, TILES_128, TILES_64 };
struct TileTimes { double small, t256, t128, t256_128; };      // how many 128 x 128 tiles; times, 4 of which are a 256 x 256 tile's
static TileTimes tile_times(const GatedArgs& a, int mode, int64_t max_rows) {
  const double cus = num_cus();
  auto tiles = [&](int rows, int cols) { return likely_tiles(a, mode, max_rows, rows, cols); };
  auto rounds = [](double t) {
    const double whole = floor(t), rest = t - whole;
    return whole < 1.0 ? 1.0 : rest > 0.0 ? whole + 0.5 + 0.5 * rest : whole;
  };
  const bool gate = mode == G_GATE;                            // (half as many columns: a tile has those of g and of u)
  TileTimes t;
  t.small = tiles(128, gate ? 64 : 128);
  t.t256 = 4.0 * rounds(tiles(256, gate ? 128 : 256) / cus);
  t.t128 = t.small <= cus ? 2.0 : 3.0 * rounds(t.small / (2.0 * cus));
  t.t256_128 = mode == G_DOWN || mode == G_DX ? 2.6 * rounds(tiles(256, 128) / cus) : 1e300;
  return t;
}
static bool short_segments(const GatedArgs& a, int64_t max_rows) { return max_rows <= 56 * (a.E < max_rows ? a.E : max_rows); }
static int tiles_for(const GatedArgs& a, int mode, int64_t max_rows) {
  const TileTimes t = tile_times(a, mode, max_rows);
  const double limit = a.j[0].Kd >= 2048 ? 0.5 : short_segments(a, max_rows) || mode == G_DOWN || mode == G_DX ? 1.5 : mode == G_GATE ? 0.6 : 0.7;
  if (mode != G_DW && t.small < limit * num_cus()) return TILES_64;
  if (t.t256_128 < (t.t256 < t.t128 ? t.t256 : t.t128)) return TILES_256_128;
  return t.t256 <= t.t128 ? TILES_256 : TILES_128;
}

int launch_gated_bf16(const GatedArgs& a, int mode, int keep, int64_t max_rows, hipStream_t stream) {
  switch (tiles_for(a, mode, max_rows)) {
    case TILES_256_128: return mode == G_DOWN ? launch_gated_cfg<GatedV, G_DOWN, KEEP_NONE, 0>(a, max_rows, stream) : launch_gated_cfg<GatedV, G_DX, KEEP_NONE, 0>(a, max_rows, stream);
    case TILES_256: return launch_gated_mode<GatedA>(a, mode, keep, max_rows, stream);
    case TILES_128: return launch_gated_mode<GatedU>(a, mode, keep, max_rows, stream);
    default: return launch_gated_rows<GatedS>(a, mode, keep, max_rows, stream);
  }
}

// DX and DW in one launch (which of the two forms, and when), us of a gradient, two launches / one:
//  * On 128 x 128 tiles (DX on 64 x 64 ones where it has under a quarter as many tiles as compute units), where both together are at most 3.5 rounds:
//    8192 rows, d = 384, F = 1536, E = 8 112 / 101; 4096, 768, 2048, 4 142 / 122; 2048, 1024, 4096, 1 164 / 147; 16384, 256, 1024, 4 126 / 108;
//    1000, 512, 2048, 2 44 / 34; 300, 512, 4096, 1 51 / 44 (DX on 128 x 128 tiles: 67); 64, 768, 2048, 1 33 / 28; also where DX fills 3/8 to 5/8 of the units
//    and DW is up to twelve rounds: 1000, 768, 2048, 16 120 / 108; 1500, 1024, 2048, 16 150 / 141; 2205, 576, 2232, 16 142 / 128; 744, 1336, 2408, 9 169 / 153; but
//    64 tiles of DX (300, 1024, 4096, 8) 134 / 145.  With short segments, whose tiles of DW have one k-tile, up to seven rounds: 1068, 376, 760, 42 (4.4) 56 / 53; 1479,
//    344, 784, 43 (5) 69 / 60; but 396, 720, 1384, 20 (7.7) 77 / 83; 54, 624, 1736, 22 (9) 88 / 98; 843, 480, 1816, 30 (10) 99 / 108.
//  * On 256 x 256 tiles, where DX has a quarter to one of them a compute unit and DW twice as many, up to 24 a unit: 2000, 768, 2048, 64 314 / 270; 8192, 768,
//    1536, 8 158 / 137; 1000, 1024, 2048, 32 217 / 190; 4096, 1536, 4096, 2 361 / 313; 8192, 768, 2048, 16 238 / 229; 6000, 512, 2048, 24 169 / 168; 8192, 1024, 2048,
//    8 237 / 237.  Beyond that two launches fill the chip for as long, and share the caches better: 16384, 1024, 4096, 8
//    752 / 792; 32768, 2048, 8192, 16 5227 / 5834; 2000, 2048, 8192, 16 896 / 962; 16384, 512, 1024, 8 152 / 162.
//    Nor where the slower half of the launch, whose tiles rarely come out even, is expected to take 1.1 times as long as two launches on the tiles
//    that suit each: 5003, 1000, 2728, 32 445 / 458; 8632, 544, 1592, 24 228 / 258; 18353, 576, 2248, 21 432 / 503; 3925, 1440, 5400, 13 666 / 753; 8660, 304, 848,
//    57 126 / 139.  Of 107 sizes, most of them drawn, that leaves out 29, of which 18 are slower in one launch, by up to 16 %, and the others faster, by up
//    to 7 % (6000, 1024, 2048, 32 303 / 285).  Segments of up to 128 rows stay in one launch: half of DX's waves leave out their products there (2959, 848,
//    952, 32 134 / 119; 2008, 1216, 4320, 21 398 / 342).
static bool pair_gains(const GatedArgs& x, const GatedArgs& w, int64_t max_rows) {
  if (max_rows <= 128 * static_cast<int64_t>(w.E)) return true;
  const TileTimes tx = tile_times(x, G_DX, max_rows), tw = tile_times(w, G_DW, max_rows);
  const double dx = std::min({tx.t256, tx.t128, tx.t256_128}), dw = std::min(tw.t256, tw.t128);
  return share_gated_pair<GatedA, GatedA>(x, w, max_rows).cost <= 1.1 * 0.25 * (dx * tile_cost<GatedA, G_DX>(x, max_rows) + dw * tile_cost<GatedA, G_DW>(w, max_rows));
}
int launch_gated_gradients_bf16(const GatedArgs& x, const GatedArgs& w, int64_t max_rows, hipStream_t stream) {
  const double cus = num_cus();
  const double xu = likely_tiles(x, G_DX, max_rows, 128, 128), wu = likely_tiles(w, G_DW, max_rows, 128, 128);
  const double xa = likely_tiles(x, G_DX, max_rows, 256, 256), wa = likely_tiles(w, G_DW, max_rows, 256, 256);
  if (xu <= 1.5 * cus && xu + wu <= 3.5 * 2.0 * cus)
    return xu < 0.25 * cus ? launch_gated_pair<GatedS, GatedU>(x, w, max_rows, stream) : launch_gated_pair<GatedU, GatedU>(x, w, max_rows, stream);
  if (xu > 0.625 * cus && xa >= 0.25 * cus && xa <= cus && wa >= 2.0 * xa && wa <= 24.0 * cus && pair_gains(x, w, max_rows))
    return launch_gated_pair<GatedA, GatedA>(x, w, max_rows, stream);
  if (xu >= 0.375 * cus && xu <= 0.625 * cus && wu <= (short_segments(x, max_rows) ? 7.0 : 12.0) * 2.0 * cus) return launch_gated_pair<GatedU, GatedU>(x, w, max_rows, stream);
  const int st = launch_gated_bf16(w, G_DW, KEEP_NONE, max_rows, stream);
  return st == SCMOE_OK ? launch_gated_bf16(x, G_DX, KEEP_NONE, max_rows, stream) : st;
}

}  // namespace scmoe
