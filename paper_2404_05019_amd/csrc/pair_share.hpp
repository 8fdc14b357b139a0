// How the workgroups of a launch that has two products are shared out between them.  No device header is needed, so that the choice can
// be looked at on the host.
#pragma once

#include <math.h>

namespace scmoe {

struct PairShare { int first; double cost; };    // workgroups an XCD (of eight) for the first product; what the slower one takes

// Tiles of either product, what one of them takes, workgroups an XCD (at least 2), compute units.  Both products are to end at the same time: the first
// has one to a few long tiles a workgroup, the second many short ones.  Of shares that are as good by that, the first product gets the most workgroups
// that are of use to it while each of the launch still has a compute unit to itself: what a few long tiles of the second leave, where many small ones of
// the first would follow one another on a few units.  dx and the weights' gradients of the gated block, us: 7001 rows, d = 80, F = 208, E = 4 (220 and 24 tiles) 45, so 28;
// 6225, 136, 152, 1 74 / 55; with more workgroups than units 8183, 320, 680, 2 58 / 66.
inline PairShare share_pair(double tiles1, double cost1, double tiles2, double cost2, int resident, int cus) {
  PairShare best{1, 1e300};
  double both = 1e300;
  for (int s = 1; s < resident; ++s) {
    const double left = 8.0 * (resident - s), r1 = ceil(tiles1 / (8.0 * s)) * cost1, r2 = ceil(tiles2 / left) * cost2, t = r1 > r2 ? r1 : r2;
    const bool apart = 8.0 * s + (tiles2 < left ? tiles2 : left) <= cus;
    if (t < best.cost || (t == best.cost && r1 + r2 < both && apart)) {
      best = {s, t};
      both = r1 + r2;
    }
  }
  return best;
}

}  // namespace scmoe
