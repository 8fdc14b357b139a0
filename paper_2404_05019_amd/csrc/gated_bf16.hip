// The gated feed-forward block's products in bf16 (gated_tiles.hpp).
#include "gated_tiles.hpp"

namespace scmoe {

using GatedU = GatedCfg<false, 128, 128, 2, 2, 2>;   // 4 waves of 64 x 64, 64 KiB LDS, two workgroups per CU

int launch_gated_bf16(const GatedArgs& a, int mode, int keep, int64_t max_rows, hipStream_t stream) {
  return launch_gated_mode<GatedU>(a, mode, keep, max_rows, stream);
}

}  // namespace scmoe
