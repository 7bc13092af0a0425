// Matrix products: x W^T of a gated projection.
#include "matmul_tiles.h"

namespace fpq {

int launch_matmul_gated(const MatmulArgs& p, int tile, hipStream_t s) { return launch_matmul_form<false, false, kGated>(p, tile, s); }

}  // namespace fpq
