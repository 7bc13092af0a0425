// Matrix products: x W^T.
#include "matmul_tiles.h"

namespace fpq {

int launch_matmul_rows(const MatmulArgs& p, int tile, hipStream_t s) { return launch_matmul_form<false, false, kStore>(p, tile, s); }

}  // namespace fpq
