// Matrix products: g^T x.
#include "matmul_tiles.h"

namespace fpq {

int launch_matmul_cols(const MatmulArgs& p, int tile, hipStream_t s) { return launch_matmul_form<true, true, kStore>(p, tile, s); }

}  // namespace fpq
