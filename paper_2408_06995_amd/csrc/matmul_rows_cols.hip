// Matrix products: g W.
#include "matmul_tiles.h"

namespace fpq {

int launch_matmul_rows_cols(const MatmulArgs& p, int tile, hipStream_t s) { return launch_matmul_form<false, true, kStore>(p, tile, s); }

}  // namespace fpq
