// Matrix products: d w and d^T x in one launch.
#include "matmul_tiles.h"

namespace fpq {

int launch_matmul_both(const MatmulArgs& x, const MatmulArgs& w, int tile, hipStream_t s) { return launch_matmul_both_form<kStore>(x, w, tile, s); }

}  // namespace fpq
