// Matrix products: d w, d^T x and the sums of d in one launch.
#include "matmul_tiles.h"

namespace fpq {

int launch_matmul_both_sums(const MatmulArgs& x, const MatmulArgs& w, int tile, hipStream_t s) { return launch_matmul_both_form<kSums>(x, w, tile, s); }

}  // namespace fpq
