// Matrix products: g^T x, and the sums of g.
#include "matmul_tiles.h"

namespace fpq {

int launch_matmul_cols_sums(const MatmulArgs& p, int tile, hipStream_t s) { return launch_matmul_form<true, true, kSums>(p, tile, s); }

}  // namespace fpq
