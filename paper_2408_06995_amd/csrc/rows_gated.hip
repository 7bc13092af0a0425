// Gated projections of few rows.
#include "rows.h"
#include <stdlib.h>

namespace fpq {

namespace {

template <typename T>
int launch(const RowsArgs& a, hipStream_t s)
{
    // (blocks that are kept are 32 outputs of one workgroup: the same sums in the same order)
    const bool blocks = a.gate.pre_scales;
    static const int v = getenv("FPQ_V") ? atoi(getenv("FPQ_V")) : 0;
    if (a.M <= 16) {
        if (v == 1 && !blocks) return launch_rows_as<T, T, 1, 1, 8, true>(a, s);
        if (v == 2 && !blocks) return launch_rows_as<T, T, 1, 1, 16, true>(a, s);
    }
    if (a.M <= 16) return blocks ? launch_rows_as<T, T, 1, 2, 4, true>(a, s) : launch_rows_as<T, T, 1, 1, 4, true>(a, s);
    if (a.M <= 32) return blocks ? launch_rows_as<T, T, 2, 2, 4, true>(a, s) : launch_rows_as<T, T, 2, 1, 4, true>(a, s);
    return blocks ? launch_rows_as<T, T, 4, 2, 4, true>(a, s) : launch_rows_as<T, T, 4, 1, 4, true>(a, s);
}

}  // namespace

int launch_rows_gated(const RowsArgs& a, hipStream_t s) { return a.f32 ? launch<float>(a, s) : launch<__bf16>(a, s); }

}  // namespace fpq
