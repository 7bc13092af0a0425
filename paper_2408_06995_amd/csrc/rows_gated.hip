// Gated projections of few rows.
#include "rows.h"

namespace fpq {

namespace {

template <typename T>
int launch(const RowsArgs& a, hipStream_t s)
{
    // (blocks that are kept are 32 outputs of one workgroup: the same sums in the same order)
    const bool blocks = a.gate.pre_scales;
    // (eight wavefronts are within 5 % either way: one row of 4096 -> 1280 10.2 us for 12.1, -> 5120 21.2 for 18.7)
    if (a.M <= 16) return blocks ? launch_rows_as<T, T, 1, 2, 4, true>(a, s) : launch_rows_as<T, T, 1, 1, 4, true>(a, s);
    if (a.M <= 32) return blocks ? launch_rows_as<T, T, 2, 2, 4, true>(a, s) : launch_rows_as<T, T, 2, 1, 4, true>(a, s);
    return blocks ? launch_rows_as<T, T, 4, 2, 4, true>(a, s) : launch_rows_as<T, T, 4, 1, 4, true>(a, s);
}

}  // namespace

int launch_rows_gated(const RowsArgs& a, hipStream_t s) { return a.f32 ? launch<float>(a, s) : launch<__bf16>(a, s); }

}  // namespace fpq
