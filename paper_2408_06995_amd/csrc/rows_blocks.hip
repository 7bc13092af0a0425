// Layers on 4-bit blocks for few rows.
#include "rows.h"

namespace fpq {

namespace {

template <typename T>
int launch(const RowsArgs& a, hipStream_t s)
{
    if (a.M <= 16) {
        // Sixteen columns and eight wavefronts where there are few columns; 32 columns read x half as often (16 rows of 5120 -> 5120: 11.4 us
        // for 15.6 in bf16, 17.3 for 24.9 in fp32), four wavefronts where there are many (-> 20480 in fp32: 45.7 for 48.6).
        if (a.N < 4096) return launch_rows_as<T, Blocks4, 1, 1, 8, false>(a, s);
        return a.N < 16384 ? launch_rows_as<T, Blocks4, 1, 2, 8, false>(a, s) : launch_rows_as<T, Blocks4, 1, 2, 4, false>(a, s);
    }
    if (a.M <= 32) return launch_rows_as<T, Blocks4, 2, 2, 8, false>(a, s);
    return launch_rows_as<T, Blocks4, 4, 2, 8, false>(a, s);
}

}  // namespace

int launch_rows_blocks(const RowsArgs& a, hipStream_t s) { return a.f32 ? launch<float>(a, s) : launch<__bf16>(a, s); }

}  // namespace fpq
