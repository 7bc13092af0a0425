// The gradients of the adapters.
#include "adapter_kernels.h"

namespace fpq {

int launch_adapter_outer(const OuterArgs& a, int x_type, hipStream_t s)
{
    const bool vec = a.vec_rows[0] && a.vec_rows[1] && a.vec_t;
    if (x_type == FPQ_TYPE_FP32) return vec ? launch_outer<float, true>(a, s) : launch_outer<float, false>(a, s);
    return vec ? launch_outer<__bf16, true>(a, s) : launch_outer<__bf16, false>(a, s);
}

}  // namespace fpq
