// The adapters' kernels for activations in fp32 and weights in fp32.
#include "adapter_kernels.h"

namespace fpq {

int launch_apply_f32(const AdapterArgs& a, bool vec_k, const AdapterPlan& plan, hipStream_t s) { return launch_apply<float, float>(a, vec_k, plan, s); }
int launch_backward_f32(const AdapterArgs& a, bool vec_n, bool vec_k, const AdapterPlan& plan, hipStream_t s)
{
    return launch_backward<float, float>(a, vec_n, vec_k, plan, s);
}

}  // namespace fpq
