// The adapters' kernels for activations in fp32 and weights in bf16.
#include "adapter_kernels.h"

namespace fpq {

int launch_apply_mixed(const AdapterArgs& a, bool vec_k, const AdapterPlan& plan, hipStream_t s) { return launch_apply<float, __bf16>(a, vec_k, plan, s); }
int launch_backward_mixed(const AdapterArgs& a, bool vec_n, bool vec_k, const AdapterPlan& plan, hipStream_t s)
{
    return launch_backward<float, __bf16>(a, vec_n, vec_k, plan, s);
}

}  // namespace fpq
