// The adapters' kernels for activations in bf16 and weights in bf16.
#include "adapter_kernels.h"

namespace fpq {

int launch_apply_bf16(const AdapterArgs& a, bool vec_k, const AdapterPlan& plan, hipStream_t s) { return launch_apply<__bf16, __bf16>(a, vec_k, plan, s); }
int launch_backward_bf16(const AdapterArgs& a, bool vec_n, bool vec_k, const AdapterPlan& plan, hipStream_t s)
{
    return launch_backward<__bf16, __bf16>(a, vec_n, vec_k, plan, s);
}

}  // namespace fpq
