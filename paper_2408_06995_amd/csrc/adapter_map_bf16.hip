// Rows through a rank: activations and weights in bf16.
#include "adapter_kernels.h"

namespace fpq {

int launch_map_bf16(const AdapterArgs& a, int waves, hipStream_t s) { return launch_map<__bf16, 1>(a, waves, s); }

}  // namespace fpq
