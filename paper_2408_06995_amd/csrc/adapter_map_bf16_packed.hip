// Rows through a rank: activations and weights in bf16, packed.
#include "adapter_kernels.h"

namespace fpq {

int launch_map_bf16_packed(const AdapterArgs& a, int waves, hipStream_t s) { return launch_map<__bf16, 2>(a, waves, s); }

}  // namespace fpq
