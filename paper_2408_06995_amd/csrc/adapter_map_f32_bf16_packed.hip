// Rows through a rank: activations in fp32, weights in bf16, packed.
#include "adapter_kernels.h"

namespace fpq {

int launch_map_f32_bf16_packed(const AdapterArgs& a, int waves, hipStream_t s) { return launch_map<float, 2>(a, waves, s); }

}  // namespace fpq
