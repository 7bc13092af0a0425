// Rows through a rank: activations in fp32, weights in bf16.
#include "adapter_kernels.h"

namespace fpq {

int launch_map_f32_bf16(const AdapterArgs& a, int waves, hipStream_t s) { return launch_map<float, 1>(a, waves, s); }

}  // namespace fpq
