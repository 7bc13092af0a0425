// Rows through a rank: activations in fp32, weights in fp32.
#include "adapter_kernels.h"

namespace fpq {

int launch_map_f32(const AdapterArgs& a, int waves, hipStream_t s) { return launch_map<float, 0>(a, waves, s); }

}  // namespace fpq
