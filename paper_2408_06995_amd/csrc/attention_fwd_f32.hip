// Forward attention in fp32.
#include "attention_forward.h"

namespace fpq {

int launch_attention_f32(const AttentionArgs& a, bool by_keys, int waves, hipStream_t s) { return launch_forward<float>(a, by_keys, waves, s); }

}  // namespace fpq
