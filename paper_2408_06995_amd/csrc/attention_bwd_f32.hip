// Backward attention in fp32.
#include "attention_backward.h"

namespace fpq {

int launch_attention_backward_f32(const AttentionArgs& aq, const AttentionArgs& ak, const AttentionPlan& p, hipStream_t s) { return launch_backward<float>(aq, ak, p, s); }

}  // namespace fpq
