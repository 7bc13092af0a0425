// Forward attention in bf16, and the call of both types.
#include "attention_forward.h"

namespace fpq {

int launch_attention_f32(const AttentionArgs& a, bool by_keys, int waves, hipStream_t s);

int launch_attention(const AttentionArgs& a, int type, const AttentionPlan& p, hipStream_t s)
{
    return type == FPQ_TYPE_FP32 ? launch_attention_f32(a, p.by_keys, p.waves, s) : launch_forward<__bf16>(a, p.by_keys, p.waves, s);
}

}  // namespace fpq
