// Backward attention in bf16, and the call of both types.
#include "attention_backward.h"

namespace fpq {

int launch_attention_backward_f32(const AttentionArgs& aq, const AttentionArgs& ak, const AttentionPlan& p, hipStream_t s);

int launch_attention_backward(const AttentionArgs& a, int type, const AttentionPlan& p, float* part_q, float* part_kv, hipStream_t s)
{
    AttentionArgs aq = a, ak = a;
    aq.blocks = p.q_blocks;
    aq.q_pad = p.q_pad;
    aq.splits = p.q_splits;
    aq.part = part_q;
    ak.blocks = p.k_blocks;
    ak.splits = p.k_splits;
    ak.part = part_kv;
    return type == FPQ_TYPE_FP32 ? launch_attention_backward_f32(aq, ak, p, s) : launch_backward<__bf16>(aq, ak, p, s);
}

}  // namespace fpq
