// Forward attention in bf16, and the plan of a call.
#include "attention_forward.h"

namespace fpq {

int launch_attention_f32(const AttentionArgs& a, bool by_keys, hipStream_t s);

// Parts of an axis of `len` in units: until there are about two workgroups per compute unit, with no fewer than `least` each.
static void cut(int64_t len, int64_t have, int unit, int64_t least, int* n, int* per)
{
    int64_t s = have > 0 ? (512 + have - 1) / have : 1;
    if (s > len / least) s = len / least;
    s = s < 1 ? 1 : s > 64 ? 64 : s;
    if (len < 1) len = 1;
    *per = (int)(((len + s - 1) / s + unit - 1) / unit * unit);
    *n = (int)((len + *per - 1) / *per);
}

AttentionPlan plan_attention(int64_t batch, int64_t kv_heads, int64_t group, int64_t q_len, int64_t kv_len, int64_t dim, int type)
{
    AttentionPlan p;
    const int64_t bh = batch * kv_heads, rows = group * q_len, wide = (rows + 127) / 128, few = type == FPQ_TYPE_FP32 ? 64 : 32;
    const int ks = (int)(dim + 15) / 16;
    // the rows form wherever its workgroups, the keys cut into parts of at least 256, fill the compute units
    p.by_keys = rows <= few || bh * wide * (kv_len / 256 > 1 ? kv_len / 256 : 1) < 256;
    p.blocks = (int)(p.by_keys ? (rows + few - 1) / few : wide);
    cut(kv_len, bh * p.blocks, 128, 256, &p.splits, &p.per_split);
    p.q_blocks = (int)wide;
    cut(kv_len, bh * wide, 128, 256, &p.q_splits, &p.q_per_split);
    p.k_blocks = (int)((kv_len + 127) / 128);
    const int tile = type == FPQ_TYPE_FP32 ? kKeysTile<3, 3> : ks <= 4 ? kKeysTile<1, 4> : ks <= 6 ? kKeysTile<1, 6> : kKeysTile<1, 8>;
    const int64_t tiles = group * ((q_len + tile - 1) / tile);
    cut(tiles, bh * p.k_blocks, 1, 128 / tile, &p.k_splits, &p.k_per_split);
    return p;
}

int launch_attention(const AttentionArgs& a, int type, const AttentionPlan& p, hipStream_t s)
{
    return type == FPQ_TYPE_FP32 ? launch_attention_f32(a, p.by_keys, s) : launch_forward<__bf16>(a, p.by_keys, s);
}

}  // namespace fpq
