// Forward attention in bf16, and the plan of a call.
#include "attention_forward.h"

namespace fpq {

int launch_attention_f32(const AttentionArgs& a, bool vec, bool by_keys, hipStream_t s);

// Keys form: 32 rows of a workgroup instead of 128, for grids that leave compute units idle.  Parts: until about two workgroups per
// compute unit, with no fewer than 256 keys (or two tiles of queries) each.
static int parts(int64_t have, int64_t units, int64_t least, int64_t want)
{
    int64_t s = (want + have - 1) / have;
    if (s > units / least) s = units / least;
    return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}

AttentionPlan plan_attention(int64_t batch, int64_t kv_heads, int64_t group, int64_t q_len, int64_t kv_len)
{
    AttentionPlan p;
    const int64_t bh = batch * kv_heads, rows = group * q_len;
    const int64_t wide = (rows + 127) / 128;
    p.by_keys = bh * wide < 256 || rows <= 32;
    p.blocks = (int)(p.by_keys ? (rows + 31) / 32 : wide);
    auto cut = [](int64_t len, int n, int unit) { return (int)(((len + n - 1) / n + unit - 1) / unit * unit); };
    auto fit = [&](int64_t len, int64_t have, int unit, int least, int* n, int* per) {
        *n = parts(have > 0 ? have : 1, len, least, 512);
        *per = cut(len > 0 ? len : 1, *n, unit);
        *n = (int)((len + *per - 1) / *per);
        if (*n < 1) *n = 1;
    };
    fit(kv_len, bh * p.blocks, 128, 256, &p.splits, &p.per_split);
    p.q_blocks = (int)wide;
    fit(kv_len, bh * p.q_blocks, 64, 256, &p.q_splits, &p.q_per_split);
    p.k_blocks = (int)((kv_len + 127) / 128);
    const int64_t tiles = group * ((q_len + KeysTile - 1) / KeysTile);
    fit(tiles, bh * p.k_blocks, 1, 4, &p.k_splits, &p.k_per_split);
    return p;
}

int launch_attention(const AttentionArgs& a, int type, bool vec, const AttentionPlan& p, hipStream_t s)
{
    if (type == FPQ_TYPE_FP32) return launch_attention_f32(a, vec, p.by_keys, s);
    return launch_forward<__bf16>(a, vec, p.by_keys, s);
}

}  // namespace fpq
