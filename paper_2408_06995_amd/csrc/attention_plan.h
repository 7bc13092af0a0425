// How an attention call is divided, by its sizes and type only: the same for the launches and for the size of the workspace.  Host code,
// but for the constants.
#pragma once
#include <stdint.h>

#include "../../include/fpq.h"

namespace fpq {

// Strides in elements: sample, token, head.
struct Strides {
    int64_t b, t, h;
};

// Of a packed tensor: [batch][heads][len][cols], cols = dim rounded up to 8.
inline Strides packed_strides(int64_t heads, int64_t len, int64_t dim)
{
    const int64_t cols = (dim + 7) / 8 * 8;
    return {heads * len * cols, cols, len * cols};
}

// Queries of a tile of the backward pass's keys kernel.
template <int NP, int KS>
constexpr int kKeysTile = NP == 3 ? 32 : KS <= 4 ? 128 : KS <= 6 ? 64 : 32;

// How a call's kernels are chosen and cut (host): by sizes and type only, the same for the size of the workspace.
struct AttentionPlan {
    int q_pad;                  // AttentionArgs
    bool by_keys;               // forward: the wavefronts of a workgroup share 32 rows and divide the keys
    int waves, blocks, splits;                        // waves: of a workgroup, with 32 rows (or keys) each
    int q_waves, q_blocks, q_splits;                  // backward, gradient of the queries
    int k_waves, k_blocks, k_splits;                  // backward, gradient of the keys and values
};

// Parts of an axis of `len`: until there are about `want` workgroups, with no fewer than `least` each.
inline int parts_of(int64_t len, int64_t have, int64_t want, int64_t least)
{
    int64_t s = have > 0 ? (want + have - 1) / have : 1;
    if (s > len / least) s = len / least;
    return s < 1 ? 1 : s > 32 ? 32 : (int)s;
}

inline AttentionPlan plan_attention(int64_t batch, int64_t kv_heads, int64_t group, int64_t q_len, int64_t kv_len, int64_t dim, int type, bool causal)
{
    AttentionPlan p;
    const bool fp32 = type == FPQ_TYPE_FP32;
    const int64_t bh = batch * kv_heads, rows = group * q_len, few = fp32 ? 64 : 32;
    const int ks = (int)(dim + 15) / 16;
    // Two workgroups of four wavefronts per compute unit in bf16, where one's arithmetic covers the other's matrix steps; fp32 has six
    // matrix steps for each.  Fewer rows than that: two wavefronts, and parts of the keys (of the queries, for the gradient of the
    // keys), of no less than takes longer than the pass that joins them.  Measured over 256 or 512 workgroups and parts of no less
    // than 64 to 512: backward of 4 x 16 heads on 4 x 2048 x 128, bf16: 684 us with 256 workgroups, 618 with 512; forward of 8 x 8 x
    // 256 x 160, bf16: 26 us with parts of 128, 14 with 256; backward of 8 x 256 x 160, fp32: 71 us with parts of 64, 127 with
    // 256.  In fp32, workgroups whose registers let a compute unit hold two are cut to 512 too where queries are kept (dimensions up to
    // 80: forward of 2 x 8 x 1024 x 80 57 -> 51 us, of 8 x 4096 x 40 199 -> 164; of 4 x 8 x 512 x 96 39 -> 40, its backward 105 -> 114).
    const int64_t want = fp32 ? 256 : 512, least = fp32 ? 64 : 256;
    auto waves = [&](int64_t n) { return bh * ((n + 127) / 128) >= want / 2 ? 4 : 2; };
    auto blocks = [](int64_t n, int waves) { return (int)((n + 32 * waves - 1) / (32 * waves)); };
    p.waves = p.q_waves = waves(rows);
    // (blocks of one head's rows where that adds no more than a tenth)
    const int64_t whole = (q_len + 32 * p.waves - 1) / (32 * p.waves) * (32 * p.waves);
    p.q_pad = (int)(group > 1 && 10 * whole <= 11 * q_len ? whole : q_len);
    p.q_blocks = blocks(group * p.q_pad, p.q_waves);
    // Under `causal` the longest workgroup has twice the average's work: parts of no more than 64 tiles of queries (32 in fp32, which
    // take six times as long, and there of 1024 keys too).  Backward of 4 x 16 heads on 4 x 2048 x 128, bf16: 413 -> 389 us, of 16 on
    // 2 x 4096 x 128 641 -> 464; fp32, 2 x 8 x 2048 x 128: forward 194 -> 174, backward 713 -> 607.  Only while workgroups are few, up to four
    // times `want`: the longest go first, so that many balance by themselves, and parts cost a pass of their own and room.  Without that limit
    // 8 x 16384 x 128 takes in fp32 3561 us forward and 13680 backward for 2842 and 11268, in bf16 backward 2774 for 2510.
    auto at_most = [&](int splits, int64_t have, int64_t len, int64_t most) {
        int64_t s = causal && have > 0 ? (len + most - 1) / most : 1;
        if (s * have > 4 * want) s = 4 * want / have;
        return s > splits ? (int)(s < 32 ? s : 32) : splits;
    };
    p.q_splits = parts_of(kv_len, bh * p.q_blocks, ks <= 5 ? 512 : want, least);
    if (fp32) p.q_splits = at_most(p.q_splits, bh * p.q_blocks, kv_len, 1024);
    // keys form: few rows, or grids of the rows form that leave half of the compute units idle
    p.by_keys = rows <= few || bh * p.q_blocks * p.q_splits < 128;
    p.blocks = p.by_keys ? (int)((rows + few - 1) / few) : p.q_blocks;
    p.splits = p.by_keys ? parts_of(kv_len, bh * p.blocks, 512, fp32 ? 128 : 256) : p.q_splits;
    p.k_waves = waves(kv_len);
    p.k_blocks = blocks(kv_len, p.k_waves);
    const int tile = fp32 ? kKeysTile<3, 3> : ks <= 4 ? kKeysTile<1, 4> : ks <= 6 ? kKeysTile<1, 6> : kKeysTile<1, 8>;
    const int64_t tiles = group * ((q_len + tile - 1) / tile);
    // (workgroups of two wavefronts in fp32: 512, one wavefront per SIMD, up to dimension 80.  Backward of 64 heads of 4096 on 77 keys x
    // 40: 304 -> 238 us, of 1024 on 77 x 80 125 -> 104; kernel of 448 heads of 2437 on 25 x 96 442 -> 508, backward of 256 on 77 x 160
    // 108 -> 127.)
    const int64_t want_k = fp32 && p.k_waves == 2 && ks <= 5 ? 512 : want;
    p.k_splits = at_most(parts_of(tiles, bh * p.k_blocks, want_k, (least + tile - 1) / tile), bh * p.k_blocks, tiles, fp32 ? 32 : 64);
    return p;
}

}  // namespace fpq
