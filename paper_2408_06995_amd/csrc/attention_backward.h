// Attention, backward.  The probabilities are computed again from the rows' log-sums, p = exp(scale q.k - lse), so nothing of size
// q_len x kv_len is kept:
//   delta_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - delta_i),  dq_i = scale sum_j ds_ij k_j,
//   dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i   (i over the queries of all heads of the group).
// Two kernels, each of which owns what it writes: no atomics, the same bits in every run.  The price is that scores and dp are
// computed twice, seven products instead of five.
//   queries: a wavefront keeps 32 rows of q and do, reads tiles of keys and values, and sums dq^T = K^T ds^T; writes delta.
//   keys:    a wavefront keeps 32 keys and values, reads tiles of queries and do, and sums dk and dv over all heads of the group.
// As in the forward pass p and ds go into the next product from the registers they were computed in.
//
// bf16, 4 x 16 heads on 4 of 2048 x 128: 618 us, 556 TFLOP/s of five products, causal 381; 4 x 8 of 4096 x 40: 597 us, 360 (padded
// as the forward pass; the three products with p and ds are taken twice, for their two planes).  Neither unit is full: the matrix unit is
// busy 0.47 - 0.52 of the cycles, vector instructions 0.62 - 0.70, LDS 0.17 - 0.26 (dimension 40); two or three wavefronts per SIMD do not
// cover a tile's chain of product, exponential, product.  fp32, 2 x 8 of 1024 x 80: 143 us, 94 TFLOP/s: six matrix steps for each product.
#pragma once
#include "attention.h"

namespace fpq {

// What the keys kernel needs of a row: -log-sum / scale and -delta, the initial values of a score and of dp in the matrix unit (a row
// without keys: -infinity, and so p = 0).  32 rows of a head at a time, first those, then these.
__device__ __forceinline__ size_t stats_at(const AttentionArgs& a, size_t head, int i)
{
    return (head * ((a.q_len + 31) / 32) + (i >> 5)) * 64 + (i & 31);
}

template <int NP, int KS, int NW>
struct QueriesShape {
    static constexpr int KT = NP == 3 || KS > 8 ? 32 : 64;
    typedef Feed<NP, KS, KT, 2, NW> Tiles;
};

template <typename T, int KS, int NW>
__global__ __launch_bounds__(64 * NW, kPlanes<T> == 1 ? (KS <= 4 ? 3 : KS <= 8 ? 2 : 1) : KS <= 5 ? 2 : 1) void attention_queries_kernel(AttentionArgs a)
{
    constexpr int NP = kPlanes<T>, PP = kPlanesP<T>, DT = (KS + 1) / 2;
    typedef QueriesShape<NP, KS, NW> Sh;
    typedef typename Sh::Tiles Tiles;
    constexpr int KT = Sh::KT, PLANE = Tiles::PLANE / 2;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const Place at = place_of(a);
    const int b = at.bh / a.kv_heads, hk = at.bh - b * a.kv_heads;
    const int rows = a.group * a.q_len, n = keys_of(a, b);
    const RowBlock mine = row_block<NW>(a, n, at.block, wave, l32);
    const RowRange range = mine.range;
    const Part keys = part_of(range.hi, KT, at.split, a.splits);
    const int kbeg = (int)keys.beg, kend = (int)keys.end;
    Tiles feed;
    feed.src[0] = a.fk;
    feed.src[1] = a.fv;
    feed.src[0].p += b * a.fk.s.b + hk * a.fk.s.h;
    feed.src[1].p += b * a.fv.s.b + hk * a.fv.s.h;
    feed.init(lds_address(lds), a.dim);
    if (kbeg < kend) feed.begin(kbeg, kend);

    const int i = mine.i, g = mine.g, end = mine.end, head = hk * a.group + g;
    const size_t row_id = (size_t)at.bh * rows + g * a.q_len + i;
    Frag<NP> qf[KS], gf[KS];
    float delta = 0.0f;
    {
        float v[KS][8], w[KS][8];
        row_all<T, KS>(static_cast<const T*>(a.go) + b * a.gos.b + i * a.gos.t + head * a.gos.h, h, a.dim, a.vec, v);
        row_all<T, KS>(static_cast<const T*>(a.o) + b * a.os.b + i * a.os.t + head * a.os.h, h, a.dim, a.vec, w);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            gf[s] = frag_of<NP>(v[s]);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf(v[s][e], w[s][e], delta);
        }
        delta += __shfl_xor(delta, 32);
        row_frags<T, KS, NP>(static_cast<const T*>(a.q) + b * a.qs.b + i * a.qs.t + head * a.qs.h, h, a.dim, a.vec, qf);
    }
    const float log_sum = a.lse[row_id];
    const float c = a.scale * kLog2e, lse2 = log_sum == -kInf ? kInf : log_sum * kLog2e;   // a row without keys: every p is 0
    Places<KS> places;
    places.init(lane);
    v16f acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = zero16();
    for (int j0 = kbeg; j0 < kend; j0 += KT) {
        feed.ready();
        const __bf16* kt = reinterpret_cast<const __bf16*>(lds) + feed.at(0);
        const __bf16* vt = reinterpret_cast<const __bf16*>(lds) + feed.at(1);
        if (j0 + KT < kend) feed.begin(j0 + KT, kend);
#pragma unroll 1
        for (int j = j0; j < min(j0 + KT, kend); j += 32) {
            v16f s = zero16(), dp = zero16();
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                mma<NP>(s, rows_at<NP, KS>(kt, PLANE, places, 0, t), qf[t]);
                mma<NP>(dp, rows_at<NP, KS>(vt, PLANE, places, 0, t), gf[t]);
            }
            if (j + 32 > min(range.lo, kend)) {
                const int left = end - j;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (8 * (e / 4) + 4 * h + e % 4 >= left) s[e] = -kInf;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c, -lse2));
            if (j == 0) {
                // Rows of at most 32 keys have them all here: their delta from the products themselves instead of from o, whose
                // rounding weighs most where o is an average of few values.
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 16; ++e) sum = fmaf(s[e], dp[e], sum);
                sum += __shfl_xor(sum, 32);
                if (end <= 32) delta = sum;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] *= dp[e] - delta;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = s[8 * t + e];
                const Frag<PP> ds = frag_of<PP>(v);
#pragma unroll
                for (int d = 0; d < DT; ++d) mma<NP>(acc[d], cols_at<NP, KS>(kt, PLANE, places, 16 * t, d), ds);
            }
            kt += 32 * Places<KS>::RS;
            vt += 32 * Places<KS>::RS;
        }
    }
    if (!mine.in) return;
    if (h == 0 && at.split == 0) {
        float* const st = a.stats + stats_at(a, (size_t)at.bh * a.group + g, i);
        st[0] = log_sum == -kInf ? -kInf : -log_sum / a.scale;
        st[32] = -delta;
    }
    float* const part = a.splits > 1 ? a.part + (size_t)at.split * a.batch * a.kv_heads * rows * a.dim : nullptr;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int col = 32 * d + 8 * t + 4 * h;
            const float v[4] = {acc[d][4 * t] * a.scale, acc[d][4 * t + 1] * a.scale, acc[d][4 * t + 2] * a.scale, acc[d][4 * t + 3] * a.scale};
            if (part)
                store4(part + row_id * a.dim, col, a.dim, a.dim % 4 == 0, v);
            else
                store4(static_cast<T*>(a.gq) + b * a.gqs.b + i * a.gqs.t + head * a.gqs.h, col, a.dim, a.vec_out, v);
        }
}

// WHAT: 1 dv, 2 dk, 3 both in one pass.  In fp32 at dimensions past 96 the planes of 32 keys and values and both sums do not fit
// a wavefront's registers together: two passes.  VLDS: the workgroup's values stay in LDS and not in registers, which lets two
// workgroups share a compute unit at a dimension of 128 in bf16.
template <int NP, int KS, int NW>
struct KeysShape {
    static constexpr int QT = kKeysTile<NP, KS>;
    static constexpr bool VLDS = NP == 1 && KS > 6 && KS <= 8;
    typedef Feed<NP, KS, QT, 2, NW> Tiles;
    typedef Feed<NP, KS, 32 * NW, 1, NW> Values;
    static constexpr int STATS = Tiles::LDS;                                   // two buffers of the rows' two statistics
    static constexpr int VALUES = STATS + 2 * QT * 8;
    static constexpr int LDS = VALUES + (VLDS ? Values::TILE : 0);
};

template <typename T, int KS, int WHAT, int NW>
__global__ __launch_bounds__(64 * NW, kPlanes<T> == 1 && KS <= 8 ? 2 : 1) void attention_keys_kernel(AttentionArgs a)
{
    constexpr int NP = kPlanes<T>, PP = kPlanesP<T>, DT = (KS + 1) / 2;
    typedef KeysShape<NP, KS, NW> Sh;
    typedef typename Sh::Tiles Tiles;
    constexpr int QT = Sh::QT, PLANE = Tiles::PLANE / 2;
    constexpr bool DV = WHAT & 1, DK = WHAT & 2, VLDS = Sh::VLDS && DK;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const Place at = place_of(a);
    const int b = at.bh / a.kv_heads, hk = at.bh - b * a.kv_heads;
    const int n = keys_of(a, b), off = n - a.q_len, j_first = at.block * 32 * NW, key = j_first + 32 * wave + l32;
    // tiles of queries, head by head, from the first that sees a key of this block
    const int tiles_all = (a.q_len + QT - 1) / QT, skip = a.causal ? min(max(0, j_first - off) / QT, tiles_all) : 0;
    const int per_head = j_first < n ? tiles_all - skip : 0, per = max(per_head, 1);
    const int64_t tiles = (int64_t)per_head * a.group;
    const Part part = part_of(tiles, 1, at.split, a.splits);
    const int64_t tbeg = part.beg, tend = part.end;
    Tiles feed;
    int g = (int)(tbeg / per), i0 = (skip + (int)(tbeg - (int64_t)g * per)) * QT, slot = 0;
    feed.src[0] = a.fq;
    feed.src[1] = a.fgo;
    feed.src[0].p += b * a.fq.s.b + (hk * a.group + g) * a.fq.s.h;
    feed.src[1].p += b * a.fgo.s.b + (hk * a.group + g) * a.fgo.s.h;
    feed.init(lds_address(lds), a.dim);
    // the rows' statistics come with a tile; rows past the last get zeros, and so p = 1 next to zeros of q and do
    auto begin = [&](int g, int i0) {
        feed.begin(i0, a.q_len);
        if (wave == 0) {
            const v4i r = make_rsrc(a.stats + stats_at(a, (size_t)at.bh * a.group + g, i0), QT * 8);
#pragma unroll
            for (int e = 0; e < QT / 32; ++e)
                dma4(r, i0 + 32 * e + l32 < a.q_len ? 4u * lane + 256u * e : 0x80000000u, lds_address(lds) + Sh::STATS + slot * QT * 8 + 256 * e);
        }
        slot ^= 1;
    };
    if (tbeg < tend) {
        if constexpr (VLDS) {
            typename Sh::Values values;
            values.src[0] = a.fv;
            values.src[0].p += b * a.fv.s.b + hk * a.fv.s.h;
            values.init(lds_address(lds) + Sh::VALUES, a.dim);
            values.begin(j_first, n);
        }
        begin(g, i0);
    }
    Frag<NP> kf[KS], vf[DK && !VLDS ? KS : 1];
    {
        const int kc = max(0, min(key, n - 1));
        const T* k = static_cast<const T*>(a.k) + b * a.ks.b + kc * a.ks.t + hk * a.ks.h;
        const T* v = static_cast<const T*>(a.v) + b * a.vs.b + kc * a.vs.t + hk * a.vs.h;
        if (tbeg < tend) {                         // (no tile: no key either, perhaps)
            row_frags<T, KS, NP>(k, h, a.dim, a.vec, kf);
            if constexpr (DK && !VLDS) row_frags<T, KS, NP>(v, h, a.dim, a.vec, vf);
        }
    }
    Places<KS> places;
    places.init(lane);
    const __bf16* const vt = reinterpret_cast<const __bf16*>(lds + Sh::VALUES) + 32 * wave * Places<KS>::RS;
    v16f av[DV ? DT : 1], ak[DK ? DT : 1];
#pragma unroll
    for (int d = 0; d < DT; ++d) {
        if constexpr (DV) av[d] = zero16();
        if constexpr (DK) ak[d] = zero16();
    }
    const float c = a.scale * kLog2e;
    for (int64_t t = tbeg; t < tend; ++t) {
        feed.ready();
        const __bf16* qt = reinterpret_cast<const __bf16*>(lds) + feed.at(0);
        const __bf16* gt = reinterpret_cast<const __bf16*>(lds) + feed.at(1);
        const float* ls = reinterpret_cast<const float*>(lds + Sh::STATS) + (slot ^ 1) * 2 * QT + 4 * h;
        const int i_now = i0, i_end = min(i0 + QT, a.q_len);
        if (t + 1 < tend) {
            i0 += QT;
            if (i0 >= a.q_len) {                   // the next head of the group
                i0 = skip * QT;
                ++g;
                feed.src[0].p += a.fq.s.h;
                feed.src[1].p += a.fgo.s.h;
            }
            begin(g, i0);
        }
#pragma unroll 1
        for (int i = i_now; i < i_end; i += 32) {
            v16f s, dp, log_sum, delta;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const v4f y = *reinterpret_cast<const v4f*>(ls + 8 * e), z = *reinterpret_cast<const v4f*>(ls + 32 + 8 * e);
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    log_sum[4 * e + f] = y[f];
                    delta[4 * e + f] = z[f];
                }
            }
            // (fp32 sums the small parts of its products first: from zero)
            s = NP == 1 ? log_sum : zero16();
            dp = NP == 1 ? delta : zero16();
#pragma unroll
            for (int x = 0; x < KS; ++x) {
                mma<NP>(s, rows_at<NP, KS>(qt, PLANE, places, 0, x), kf[x]);
                if constexpr (VLDS)
                    mma<NP>(dp, rows_at<NP, KS>(gt, PLANE, places, 0, x), rows_at<NP, KS>(vt, 0, places, 0, x));
                else if constexpr (DK)
                    mma<NP>(dp, rows_at<NP, KS>(gt, PLANE, places, 0, x), vf[x]);
            }
            if (a.causal && j_first + 32 * NW - 1 > i + off) {
                const int from = key - off - i;    // the first query that sees the key
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (8 * (e / 4) + 4 * h + e % 4 < from) s[e] = -kInf;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[e] = __builtin_amdgcn_exp2f((NP == 1 ? s[e] : s[e] + log_sum[e]) * c);
                if constexpr (DK) dp[e] = s[e] * (NP == 1 ? dp[e] : dp[e] + delta[e]);
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                float v[8];
                if constexpr (DV) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = s[8 * x + e];
                    const Frag<PP> p = frag_of<PP>(v);
#pragma unroll
                    for (int d = 0; d < DT; ++d) mma<PP>(av[d], p, cols_at<NP, KS>(gt, PLANE, places, 16 * x, d));
                }
                if constexpr (DK) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = dp[8 * x + e];
                    const Frag<PP> ds = frag_of<PP>(v);
#pragma unroll
                    for (int d = 0; d < DT; ++d) mma<PP>(ak[d], ds, cols_at<NP, KS>(qt, PLANE, places, 16 * x, d));
                }
            }
            qt += 32 * Places<KS>::RS;
            gt += 32 * Places<KS>::RS;
            ls += 64;
        }
    }
    // lane: column l32 of the 16 keys that its values stand for; keys that the sample does not have get zeros
    const size_t keys_all = (size_t)a.batch * a.kv_heads * a.kv_len;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int j = j_first + 32 * wave + 8 * (e / 4) + 4 * h + e % 4;
        if (j >= a.kv_len) continue;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int col = 32 * d + l32;
            if (col >= a.dim) continue;
            if constexpr (DV) {
                const float v = j < n ? av[d][e] : 0.0f;
                if (a.splits > 1)
                    a.part[((size_t)at.split * 2 * keys_all + keys_all + (size_t)at.bh * a.kv_len + j) * a.dim + col] = v;
                else
                    static_cast<T*>(a.gv)[b * a.gvs.b + j * a.gvs.t + hk * a.gvs.h + col] = (T)v;
            }
            if constexpr (DK) {
                const float v = j < n ? ak[d][e] * a.scale : 0.0f;
                if (a.splits > 1)
                    a.part[((size_t)at.split * 2 * keys_all + (size_t)at.bh * a.kv_len + j) * a.dim + col] = v;
                else
                    static_cast<T*>(a.gk)[b * a.gks.b + j * a.gks.t + hk * a.gks.h + col] = (T)v;
            }
        }
    }
}

// out[b, t, head] = the sum of the parts, in order: up to three results in one launch, a row per 32 lanes.
struct SumOut {
    const float* part;
    size_t stride;              // from one part to the next
    int parts, len, heads;
    int64_t rows;               // 0: none
    void* out;
    Strides s;
};
struct SumArgs {
    SumOut m[3];
    int dim;
};
template <typename T>
__global__ __launch_bounds__(256) void attention_sum_kernel(SumArgs a)
{
    const SumOut& m = a.m[blockIdx.y];
    const int lane = threadIdx.x & 31;
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < m.rows; row += (int64_t)gridDim.x * 8) {
        const int64_t bh = row / m.len, b = bh / m.heads;
        T* const out = static_cast<T*>(m.out) + b * m.s.b + (row - bh * m.len) * m.s.t + (bh - b * m.heads) * m.s.h;
        const float* const in = m.part + row * a.dim;
        float v[5] = {0, 0, 0, 0, 0};
        for (int s0 = 0; s0 < m.parts; s0 += 4) {
            float p[4][5];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int d = 0; d < 5; ++d) p[u][d] = in[min(s0 + u, m.parts - 1) * m.stride + min(lane + 32 * d, a.dim - 1)];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int d = 0; d < 5; ++d) v[d] += s0 + u < m.parts ? p[u][d] : 0.0f;
        }
#pragma unroll
        for (int d = 0; d < 5; ++d)
            if (lane + 32 * d < a.dim) out[lane + 32 * d] = (T)v[d];
    }
}

template <typename T, int KS, int NW>
int launch_queries(const AttentionArgs& a, hipStream_t s)
{
    constexpr int lds = QueriesShape<kPlanes<T>, KS, NW>::Tiles::LDS;
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&attention_queries_kernel<T, KS, NW>), lds, done)) return FPQ_ERR_LAUNCH;
    const int64_t grid = (int64_t)a.batch * a.kv_heads * a.blocks * a.splits;
    attention_queries_kernel<T, KS, NW><<<dim3((unsigned)grid), dim3(64 * NW), lds, s>>>(a);
    return FPQ_OK;
}

template <typename T, int KS, int WHAT, int NW>
int launch_keys(const AttentionArgs& a, hipStream_t s)
{
    constexpr int lds = KeysShape<kPlanes<T>, KS, NW>::LDS;
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&attention_keys_kernel<T, KS, WHAT, NW>), lds, done)) return FPQ_ERR_LAUNCH;
    const int64_t grid = (int64_t)a.batch * a.kv_heads * a.blocks * a.splits;
    attention_keys_kernel<T, KS, WHAT, NW><<<dim3((unsigned)grid), dim3(64 * NW), lds, s>>>(a);
    return FPQ_OK;
}

template <typename T, int KS, int WHAT>
int launch_keys(const AttentionArgs& a, int waves, hipStream_t s)
{
    return waves == 4 ? launch_keys<T, KS, WHAT, 4>(a, s) : launch_keys<T, KS, WHAT, 2>(a, s);
}

template <typename T, int KS>
int launch_queries(const AttentionArgs& a, int waves, hipStream_t s)
{
    return waves == 4 ? launch_queries<T, KS, 4>(a, s) : launch_queries<T, KS, 2>(a, s);
}
template <typename T, int KS>
int launch_both(const AttentionArgs& aq, const AttentionArgs& ak, const AttentionPlan& p, hipStream_t s)
{
    // (the keys kernel reads what the queries kernel writes)
    int st = FPQ_OK;
    if (aq.q_len > 0) st = launch_queries<T, KS>(aq, p.q_waves, s);
    if (st != FPQ_OK || ak.kv_len == 0) return st;
    if constexpr (sizeof(T) == 4 && KS > 6) {
        st = launch_keys<T, KS, 1>(ak, p.k_waves, s);
        return st != FPQ_OK ? st : launch_keys<T, KS, 2>(ak, p.k_waves, s);
    } else {
        return launch_keys<T, KS, 3>(ak, p.k_waves, s);
    }
}

template <typename T>
int launch_backward(const AttentionArgs& aq, const AttentionArgs& ak, const AttentionPlan& p, hipStream_t s)
{
    const int ks = (aq.dim + 15) / 16;
    int st = ks <= 3 ? launch_both<T, 3>(aq, ak, p, s) : ks == 4 ? launch_both<T, 4>(aq, ak, p, s) : ks == 5 ? launch_both<T, 5>(aq, ak, p, s)
           : ks == 6 ? launch_both<T, 6>(aq, ak, p, s) : ks <= 8 ? launch_both<T, 8>(aq, ak, p, s) : launch_both<T, 10>(aq, ak, p, s);
    if (st != FPQ_OK) return st;
    SumArgs sums{};
    sums.dim = aq.dim;
    int count = 0;
    int64_t most = 0;
    auto add = [&](const AttentionArgs& a, const float* part, size_t stride, int len, int heads, void* out, const Strides& st) {
        const int64_t rows = (int64_t)a.batch * heads * len;
        sums.m[count++] = SumOut{part, stride, a.splits, len, heads, rows, out, st};
        if (rows > most) most = rows;
    };
    if (aq.splits > 1)
        add(aq, aq.part, (size_t)aq.batch * aq.kv_heads * aq.group * aq.q_len * aq.dim, aq.q_len, aq.kv_heads * aq.group, aq.gq, aq.gqs);
    if (ak.splits > 1) {
        const size_t keys = (size_t)ak.batch * ak.kv_heads * ak.kv_len * ak.dim;
        add(ak, ak.part, 2 * keys, ak.kv_len, ak.kv_heads, ak.gk, ak.gks);
        add(ak, ak.part + keys, 2 * keys, ak.kv_len, ak.kv_heads, ak.gv, ak.gvs);
    }
    if (most) {
        const int64_t want = (most + 7) / 8;
        attention_sum_kernel<T><<<dim3((unsigned)(want < 16384 ? want : 16384), count), dim3(256), 0, s>>>(sums);
    }
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

}  // namespace fpq
