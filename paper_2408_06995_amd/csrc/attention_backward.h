// Attention, backward.  The probabilities are computed again from the rows' log-sums, p = exp(scale q.k - lse), so nothing of size
// q_len x kv_len is kept:
//   delta_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - delta_i),  dq_i = scale sum_j ds_ij k_j,
//   dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i   (i over the queries of all heads of the group).
// Two kernels, each of which owns what it writes: no atomics, the same bits in every run.  The price is that scores and dp are
// computed twice, seven products instead of five.
//   queries: a wavefront keeps 32 rows of q and do, reads tiles of keys and values, and sums dq^T = K^T ds^T; writes delta.
//   keys:    a wavefront keeps 32 keys and values, reads tiles of queries and do, and sums dk and dv over all heads of the group.
// As in the forward pass p and ds go into the next product from the registers they were computed in.
#pragma once
#include "attention.h"

namespace fpq {

template <int NP, int KS>
struct QueriesShape {
    static constexpr int KT = NP == 3 ? 32 : KS <= 4 ? 128 : KS <= 8 ? 64 : 32;
    typedef Feed<NP, KS, KT, 2> Tiles;
};

template <typename T, int KS>
__global__ __launch_bounds__(256, kPlanes<T> == 1 && KS <= 8 ? 2 : 1) void attention_queries_kernel(AttentionArgs a)
{
    constexpr int NP = kPlanes<T>, DT = (KS + 1) / 2;
    typedef QueriesShape<NP, KS> Sh;
    typedef typename Sh::Tiles Tiles;
    constexpr int KT = Sh::KT, PLANE = Tiles::PLANE / 2;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const Place at = place_of(a);
    const int b = at.bh / a.kv_heads, hk = at.bh - b * a.kv_heads;
    const int rows = a.group * a.q_len, n = keys_of(a, b);
    const int block = a.causal ? a.blocks - 1 - at.block : at.block;
    const int r_first = block * 128, r = r_first + 32 * wave + l32;
    const RowRange range = visible(a, n, r_first, min(r_first + 128, rows) - 1);
    const int kbeg = min((int64_t)at.split * a.per_split, (int64_t)range.hi), kend = min((int64_t)kbeg + a.per_split, (int64_t)range.hi);
    Tiles feed;
    feed.src[0] = a.fk;
    feed.src[1] = a.fv;
    feed.src[0].p += b * a.fk.s.b + hk * a.fk.s.h;
    feed.src[1].p += b * a.fv.s.b + hk * a.fv.s.h;
    feed.init(lds_address(lds), a.dim);
    if (kbeg < kend) feed.begin(kbeg, kend);

    const int rc = min(r, rows - 1), g = rc / a.q_len, i = rc - g * a.q_len, head = hk * a.group + g;
    const int end = a.causal ? max(0, min(n, i + n - a.q_len + 1)) : n;
    const size_t row_id = (size_t)at.bh * rows + rc;
    Frag<NP> qf[KS], gf[KS];
    float delta = 0.0f;
    {
        const T* q = static_cast<const T*>(a.q) + b * a.qs.b + i * a.qs.t + head * a.qs.h;
        const T* o = static_cast<const T*>(a.o) + b * a.os.b + i * a.os.t + head * a.os.h;
        const T* go = static_cast<const T*>(a.go) + b * a.gos.b + i * a.gos.t + head * a.gos.h;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            float v[8], w[8];
            row8(q, 16 * s + 8 * h, a.dim, a.vec, v);
            qf[s] = frag_of<NP>(v);
            row8(go, 16 * s + 8 * h, a.dim, a.vec, v);
            gf[s] = frag_of<NP>(v);
            row8(o, 16 * s + 8 * h, a.dim, a.vec, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf(v[e], w[e], delta);
        }
        delta += __shfl_xor(delta, 32);
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
                const Frag<NP> ds = frag_of<NP>(v);
#pragma unroll
                for (int d = 0; d < DT; ++d) mma<NP>(acc[d], cols_at<NP, KS>(kt, PLANE, places, 16 * t, d), ds);
            }
            kt += 32 * Places<KS>::RS;
            vt += 32 * Places<KS>::RS;
        }
    }
    if (r >= rows) return;
    if (h == 0 && at.split == 0) reinterpret_cast<float2*>(a.stats)[row_id] = make_float2(lse2, delta);
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

// WHAT: 1 dv, 2 dk, 3 both in one pass.  In fp32 at the largest dimension the planes of 32 keys and values and both sums do not fit
// a wavefront's registers together: two passes.  VLDS: the workgroup's values stay in LDS and not in registers, which lets two
// workgroups share a compute unit at a dimension of 128 in bf16.
template <int NP, int KS>
struct KeysShape {
    static constexpr int QT = kKeysTile<NP, KS>;
    static constexpr bool VLDS = NP == 1 && KS > 6 && KS <= 8;
    typedef Feed<NP, KS, QT, 2> Tiles;
    typedef Feed<NP, KS, 128, 1> Values;
    static constexpr int STATS = Tiles::LDS, PAIRS = QT < 32 ? 32 : QT;        // two buffers of the rows' pairs of log-sum and delta
    static constexpr int VALUES = STATS + 2 * PAIRS * 8;
    static constexpr int LDS = VALUES + (VLDS ? Values::TILE : 0);
};

template <typename T, int KS, int WHAT>
__global__ __launch_bounds__(256, kPlanes<T> == 1 && KS <= 8 ? 2 : 1) void attention_keys_kernel(AttentionArgs a)
{
    constexpr int NP = kPlanes<T>, DT = (KS + 1) / 2;
    typedef KeysShape<NP, KS> Sh;
    typedef typename Sh::Tiles Tiles;
    constexpr int QT = Sh::QT, PLANE = Tiles::PLANE / 2;
    constexpr bool DV = WHAT & 1, DK = WHAT & 2, VLDS = Sh::VLDS && DK;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const Place at = place_of(a);
    const int b = at.bh / a.kv_heads, hk = at.bh - b * a.kv_heads;
    const int n = keys_of(a, b), off = n - a.q_len, j_first = at.block * 128, key = j_first + 32 * wave + l32;
    // tiles of queries, head by head, from the first that sees a key of this block
    const int tiles_all = (a.q_len + QT - 1) / QT, skip = a.causal ? min(max(0, j_first - off) / QT, tiles_all) : 0;
    const int per_head = j_first < n ? tiles_all - skip : 0, per = max(per_head, 1);
    const int64_t tiles = (int64_t)per_head * a.group;
    const int64_t tbeg = min((int64_t)at.split * a.per_split, tiles), tend = min(tbeg + a.per_split, tiles);
    Tiles feed;
    int g = (int)(tbeg / per), i0 = (skip + (int)(tbeg - (int64_t)g * per)) * QT, slot = 0;
    feed.src[0] = a.fq;
    feed.src[1] = a.fgo;
    feed.src[0].p += b * a.fq.s.b + (hk * a.group + g) * a.fq.s.h;
    feed.src[1].p += b * a.fgo.s.b + (hk * a.group + g) * a.fgo.s.h;
    feed.init(lds_address(lds), a.dim);
    // the rows' pairs come with a tile; rows past the last get zeros, and so p = 1 next to zeros of q and do
    auto begin = [&](int g, int i0) {
        feed.begin(i0, a.q_len);
        if (wave == 0) {
            const v4i r = make_rsrc(a.stats + 2 * (((size_t)at.bh * a.group + g) * a.q_len + i0), 8u * (unsigned)min(QT, a.q_len - i0));
#pragma unroll
            for (int e = 0; e < Sh::PAIRS / 32; ++e) dma4(r, 4u * lane + 256u * e, lds_address(lds) + Sh::STATS + slot * Sh::PAIRS * 8 + 256 * e);
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
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                float x[8];
                row8(k, 16 * s + 8 * h, a.dim, a.vec, x);
                kf[s] = frag_of<NP>(x);
                if constexpr (DK && !VLDS) {
                    row8(v, 16 * s + 8 * h, a.dim, a.vec, x);
                    vf[s] = frag_of<NP>(x);
                }
            }
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
        const float* ls = reinterpret_cast<const float*>(lds + Sh::STATS) + (slot ^ 1) * 2 * Sh::PAIRS + 8 * h;
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
            v16f s = zero16(), dp = zero16();
#pragma unroll
            for (int x = 0; x < KS; ++x) {
                mma<NP>(s, rows_at<NP, KS>(qt, PLANE, places, 0, x), kf[x]);
                if constexpr (VLDS)
                    mma<NP>(dp, rows_at<NP, KS>(gt, PLANE, places, 0, x), rows_at<NP, KS>(vt, 0, places, 0, x));
                else if constexpr (DK)
                    mma<NP>(dp, rows_at<NP, KS>(gt, PLANE, places, 0, x), vf[x]);
            }
            if (a.causal && j_first + 127 > i + off) {
                const int from = key - off - i;    // the first query that sees the key
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (8 * (e / 4) + 4 * h + e % 4 < from) s[e] = -kInf;
            }
#pragma unroll
            for (int e = 0; e < 16; e += 2) {      // two rows' pairs at a time
                const float4 y = *reinterpret_cast<const float4*>(ls + 2 * (8 * (e / 4) + e % 4));
                s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c, -y.x));
                s[e + 1] = __builtin_amdgcn_exp2f(fmaf(s[e + 1], c, -y.z));
                if constexpr (DK) {
                    dp[e] = s[e] * (dp[e] - y.y);
                    dp[e + 1] = s[e + 1] * (dp[e + 1] - y.w);
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                float v[8];
                if constexpr (DV) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = s[8 * x + e];
                    const Frag<NP> p = frag_of<NP>(v);
#pragma unroll
                    for (int d = 0; d < DT; ++d) mma<NP>(av[d], p, cols_at<NP, KS>(gt, PLANE, places, 16 * x, d));
                }
                if constexpr (DK) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = dp[8 * x + e];
                    const Frag<NP> ds = frag_of<NP>(v);
#pragma unroll
                    for (int d = 0; d < DT; ++d) mma<NP>(ak[d], ds, cols_at<NP, KS>(qt, PLANE, places, 16 * x, d));
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

// out[b, t, head] = the sum of the parts, in order.
template <typename T>
__global__ __launch_bounds__(256) void attention_sum_kernel(const float* part, int parts, size_t part_stride, size_t n, int len, int heads, int dim,
                                                            T* out, Strides st)
{
    for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (size_t)gridDim.x * 256) {
        float v = part[e];
        for (int s = 1; s < parts; ++s) v += part[s * part_stride + e];
        const size_t row = e / dim, bh = row / len;
        const int64_t b = bh / heads, head = bh - (size_t)b * heads;
        out[b * st.b + (int64_t)(row - bh * len) * st.t + head * st.h + (int64_t)(e - row * dim)] = (T)v;
    }
}

template <typename T>
int launch_sum(const float* part, int parts, size_t part_stride, size_t rows, int len, int heads, int dim, void* out, const Strides& st, hipStream_t s)
{
    const size_t n = rows * dim, want = (n + 255) / 256;
    attention_sum_kernel<T><<<dim3((unsigned)(want < 4096 ? want : 4096)), dim3(256), 0, s>>>(part, parts, part_stride, n, len, heads, dim,
                                                                                             static_cast<T*>(out), st);
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

template <typename T, int KS>
int launch_queries(const AttentionArgs& a, hipStream_t s)
{
    constexpr int lds = QueriesShape<kPlanes<T>, KS>::Tiles::LDS;
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&attention_queries_kernel<T, KS>), lds, done)) return FPQ_ERR_LAUNCH;
    const int64_t grid = (int64_t)a.batch * a.kv_heads * a.blocks * a.splits;
    attention_queries_kernel<T, KS><<<dim3((unsigned)grid), dim3(256), lds, s>>>(a);
    return FPQ_OK;
}

template <typename T, int KS, int WHAT>
int launch_keys(const AttentionArgs& a, hipStream_t s)
{
    constexpr int lds = KeysShape<kPlanes<T>, KS>::LDS;
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&attention_keys_kernel<T, KS, WHAT>), lds, done)) return FPQ_ERR_LAUNCH;
    const int64_t grid = (int64_t)a.batch * a.kv_heads * a.blocks * a.splits;
    attention_keys_kernel<T, KS, WHAT><<<dim3((unsigned)grid), dim3(256), lds, s>>>(a);
    return FPQ_OK;
}

template <typename T, int KS>
int launch_both(const AttentionArgs& aq, const AttentionArgs& ak, hipStream_t s)
{
    // (the keys kernel reads the pairs that the queries kernel writes)
    int st = aq.q_len > 0 ? launch_queries<T, KS>(aq, s) : FPQ_OK;
    if (st != FPQ_OK || ak.kv_len == 0) return st;
    if constexpr (sizeof(T) == 4 && KS > 8) {
        st = launch_keys<T, KS, 1>(ak, s);
        return st != FPQ_OK ? st : launch_keys<T, KS, 2>(ak, s);
    } else {
        return launch_keys<T, KS, 3>(ak, s);
    }
}

template <typename T>
int launch_backward(const AttentionArgs& aq, const AttentionArgs& ak, hipStream_t s)
{
    const int ks = (aq.dim + 15) / 16;
    int st = ks <= 3 ? launch_both<T, 3>(aq, ak, s) : ks == 4 ? launch_both<T, 4>(aq, ak, s) : ks == 5 ? launch_both<T, 5>(aq, ak, s)
           : ks == 6 ? launch_both<T, 6>(aq, ak, s) : ks <= 8 ? launch_both<T, 8>(aq, ak, s) : launch_both<T, 10>(aq, ak, s);
    if (st != FPQ_OK) return st;
    if (aq.splits > 1) {
        const size_t rows = (size_t)aq.batch * aq.kv_heads * aq.group * aq.q_len;
        st = launch_sum<T>(aq.part, aq.splits, rows * aq.dim, rows, aq.q_len, aq.kv_heads * aq.group, aq.dim, aq.gq, aq.gqs, s);
        if (st != FPQ_OK) return st;
    }
    if (ak.splits > 1) {
        const size_t rows = (size_t)ak.batch * ak.kv_heads * ak.kv_len;
        st = launch_sum<T>(ak.part, ak.splits, 2 * rows * ak.dim, rows, ak.kv_len, ak.kv_heads, ak.dim, ak.gk, ak.gks, s);
        if (st != FPQ_OK) return st;
        st = launch_sum<T>(ak.part + rows * ak.dim, ak.splits, 2 * rows * ak.dim, rows, ak.kv_len, ak.kv_heads, ak.dim, ak.gv, ak.gvs, s);
        if (st != FPQ_OK) return st;
    }
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

}  // namespace fpq
