// Attention, forward: o = softmax(scale q k^T) v in one pass over the keys, with the running maximum m (a lower bound of it, within
// 2^8 after the exponential) and sum l of a row's exponentials; o and l are rescaled when m grows.  m, l and o are held in 32
// bits; the probabilities keep 16 bits for bf16 results and 24 for fp32 where they enter the second product.
//
// A wavefront has 32 rows of queries in registers and takes S^T = K Q^T per 32 keys, so that a lane holds 16 scores of one row and
// its maximum and sum need one exchange with the lane 32 on; P^T is then the operand of O^T = V^T P^T as it lies.
//   rows form: two or four wavefronts with 32 rows each share tiles of keys and values in LDS.
//   keys form: the wavefronts share one or two sets of 32 rows and divide each tile's keys; their results are joined at the end.
//     For few rows: single tokens, small batches.
//
// Rows form, useful operations (4 q_len kv_len dim per head): bf16, 4 x 16 heads on 4 of 2048 x 128: 215 us, 640 TFLOP/s, causal 113;
// 4 x 16 of 2048 x 64: 116 us, 592; 4 x 8 of 4096 x 40: 203 us, 423 (dimensions are whole steps of 16 and results of 32 columns, 48 and
// 64 here; the second product is taken twice, for two planes of the probabilities).  What binds: vector instructions, above all 32
// exponentials at a quarter of the rate per 2048 scores and one multiply-add, one sum and the split into planes each (busy 0.77 of the
// cycles at dimension 40, the matrix unit 0.45).  fp32, 2 x 8 of 2048 x 64: 106 us, 162 TFLOP/s: six products and the splitting of the
// probabilities into planes.
// Keys form: 16 x 32 heads on 8, one query, up to 4096 keys of dimension 128, bf16: 36 us, 5.4 TB/s of keys and values, and 5 for the
// join; 8 heads of 64 x 64 x 160 in fp32: 15 us, latency of eight workgroups (loads, split, two products, the join in LDS).
#pragma once
#include "attention.h"

namespace fpq {

// The softmax of NS x 32 keys: scores in, exponentials out.  `left` > 0 under MASKED: keys from it on are hidden from the row.
template <int NS, int DT>
__device__ __forceinline__ void softmax_step(v16f (&s)[NS], v16f (&acc)[DT], float& m, float& l, float c, float slack, bool masked, int left, int h)
{
    if (masked) {
#pragma unroll
        for (int u = 0; u < NS; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (32 * u + 8 * (e / 4) + 4 * h + e % 4 >= left) s[u][e] = -kInf;
    }
    float top = s[0][0];
#pragma unroll
    for (int u = 0; u < NS; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
    top = fmaxf(top, __shfl_xor(top, 32));
    // m follows the maximum only when it lags by more than a factor of 2^8: until then exponentials are up to 2^8, which
    // neither the sums nor the operands notice, and o and l need no rescaling.
    if (__any(top > m + slack)) {
        const float next = fmaxf(m, top), by = m == next ? 1.0f : __builtin_amdgcn_exp2f((m - next) * c);
        m = next;
        l *= by;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[d][e] *= by;
    }
    const float mc = m == -kInf ? 0.0f : m * c;
#pragma unroll
    for (int u = 0; u < NS; ++u) {
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[u][e] = __builtin_amdgcn_exp2f(fmaf(s[u][e], c, -mc));
            sum[e % 4] += s[u][e];
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
}

__device__ __forceinline__ float inverse(float sum)       // no key: zeros; a sum that is no number stays one
{
    return sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
}

template <int NP, int KS, int NW>
struct RowsShape {
    static constexpr int KT = NP == 3 || KS > 8 ? 32 : 64, NS = KT < 64 ? 1 : 2;
    typedef Feed<NP, KS, KT, 2, NW> Tiles;
};

template <typename T, int KS, int NW>
__global__ __launch_bounds__(64 * NW, kPlanes<T> == 1 ? (KS <= 4 ? 4 : 2) : KS <= 6 ? 2 : 1) void attention_rows_kernel(AttentionArgs a)
{
    constexpr int NP = kPlanes<T>, PP = kPlanesP<T>, DT = (KS + 1) / 2;
    typedef RowsShape<NP, KS, NW> Sh;
    typedef typename Sh::Tiles Tiles;
    constexpr int KT = Sh::KT, NS = Sh::NS, PLANE = Tiles::PLANE / 2;
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

    const int i = mine.i, end = mine.end, head = hk * a.group + mine.g;
    Frag<NP> qf[KS];
    row_frags<T, KS, NP>(static_cast<const T*>(a.q) + b * a.qs.b + i * a.qs.t + head * a.qs.h, h, a.dim, a.vec, qf);
    Places<KS> places;
    places.init(lane);
    v16f acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = zero16();
    const float c = a.scale * kLog2e, slack = 8.0f / c;
    float m = -kInf, l = 0.0f;                     // of the raw scores; l over this lane's keys only
    for (int j0 = kbeg; j0 < kend; j0 += KT) {
        feed.ready();
        const __bf16* kt = reinterpret_cast<const __bf16*>(lds) + feed.at(0);
        const __bf16* vt = reinterpret_cast<const __bf16*>(lds) + feed.at(1);
        if (j0 + KT < kend) feed.begin(j0 + KT, kend);
#pragma unroll 1
        for (int j = j0; j < min(j0 + KT, kend); j += 32 * NS) {
            v16f s[NS];
#pragma unroll
            for (int u = 0; u < NS; ++u) {
                s[u] = zero16();
#pragma unroll
                for (int t = 0; t < KS; ++t) mma<NP>(s[u], rows_at<NP, KS>(kt, PLANE, places, u, t), qf[t]);
            }
            softmax_step<NS, DT>(s, acc, m, l, c, slack, j + 32 * NS > min(range.lo, kend), end - j, h);
#pragma unroll
            for (int u = 0; u < NS; ++u)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = s[u][8 * t + e];
                    const Frag<PP> pf = frag_of<PP>(v);
#pragma unroll
                    for (int d = 0; d < DT; ++d) mma<NP>(acc[d], cols_at<NP, KS>(vt, PLANE, places, 32 * u + 16 * t, d), pf);
                }
            kt += 32 * NS * Places<KS>::RS;
            vt += 32 * NS * Places<KS>::RS;
        }
    }
    l += __shfl_xor(l, 32);
    if (!mine.in) return;

    const size_t row_id = (size_t)at.bh * rows + mine.g * a.q_len + i;        // = (b heads + head) q_len + i
    float* const part = a.splits > 1 ? a.part + (size_t)at.split * a.batch * a.kv_heads * rows * a.dim : nullptr;
    float* const lse = a.splits > 1 ? a.part_lse + (size_t)at.split * a.batch * a.kv_heads * rows : a.lse;
    const float inv = inverse(l);
    if (h == 0 && lse) lse[row_id] = l == 0.0f ? -kInf : m * a.scale + logf(l);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int col = 32 * d + 8 * t + 4 * h;
            const float v[4] = {acc[d][4 * t] * inv, acc[d][4 * t + 1] * inv, acc[d][4 * t + 2] * inv, acc[d][4 * t + 3] * inv};
            if (part)
                store4(part + row_id * a.dim, col, a.dim, a.dim % 4 == 0, v);
            else
                store4(static_cast<T*>(a.out) + b * a.os.b + i * a.os.t + head * a.os.h, col, a.dim, a.vec_out, v);
        }
}

// Keys form.  Tiles pass through registers (fp32: split on the way): a workgroup reads its keys for so few rows that packing them
// ahead would cost more.  bf16: four wavefronts share 32 rows; fp32: two pairs of wavefronts with 32 rows each.
template <typename T, int KS>
struct KeysFormShape {
    static constexpr int NP = kPlanes<T>, RS = kRowStride<KS>, DT = (KS + 1) / 2;
    static constexpr int RG = NP == 3 ? 2 : 1, KG = 4 / RG, KT = 32 * KG;      // sets of rows, wavefronts that divide the keys
    static_assert(KS % 2 == 0, "results of 32 columns are read from a tile");
    static constexpr int TILE = NP * KT * RS, TILES = 2 * TILE * 2;
    static constexpr int JOIN = (2 * 4 * 32 + 32 * RG + 4 * DT * 32 * 33) * 4;
    static constexpr int LDS = TILES > JOIN ? TILES : JOIN;
};

template <typename T, int KS, bool VEC>
__global__ __launch_bounds__(256, sizeof(T) == 2 && VEC && KS <= 8 ? 2 : 1) void attention_keys_form_kernel(AttentionArgs a)
{
    typedef KeysFormShape<T, KS> Sh;
    constexpr int NP = Sh::NP, PP = kPlanesP<T>, RS = Sh::RS, DT = Sh::DT, KT = Sh::KT, RG = Sh::RG, KG = Sh::KG, RB = 32 * RG;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    __bf16* const kt = reinterpret_cast<__bf16*>(lds);
    __bf16* const vt = kt + Sh::TILE;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const int rg = wave / KG, kg = wave % KG;
    const Place at = place_of(a);
    const int b = at.bh / a.kv_heads, hk = at.bh - b * a.kv_heads;
    const int rows = a.group * a.q_len, n = keys_of(a, b);
    const int block = a.causal ? a.blocks - 1 - at.block : at.block;
    const int r_first = block * RB, r = r_first + 32 * rg + l32;
    const RowRange range = visible(a, n, r_first, min(r_first + RB, rows) - 1);
    const Part keys = part_of(range.hi, KT, at.split, a.splits);
    const int kbeg = (int)keys.beg, kend = (int)keys.end;
    const T* const kbase = static_cast<const T*>(a.k) + b * a.ks.b + hk * a.ks.h;
    const T* const vbase = static_cast<const T*>(a.v) + b * a.vs.b + hk * a.vs.h;
    Stage<T, KS, VEC, KT, 256> sk, sv;
    if (kbeg < kend) {
        sk.load(kbase, a.ks.t, kbeg, kend - 1, a.dim, tid);
        sv.load(vbase, a.vs.t, kbeg, kend - 1, a.dim, tid);
    }
    const int rc = min(r, rows - 1), g = rc / a.q_len, i = rc - g * a.q_len, head = hk * a.group + g;
    const int end = a.causal ? max(0, min(n, i + n - a.q_len + 1)) : n;
    Frag<NP> qf[KS];
    row_frags<T, KS, NP>(static_cast<const T*>(a.q) + b * a.qs.b + i * a.qs.t + head * a.qs.h, h, a.dim, VEC, qf);
    v16f acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = zero16();
    const float c = a.scale * kLog2e, slack = 8.0f / c;
    float m = -kInf, l = 0.0f;
    for (int j0 = kbeg; j0 < kend; j0 += KT) {
        __syncthreads();
        sk.store(kt, j0, kend, a.dim, tid);
        sv.store(vt, j0, kend, a.dim, tid);
        __syncthreads();
        if (j0 + KT < kend) {
            sk.load(kbase, a.ks.t, j0 + KT, kend - 1, a.dim, tid);
            sv.load(vbase, a.vs.t, j0 + KT, kend - 1, a.dim, tid);
        }
        v16f s[1];
        s[0] = zero16();
#pragma unroll
        for (int t = 0; t < KS; ++t) mma<NP>(s[0], row_frag<NP, RS, KT>(kt, 32 * kg + l32, 16 * t + 8 * h), qf[t]);
        softmax_step<1, DT>(s, acc, m, l, c, slack, j0 + KT > min(range.lo, kend), end - j0 - 32 * kg, h);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = s[0][8 * t + e];
            const Frag<PP> pf = frag_of<PP>(v);
#pragma unroll
            for (int d = 0; d < DT; ++d) mma<NP>(acc[d], col_frag<NP, RS, KT>(vt, 32 * kg + 16 * t, 32 * d, lane), pf);
        }
    }
    l += __shfl_xor(l, 32);

    float* const part = a.splits > 1 ? a.part + (size_t)at.split * a.batch * a.kv_heads * rows * a.dim : nullptr;
    float* const lse = a.splits > 1 ? a.part_lse + (size_t)at.split * a.batch * a.kv_heads * rows : a.lse;
    float* const rm = reinterpret_cast<float*>(lds);                          // [4][32] maxima, sums, [RG][32] 1 / sum, [4][32 DT][33]
    float* const rl = rm + 4 * 32;
    float* const ri = rl + 4 * 32;
    float* const ro = ri + 32 * RG;
    __syncthreads();
    if (h == 0) {
        rm[wave * 32 + l32] = m;
        rl[wave * 32 + l32] = l;
    }
    __syncthreads();
    float top = -kInf, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < KG; ++w) top = fmaxf(top, rm[(rg * KG + w) * 32 + l32]);
#pragma unroll
    for (int w = 0; w < KG; ++w) {
        const float mw = rm[(rg * KG + w) * 32 + l32], lw = rl[(rg * KG + w) * 32 + l32];
        sum += mw == -kInf ? lw : lw * __builtin_amdgcn_exp2f((mw - top) * c);                     // (0, or no number)
    }
    const float by = m == -kInf ? l : __builtin_amdgcn_exp2f((m - top) * c);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) ro[(wave * 32 * DT + 32 * d + 8 * (e / 4) + 4 * h + e % 4) * 33 + l32] = acc[d][e] * by;
    if (kg == 0 && h == 0) {
        ri[rg * 32 + l32] = inverse(sum);
        if (r < rows && lse) lse[(size_t)at.bh * rows + r] = sum == 0.0f ? -kInf : top * a.scale + logf(sum);
    }
    __syncthreads();
    for (int id = tid; id < RB * 8 * DT; id += 256) {
        const int row = id / (8 * DT), col = (id - row * 8 * DT) * 4, rr = r_first + row;
        if (rr >= rows || col >= a.dim) continue;
        const int gg = rr / a.q_len, ii = rr - gg * a.q_len;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = 0.0f;
#pragma unroll
            for (int w = 0; w < KG; ++w) v[e] += ro[((row / 32 * KG + w) * 32 * DT + col + e) * 33 + row % 32];
            v[e] *= ri[row];
        }
        if (part)
            store4(part + ((size_t)at.bh * rows + rr) * a.dim, col, a.dim, a.dim % 4 == 0, v);
        else
            store4(static_cast<T*>(a.out) + b * a.os.b + ii * a.os.t + (hk * a.group + gg) * a.os.h, col, a.dim, a.vec_out, v);
    }
}

// The parts of a row, each normalised with its own log-sum, joined: o = sum_s exp(lse_s - lse) o_s.  32 lanes per row.
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a)
{
    const size_t rows = (size_t)a.batch * a.kv_heads * a.group * a.q_len;
    const size_t at = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5), row = at < rows ? at : rows - 1;
    const int lane = threadIdx.x & 31;
    // four parts at a time, their log-sums and values loaded together, with a running maximum
    float base = -kInf, sum = 0.0f, v[5] = {0, 0, 0, 0, 0};
    for (int s0 = 0; s0 < a.splits; s0 += 4) {
        float ls[4], p[4][5];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const size_t s = min(s0 + u, a.splits - 1);
            ls[u] = a.part_lse[s * rows + row];
#pragma unroll
            for (int d = 0; d < 5; ++d) p[u][d] = a.part[(s * rows + row) * a.dim + min(lane + 32 * d, a.dim - 1)];
        }
        float top = base;
#pragma unroll
        for (int u = 0; u < 4; ++u) top = fmaxf(top, ls[u]);
        const float to = top == -kInf ? 0.0f : top, by = __builtin_amdgcn_exp2f((base - to) * kLog2e);
        sum *= by;
#pragma unroll
        for (int d = 0; d < 5; ++d) v[d] *= by;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float w = s0 + u < a.splits ? __builtin_amdgcn_exp2f((ls[u] - to) * kLog2e) : 0.0f;
            sum += w;
#pragma unroll
            for (int d = 0; d < 5; ++d) v[d] += w == 0.0f ? 0.0f : w * p[u][d];
        }
        base = top;
    }
    if (at >= rows) return;
    if (lane == 0 && a.lse) a.lse[row] = sum == 0.0f ? -kInf : base + logf(sum);
    const size_t bh = row / a.q_len;
    const int i = (int)(row - bh * a.q_len), heads = a.kv_heads * a.group;
    const int64_t b = bh / heads, head = bh - (size_t)b * heads;
    T* const out = static_cast<T*>(a.out) + b * a.os.b + i * a.os.t + head * a.os.h;
    const float inv = inverse(sum);
#pragma unroll
    for (int d = 0; d < 5; ++d)
        if (lane + 32 * d < a.dim) out[lane + 32 * d] = (T)(v[d] * inv);
}

template <typename T, int KS, int NW>
int launch_rows(const AttentionArgs& a, hipStream_t s)
{
    constexpr int lds = RowsShape<kPlanes<T>, KS, NW>::Tiles::LDS;
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&attention_rows_kernel<T, KS, NW>), lds, done)) return FPQ_ERR_LAUNCH;
    const int64_t grid = (int64_t)a.batch * a.kv_heads * a.blocks * a.splits;
    attention_rows_kernel<T, KS, NW><<<dim3((unsigned)grid), dim3(64 * NW), lds, s>>>(a);
    return FPQ_OK;
}
template <typename T, int KS>
int launch_rows(const AttentionArgs& a, int waves, hipStream_t s)
{
    return waves == 4 ? launch_rows<T, KS, 4>(a, s) : launch_rows<T, KS, 2>(a, s);
}

template <typename T, int KS, bool VEC>
int launch_keys_form(const AttentionArgs& a, hipStream_t s)
{
    constexpr int lds = KeysFormShape<T, KS>::LDS;
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&attention_keys_form_kernel<T, KS, VEC>), lds, done)) return FPQ_ERR_LAUNCH;
    const int64_t grid = (int64_t)a.batch * a.kv_heads * a.blocks * a.splits;
    attention_keys_form_kernel<T, KS, VEC><<<dim3((unsigned)grid), dim3(256), lds, s>>>(a);
    return FPQ_OK;
}

template <typename T>
int launch_forward(const AttentionArgs& a, bool by_keys, int waves, hipStream_t s)
{
    const int ks = (a.dim + 15) / 16;
    int st;
    if (!by_keys)
        st = ks <= 3 ? launch_rows<T, 3>(a, waves, s) : ks == 4 ? launch_rows<T, 4>(a, waves, s) : ks == 5 ? launch_rows<T, 5>(a, waves, s)
           : ks == 6 ? launch_rows<T, 6>(a, waves, s) : ks <= 8 ? launch_rows<T, 8>(a, waves, s) : launch_rows<T, 10>(a, waves, s);
    else if (a.vec)
        st = ks <= 4 ? launch_keys_form<T, 4, true>(a, s) : ks <= 6 ? launch_keys_form<T, 6, true>(a, s)
           : ks <= 8 ? launch_keys_form<T, 8, true>(a, s) : launch_keys_form<T, 10, true>(a, s);
    else
        st = ks <= 4 ? launch_keys_form<T, 4, false>(a, s) : ks <= 8 ? launch_keys_form<T, 8, false>(a, s) : launch_keys_form<T, 10, false>(a, s);
    if (st != FPQ_OK) return st;
    if (a.splits > 1) {
        const size_t rows = (size_t)a.batch * a.kv_heads * a.group * a.q_len;
        attention_join_kernel<T><<<dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, s>>>(a);
    }
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

}  // namespace fpq
