// Attention, forward: o = softmax(scale q k^T) v in one pass over the keys, with the running maximum m (a lower bound
// of it, within 2^8 after the exponential) and sum l of a row's exponentials; o and l are rescaled when m grows.  m, l and o are held in 32 bits; the probabilities are rounded to the
// operand's planes (8 bits for bf16 results, 24 for fp32) where they enter the second product.
//
// A wavefront has 32 rows of queries in registers and takes S^T = K Q^T per 32 keys, so that a lane holds 16 scores of one row and
// its maximum and sum need one exchange with the lane 32 on; P^T is then the operand of O^T = V^T P^T as it lies.
//   rows form: four wavefronts with 32 rows each share tiles of keys and values in LDS.
//   keys form (KEYS): the wavefronts share 32 rows and take 32 keys each of a tile; their results are joined at the end.  For few
//   rows: single tokens, small batches.
#pragma once
#include "attention.h"

namespace fpq {

template <typename T, int KS, bool VEC, bool KEYS>
struct ForwardShape {
    static constexpr int NP = kPlanes<T>, RS = kRowStride<KS>, DT = (KS + 1) / 2;
    static constexpr int NW = KEYS && NP == 3 ? 2 : 4;
    static constexpr int KT = KEYS ? 32 * NW : NP == 3 || KS > 8 ? 32 : 64;
    typedef Feed<T, KS, VEC, KT, NW, sizeof(T) == 2 && VEC && !KEYS> Tiles;
    static constexpr int TILES = Tiles::LDS;
    static constexpr int JOIN = KEYS ? (2 * NW * 32 + 32 + NW * DT * 32 * 33) * 4 : 0;
    static constexpr int LDS = TILES > JOIN ? TILES : JOIN;
    static constexpr bool AHEAD = !(KEYS && NP == 3);     // a tile waits in registers while the one before is multiplied
};

template <typename T, int KS, bool VEC, bool KEYS>
__global__ __launch_bounds__((64 * ForwardShape<T, KS, VEC, KEYS>::NW), sizeof(T) == 2 && VEC && KS <= 8 ? 2 : 1) void attention_kernel(AttentionArgs a)
{
    typedef ForwardShape<T, KS, VEC, KEYS> Sh;
    constexpr int NP = Sh::NP, RS = Sh::RS, DT = Sh::DT, NW = Sh::NW, KT = Sh::KT, NT = 64 * NW, NS = KEYS ? 1 : KT / 32;
    constexpr int RB = KEYS ? 32 : 32 * NW;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const Place at = place_of(a);
    const int b = at.bh / a.kv_heads, hk = at.bh - b * a.kv_heads;
    const int rows = a.group * a.q_len, n = keys_of(a, b);
    const int block = a.causal ? a.blocks - 1 - at.block : at.block;          // the longest rows first
    const int r_first = block * RB, r = r_first + (KEYS ? 0 : 32 * wave) + l32;
    const RowRange range = visible(a, n, r_first, min(r_first + RB, rows) - 1);
    const int kbeg = min((int64_t)at.split * a.per_split, (int64_t)range.hi), kend = min((int64_t)kbeg + a.per_split, (int64_t)range.hi);

    const int rc = min(r, rows - 1), g = rc / a.q_len, i = rc - g * a.q_len, head = hk * a.group + g;
    const int end = a.causal ? max(0, min(n, i + n - a.q_len + 1)) : n;       // the row sees keys below it
    Frag<NP> qf[KS];
    {
        const T* row = static_cast<const T*>(a.q) + b * a.qs.b + i * a.qs.t + head * a.qs.h;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            float v[8];
            row8<T, VEC>(row, 16 * s + 8 * h, a.dim, v);
            qf[s] = frag_of<NP>(v);
        }
    }
    const T* const kbase = static_cast<const T*>(a.k) + b * a.ks.b + hk * a.ks.h;
    const T* const vbase = static_cast<const T*>(a.v) + b * a.vs.b + hk * a.vs.h;

    v16f acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = zero16();
    const float c = a.scale * kLog2e, slack = 8.0f / c;
    float m = -kInf, l = 0.0f;                     // of the raw scores; l over this lane's keys only
    typename Sh::Tiles feed;
    feed.init(lds, kbase, a.ks.t, vbase, a.vs.t, a.dim);
    if (Sh::AHEAD && kbeg < kend) feed.begin(kbeg, kend);
    for (int j0 = kbeg; j0 < kend; j0 += KT) {
        if (!Sh::AHEAD) {
            __syncthreads();
            feed.begin(j0, kend);
        }
        feed.ready(j0, kend);
        const __bf16* const kt = reinterpret_cast<const __bf16*>(lds) + feed.at(0);
        const __bf16* const vt = reinterpret_cast<const __bf16*>(lds) + feed.at(1);
        if (Sh::AHEAD && j0 + KT < kend) feed.begin(j0 + KT, kend);
        const int sub0 = KEYS ? 32 * wave : 0;
        v16f s[NS];
#pragma unroll
        for (int u = 0; u < NS; ++u) {
            s[u] = zero16();
#pragma unroll
            for (int t = 0; t < KS; ++t) mma<NP>(s[u], row_frag<NP, RS, KT>(kt, sub0 + 32 * u + l32, 16 * t + 8 * h), qf[t]);
        }
        if (j0 + KT > min(range.lo, kend)) {       // some key is hidden from some row
            const int left = end - j0 - sub0;
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
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[u][e] = __builtin_amdgcn_exp2f(fmaf(s[u][e], c, -mc));
                l += s[u][e];
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = s[u][8 * t + e];
                const Frag<NP> pf = frag_of<NP>(v);
#pragma unroll
                for (int d = 0; d < DT; ++d) mma<NP>(acc[d], col_frag<NP, RS, KT>(vt, sub0 + 32 * u + 16 * t, 32 * d, lane), pf);
            }
        }
    }
    l += __shfl_xor(l, 32);

    const size_t row_id = ((size_t)at.bh * a.group * a.q_len) + rc;           // = (b heads + head) q_len + i
    float* const part = a.splits > 1 ? a.part + (size_t)at.split * a.batch * a.kv_heads * rows * a.dim : nullptr;
    float* const lse = a.splits > 1 ? a.part_lse + (size_t)at.split * a.batch * a.kv_heads * rows : a.lse;
    if constexpr (!KEYS) {
        if (r >= rows) return;
        const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;         // no key: zeros; a sum that is no number stays one
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
    } else {
        float* const rm = reinterpret_cast<float*>(lds);                      // [NW][32] maxima, sums, [32] 1 / sum, [NW][32 DT][33]
        float* const rl = rm + NW * 32;
        float* const ri = rl + NW * 32;
        float* const ro = ri + 32;
        __syncthreads();
        if (h == 0) {
            rm[wave * 32 + l32] = m;
            rl[wave * 32 + l32] = l;
        }
        __syncthreads();
        float top = rm[l32], sum = 0.0f;
#pragma unroll
        for (int w = 1; w < NW; ++w) top = fmaxf(top, rm[w * 32 + l32]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float mw = rm[w * 32 + l32];
            sum += mw == -kInf ? rl[w * 32 + l32] : rl[w * 32 + l32] * __builtin_amdgcn_exp2f((mw - top) * c);    // (0, or no number)
        }
        const float by = m == -kInf ? l : __builtin_amdgcn_exp2f((m - top) * c);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) ro[(wave * 32 * DT + 32 * d + 8 * (e / 4) + 4 * h + e % 4) * 33 + l32] = acc[d][e] * by;
        if (wave == 0 && h == 0) {
            ri[l32] = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
            if (r < rows && lse) lse[row_id] = sum == 0.0f ? -kInf : top * a.scale + logf(sum);
        }
        __syncthreads();
        for (int id = tid; id < 32 * 8 * DT; id += NT) {
            const int row = id / (8 * DT), col = (id - row * 8 * DT) * 4, rr = r_first + row;
            if (rr >= rows || col >= a.dim) continue;
            const int gg = rr / a.q_len, ii = rr - gg * a.q_len;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = 0.0f;
#pragma unroll
                for (int w = 0; w < NW; ++w) v[e] += ro[(w * 32 * DT + col + e) * 33 + row];
                v[e] *= ri[row];
            }
            if (part)
                store4(part + ((size_t)at.bh * rows + rr) * a.dim, col, a.dim, a.dim % 4 == 0, v);
            else
                store4(static_cast<T*>(a.out) + b * a.os.b + ii * a.os.t + (hk * a.group + gg) * a.os.h, col, a.dim, a.vec_out, v);
        }
    }
}

// The parts of a row, each normalised with its own log-sum, joined: o = sum_s exp(lse_s - lse) o_s.  One wavefront per row.
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a)
{
    const size_t rows = (size_t)a.batch * a.kv_heads * a.group * a.q_len, row = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= rows) return;
    float top = -kInf, sum = 0.0f;
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, a.part_lse[s * rows + row]);
    const float base = top == -kInf ? 0.0f : top;
    for (int s = 0; s < a.splits; ++s) sum += __builtin_amdgcn_exp2f((a.part_lse[s * rows + row] - base) * kLog2e);
    const float lse = sum == 0.0f ? -kInf : base + logf(sum);
    if (lane == 0 && a.lse) a.lse[row] = lse;
    const size_t bh = row / a.q_len;
    const int i = (int)(row - bh * a.q_len), heads = a.kv_heads * a.group;
    const int64_t b = bh / heads, head = bh - (size_t)b * heads;
    T* const out = static_cast<T*>(a.out) + b * a.os.b + i * a.os.t + head * a.os.h;
    const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
    for (int d = lane; d < a.dim; d += 64) {
        float v = 0.0f;
        for (int s = 0; s < a.splits; ++s) {
            const float w = __builtin_amdgcn_exp2f((a.part_lse[s * rows + row] - base) * kLog2e);
            v += w * a.part[(s * rows + row) * a.dim + d];
        }
        out[d] = (T)(v * inv);
    }
}

template <typename T, int KS, bool VEC, bool KEYS>
int launch_forward(const AttentionArgs& a, hipStream_t s)
{
    typedef ForwardShape<T, KS, VEC, KEYS> Sh;
    static std::atomic<uint64_t> done{0};
    const void* kernel = reinterpret_cast<const void*>(&attention_kernel<T, KS, VEC, KEYS>);
    if (!allow_dynamic_lds(kernel, Sh::LDS, done)) return FPQ_ERR_LAUNCH;
    const int64_t grid = (int64_t)a.batch * a.kv_heads * a.blocks * a.splits;
    attention_kernel<T, KS, VEC, KEYS><<<dim3((unsigned)grid), dim3(64 * Sh::NW), Sh::LDS, s>>>(a);
    return FPQ_OK;
}

template <typename T, int KS, bool VEC>
int launch_forward(const AttentionArgs& a, bool by_keys, hipStream_t s)
{
    return by_keys ? launch_forward<T, KS, VEC, true>(a, s) : launch_forward<T, KS, VEC, false>(a, s);
}

template <typename T>
int launch_forward(const AttentionArgs& a, bool vec, bool by_keys, hipStream_t s)
{
    const int ks = (a.dim + 15) / 16;
    int st;
    if (vec)
        st = ks <= 3 ? launch_forward<T, 3, true>(a, by_keys, s) : ks == 4 ? launch_forward<T, 4, true>(a, by_keys, s)
           : ks == 5 ? launch_forward<T, 5, true>(a, by_keys, s) : ks == 6 ? launch_forward<T, 6, true>(a, by_keys, s)
           : ks <= 8 ? launch_forward<T, 8, true>(a, by_keys, s) : launch_forward<T, 10, true>(a, by_keys, s);
    else
        st = ks <= 4 ? launch_forward<T, 4, false>(a, by_keys, s) : ks <= 8 ? launch_forward<T, 8, false>(a, by_keys, s)
           : launch_forward<T, 10, false>(a, by_keys, s);
    if (st != FPQ_OK) return st;
    if (a.splits > 1) {
        const size_t rows = (size_t)a.batch * a.kv_heads * a.group * a.q_len;
        attention_join_kernel<T><<<dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s>>>(a);
    }
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

}  // namespace fpq
