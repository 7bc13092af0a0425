// Products of few rows (a token of each request) with weights that are read once: layers on 4-bit blocks, gated projections.
//
// Bound by the weights' bytes.  A workgroup makes 16 NT results of every row (gated: 16 NT values and their gates); its wavefronts take turns
// along k, 128 bytes of each weight row at a time (64 of 4-bit blocks), and are summed through LDS at the end.  A lane's weights are 16
// neighbouring bytes of one row: for 16 x 16 x 32 steps of the matrix instruction any order of k will do if both operands agree, so the
// rows x, which the caches serve, are read in the order in which the weights lie.  Weights are the A operand: a lane then holds four
// neighbouring results of a row.  4-bit codes become bf16 with their scale in the conversion instruction, two at a time; fp32 operands are
// split into three planes in registers.  One row of 4096 -> 2 x 10240 in bf16: 33 us (5.1 TB/s); 16 rows of 5120 -> 5120 on 4-bit blocks
// 11.3 us in bf16, 17.0 in fp32, where the splitting of x in every workgroup is what takes the time.
#pragma once
#include "matmul.h"

namespace fpq {

constexpr int kFewRows = 64;            // rows that this form takes

struct RowsArgs {
    const void* x;
    int64_t ld_x;
    int M, N, K;
    const void* w;
    int64_t ld_w;                       // elements (4-bit blocks: bytes)
    const uint8_t* scales;              // of 4-bit blocks, ld_s a row
    int64_t ld_s;
    const float* bias;
    void* out;                          // not gated
    int64_t ld_out;
    int f32;                            // type of x and the results
    Gate gate;
};

// Blocks4: 4-bit blocks, float or __bf16
struct Blocks4 {};

template <int NA, int NB>
__device__ __forceinline__ void mma16(v4f& c, const Frag<NA>& a, const Frag<NB>& b)
{
    auto step = [&](int p, int q) { c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[p], b.p[q], c, 0, 0, 0); };
    if constexpr (NA == 3 && NB == 3) {             // small products first
        step(2, 0);
        step(0, 2);
        step(1, 1);
        step(1, 0);
        step(0, 1);
    }
    if constexpr (NA == 1 && NB == 3) {
        step(0, 2);
        step(0, 1);
    }
    step(0, 0);
}

// Eight values of a row of x from k on as an operand; zeros for rows and columns that are not there.
template <typename T>
struct RowPiece {
    piece16 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* row, int k, int K, bool in)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = piece16{0, 0, 0, 0};
        if (!in || k >= K) return;
        if (k + 8 <= K) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = reinterpret_cast<const piece16*>(row + k)[i];
        } else {
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = k + i < K ? row[k + i] : (T)0.0f;
            __builtin_memcpy(v, e, sizeof e);
        }
    }
    __device__ __forceinline__ Frag<kPlanes<T>> frag() const
    {
        if constexpr (sizeof(T) == 2) {
            Frag<1> f;
            f.p[0] = __builtin_bit_cast(v8bf, v[0]);
            return f;
        } else {
            float e[8];
            __builtin_memcpy(e, v, sizeof e);
            return frag_of<3>(e);
        }
    }
};

// A lane's weights of a row for one turn: 128 bytes of the row, 16 (fp32: 32) of them in each of its lanes' loads.  STEPS: of 32 k in a turn;
// k(s): the lane's first k of step s, within the turn.
template <typename W>
struct Turn {
    static constexpr int STEPS = sizeof(W) == 4 ? 1 : 2, K = 32 * STEPS;
    RowPiece<W> p[STEPS];
    static __device__ __forceinline__ int k(int s, int q) { return 32 * s + 8 * q; }
    __device__ __forceinline__ void load(const RowsArgs& a, int64_t row, int k0, int q)
    {
        const W* const w = static_cast<const W*>(a.w) + row * a.ld_w;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) p[s].load(w, k0 + k(s, q), a.K, true);
    }
    __device__ __forceinline__ void settle() {}
    __device__ __forceinline__ Frag<kPlanes<W>> frag(int s) const { return p[s].frag(); }
};
// w[i] of the lanes 16 q .. 16 q + 15 becomes w[q] of the lanes 16 i ..
__device__ __forceinline__ void exchange4(uint32_t (&w)[4])
{
    typedef unsigned v2u __attribute__((ext_vector_type(2)));
    auto swap32 = [](uint32_t& a, uint32_t& b) {
        const v2u r = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane32_swap(a, b, false, false));
        a = r.x;
        b = r.y;
    };
    auto swap16 = [](uint32_t& a, uint32_t& b) {
        const v2u r = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane16_swap(a, b, false, false));
        a = r.x;
        b = r.y;
    };
    swap32(w[0], w[2]);
    swap32(w[1], w[3]);
    swap16(w[0], w[1]);
    swap16(w[2], w[3]);
}

// A lane loads a whole block; exchanged among the four lanes of a row, they have eight codes each of every block: then the lanes' pieces of x
// are neighbours, 64 or 128 bytes of a row in one load instead of four places.
template <>
struct Turn<Blocks4> {
    static constexpr int STEPS = 4, K = 128;
    uint32_t c[4], s[4];
    static __device__ __forceinline__ int k(int s, int q) { return 32 * s + 8 * q; }
    __device__ __forceinline__ void load(const RowsArgs& a, int64_t row, int k0, int q)
    {
        const int k = k0 + 32 * q;
        uint4 v = make_uint4(0, 0, 0, 0);
        s[0] = 127;
        if (k < a.K) {
            v = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.w) + row * a.ld_w + k / 2);
            s[0] = a.scales[row * a.ld_s + k / 32];
        }
        c[0] = v.x, c[1] = v.y, c[2] = v.z, c[3] = v.w;
    }
    __device__ __forceinline__ void settle()
    {
        exchange4(c);
        s[1] = s[2] = s[3] = s[0];
        exchange4(s);
    }
    __device__ __forceinline__ Frag<1> frag(int step) const
    {
        const uint32_t x = c[step];
        const float f = scale_of(s[step]);
        uint32_t o[4];
        o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, f, 0));
        o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, f, 1));
        o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, f, 2));
        o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, f, 3));
        Frag<1> r;
        r.p[0] = __builtin_bit_cast(v8bf, make_uint4(o[0], o[1], o[2], o[3]));
        return r;
    }
};

// T: of x and the results; MT: 16-row tiles of x; WV: wavefronts
template <typename T, typename W, int MT, int NT, int WV, bool GATED>
__global__ __launch_bounds__(64 * WV) void rows_kernel(RowsArgs a)
{
    constexpr int G = GATED ? 2 : 1, TILES = NT * G;
    using U = Turn<W>;
    __shared__ float room[WV * TILES * MT * 256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16 * NT;
    int64_t row[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) row[t] = min(n0 + 16 * (t / G) + r, a.N - 1) + (int64_t)(t % G) * a.N;
    const T* x[MT];
#pragma unroll
    for (int u = 0; u < MT; ++u) x[u] = static_cast<const T*>(a.x) + (int64_t)min(16 * u + r, a.M - 1) * a.ld_x;
    v4f acc[MT][TILES];
#pragma unroll
    for (int u = 0; u < MT; ++u)
#pragma unroll
        for (int t = 0; t < TILES; ++t) acc[u][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    // The rows of a turn, ahead of the next turn's weights: loads come back in order, and a wait for the rows must not be one for those.
    RowPiece<T> p[MT][U::STEPS];
    U now[TILES], next[TILES];
    auto load_x = [&](int k0) {
#pragma unroll
        for (int s = 0; s < U::STEPS; ++s)
#pragma unroll
            for (int u = 0; u < MT; ++u) p[u][s].load(x[u], k0 + U::k(s, q), a.K, 16 * u + r < a.M);
    };
    auto load_w = [&](int k0) {
#pragma unroll
        for (int t = 0; t < TILES; ++t) next[t].load(a, row[t], k0, q);
    };
    int k0 = wave * U::K;
    if (k0 < a.K) {
        load_x(k0);
        load_w(k0);
    }
    for (; k0 < a.K; k0 += WV * U::K) {
        const bool more = k0 + WV * U::K < a.K;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            now[t] = next[t];
            now[t].settle();
        }
        if constexpr (MT == 1) {
            RowPiece<T> c[U::STEPS];
#pragma unroll
            for (int s = 0; s < U::STEPS; ++s) c[s] = p[0][s];
            if (more) {
                load_x(k0 + WV * U::K);
                load_w(k0 + WV * U::K);
            }
#pragma unroll
            for (int s = 0; s < U::STEPS; ++s) {
                const Frag<kPlanes<T>> f = c[s].frag();
#pragma unroll
                for (int t = 0; t < TILES; ++t) mma16(acc[0][t], now[t].frag(s), f);
            }
        } else {
            if (more) load_w(k0 + WV * U::K);
#pragma unroll
            for (int s = 0; s < U::STEPS; ++s) {
                Frag<kPlanes<T>> f[MT];
#pragma unroll
                for (int u = 0; u < MT; ++u) f[u] = p[u][s].frag();
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    const auto w = now[t].frag(s);
#pragma unroll
                    for (int u = 0; u < MT; ++u) mma16(acc[u][t], w, f[u]);
                }
            }
            if (more) load_x(k0 + WV * U::K);
        }
    }
    // [wave][tile][u][m][n]
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int u = 0; u < MT; ++u)
            *reinterpret_cast<v4f*>(&room[((wave * TILES + t) * MT + u) * 256 + r * 16 + 4 * q]) = acc[u][t];
    __syncthreads();
    auto sum = [&](int t, int u, int at) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WV; ++w) v += room[((w * TILES + t) * MT + u) * 256 + at];
        return v;
    };
    constexpr int ALL = NT * MT * 256;
    for (int id = threadIdx.x; id < ALL; id += 64 * WV) {
        // (neighbours in n are neighbours in the workgroup)
        const int n = id % (16 * NT), m = id / (16 * NT), t = n / 16, at = (m & 15) * 16 + (n & 15), col = n0 + n;
        const bool in = m < a.M && col < a.N;
        if constexpr (GATED) {
            float va = sum(2 * t, m / 16, at), vg = sum(2 * t + 1, m / 16, at);
            if (a.bias && in) {
                va += a.bias[col];
                vg += a.bias[a.N + col];
            }
            if constexpr (NT == 2)
                if (a.gate.pre_scales) {                // a block is 32 lanes'
                    const int np = (a.N + 31) & ~31;
                    uint32_t ta = in ? __float_as_uint(va) & 0x7fffffffu : 0u, tg = in ? __float_as_uint(vg) & 0x7fffffffu : 0u;
#pragma unroll
                    for (int off = 1; off < 32; off <<= 1) {
                        ta = max(ta, (uint32_t)__shfl_xor((int)ta, off, 64));
                        tg = max(tg, (uint32_t)__shfl_xor((int)tg, off, 64));
                    }
                    if (m < a.M) {
                        const uint32_t ea = block_scale8(ta), eg = block_scale8(tg);
                        uint8_t* const c = static_cast<uint8_t*>(a.gate.pre) + m * (2 * (int64_t)np) + col;
                        c[0] = (uint8_t)codes8(in ? va * inverse_scale(ea) : 0.0f, 0.0f, 0.0f, 0.0f);
                        c[np] = (uint8_t)codes8(in ? vg * inverse_scale(eg) : 0.0f, 0.0f, 0.0f, 0.0f);
                        if (n == 0) {
                            uint8_t* const s = a.gate.pre_scales + m * (2 * (np / 32)) + n0 / 32;
                            s[0] = (uint8_t)ea;
                            s[np / 32] = (uint8_t)eg;
                        }
                    }
                }
            if (!in) continue;
            static_cast<T*>(a.gate.h)[m * a.gate.ld_h + col] = (T)(va * gate_of<false>(a.gate.act, vg, nullptr));
            if (a.gate.pre && !a.gate.pre_scales) {
                T* const pre = static_cast<T*>(a.gate.pre) + m * a.gate.ld_pre;
                pre[col] = (T)va;
                pre[a.N + col] = (T)vg;
            }
        } else if (in) {
            static_cast<T*>(a.out)[m * a.ld_out + col] = (T)(sum(t, m / 16, at) + (a.bias ? a.bias[col] : 0.0f));
        }
    }
}

template <typename T, typename W, int MT, int NT, int WV, bool GATED>
int launch_rows_as(const RowsArgs& a, hipStream_t s)
{
    rows_kernel<T, W, MT, NT, WV, GATED><<<dim3((unsigned)((a.N + 16 * NT - 1) / (16 * NT))), dim3(64 * WV), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

// The form of one to four rows keeps x in LDS, up to 64 KB.
static inline int64_t token_blocks_lds(int64_t M, int64_t K, int f32) { return M * ((K + 2047) / 2048 * 2048) * (f32 ? 4 : 2); }
int launch_token_blocks(const RowsArgs& a, hipStream_t s);
int launch_rows_blocks(const RowsArgs& a, hipStream_t s);
int launch_rows_gated(const RowsArgs& a, hipStream_t s);

}  // namespace fpq
