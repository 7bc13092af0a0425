// Matrix products of the operators around the projections (gated projections, gradients of linear layers, layers on 4-bit blocks):
//
//   out[m, n] = sum_k A(m, k) B(n, k)
//
// Operands are one to three planes of bf16 (fp32 values x = h + m + l, as in attention.h, or h + m; of nine products the six largest are taken,
// beside an operand of one plane all).  Each operand lies either with the contraction along its rows (ROW: p[m ld + k]) or along
// its columns (COL: p[k ld + m]), so that x W^T, g W and g^T x are one kernel without a transposed copy.
//
// A workgroup makes a tile of BM x BN results in steps of 32 or 64 along k; tiles go from memory to LDS directly into a ring of stages, of which
// all but one are on their way.  ROW tiles are read as 16 bytes of a row, COL tiles by the transposing read, which gives a lane four k of its
// column; both in the same order of k, eight neighbours per lane.  Places of 16 bytes are exchanged within a row so that neither read meets a
// bank twice: of a ROW tile 16 rows of one piece lie in the 16 groups of four banks, of a COL tile four rows of 64 bytes each.
// B is the A operand of the instruction: a lane then holds four neighbouring columns n of one row m of the result.  Operands are read one
// product of 16 k ahead, across the barrier too, so that the matrix unit has work while the workgroup meets.
//
// Large products are bound by the matrix unit and the power it may draw (a loop of nothing but its instructions reaches 1.85 PFLOP/s): 4096 x 4096 x 4096 in bf16
// with either operand by columns 108 us, 1.27 PFLOP/s; the gated forward of 8192 x 1280 -> 2 x 5120 with blocks kept 222 us on its own, 0.97, and
// 241 to 261 among a training step's kernels, of which some 40 are the ends of its five rounds; in fp32 2048 x 1280 -> 2 x 5120 300 us, 1.07 in bf16 products.  Smaller ones wait for their first loads and are
// quantized by tiles (the choice is made in matmul.hip).
#pragma once
#include "attention.h"
#include "gemm_common.h"

namespace fpq {

// Sixteen bytes at the address of any element: the hardware takes them in one access, which costs more only where a line ends within.
typedef uint32_t piece16 __attribute__((ext_vector_type(4), aligned(2), may_alias));

struct Operand {
    const __bf16* p;
    int64_t ld, plane;          // in elements
};

// Rows of `per` units each, for kernels whose threads take a unit: the row of unit `id`.
struct RowOf {
    int64_t per;
    Divisor by;
    int fits;                   // all numbers of units fit 31 bits
};
static inline RowOf row_of(int64_t rows, int64_t per) { return RowOf{per, divisor(per < ((int64_t)1 << 31) ? per : 1), rows * per < (int64_t)1 << 31}; }
__device__ __forceinline__ int64_t row_at(const RowOf& r, int64_t id) { return r.fits ? (int64_t)divide((int)id, r.by) : id / r.per; }

// What the results of a tile become.  kSums: stored, and the sums of A over k beside them (a bias's gradient beside the weights').
enum MatmulEnd : int { kStore = 0, kGated = 1, kSums = 2 };

struct Gate {
    int act;                    // fpq_gate
    void* h;
    int64_t ld_h;
    void* pre;                  // [M, 2 N] of the type, or codes [M, 2 Np], or null
    int64_t ld_pre;             // (type only)
    uint8_t* pre_scales;        // codes' scales or null
};

struct MatmulArgs {
    Operand a, b;
    int M, N, K;                // gated: N outputs, B has 2 N rows, values first
    int steps;                  // along K
    uint32_t order_a, order_b;  // planes of each pass, four bits each, the first pass lowest
    int passes, total;          // passes x steps
    int slices;                 // of `total`
    int tiles_m, tiles_n;
    void* out;                  // kStore; slices > 1: fp32 [slice][M][N] (gated: [slice][M][2 N]) whatever the end
    int64_t ld_out;
    int out_f32;
    const float* bias;          // [N] or [2 N] or null (slices == 1)
    float* sums;                // kSums: [slice][M]
    Gate gate;
};

// Block scales: a power of two as its biased exponent; 255 stands for NaN.
__device__ __forceinline__ float scale_of(uint32_t e) { return e ? __uint_as_float(e == 255 ? 0x7fc00000u : e << 23) : 0x1p-127f; }
// The least power of two with which a largest magnitude (its bits) is at most (1 + top / 2^23) 2^max_exp; 1 for zero.
__device__ __forceinline__ uint32_t block_scale(uint32_t bits, int max_exp, uint32_t top)
{
    if (bits >= 0x7f800000u) return 255u;
    if (bits == 0) return 127u;
    const int e = (int)(bits >> 23) - max_exp + ((bits & 0x7fffffu) > top ? 1 : 0);
    return (uint32_t)max(e, 1);
}
__device__ __forceinline__ uint32_t block_scale8(uint32_t bits) { return block_scale(bits, 8, 0x600000u); }      // 448 = 1.75 2^8
__device__ __forceinline__ uint32_t block_scale4(uint32_t bits) { return block_scale(bits, 2, 0x400000u); }      // 6 = 1.5 2^2
// 1 / scale, exact
__device__ __forceinline__ float inverse_scale(uint32_t e) { return __uint_as_float(e == 255 ? 0x7fc00000u : (254u - e) << 23); }

__device__ __forceinline__ uint32_t codes8(float a, float b, float c, float d)
{
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// act(g) and its derivative.  SiLU: g z and z (1 + g (1 - z)) with z = 1 / (1 + e^-g), off by at most (4 + |g|) 2^-23 of z (the exponent's
// product is rounded, exponential and reciprocal are the hardware's; below 2^-126, g of -87.3, it may be zero).  GELU: g Phi(g) and Phi(g) + g phi(g), Phi by the formula of
// act_gelu, off by at most 4e-7.
template <bool SLOPE>
__device__ __forceinline__ float gate_of(int act, float g, float* slope)
{
    if (act == FPQ_GATE_SILU) {
        const float z = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * g));
        if constexpr (SLOPE) *slope = z * fmaf(g, 1.0f - z, 1.0f);
        return g * z;
    }
    if constexpr (!SLOPE) return act_gelu(g);
    const float m = fminf(fabsf(g), 1e18f), s = m * 0.84932180028801907f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.23164188f, m, 1.0f)), e = __builtin_amdgcn_exp2f(-s * s);
    float p = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
    p = fmaf(t, p, 0.5f * 1.421413741f);
    p = fmaf(t, p, 0.5f * -0.284496736f);
    p = fmaf(t, p, 0.5f * 0.254829592f);
    const float half = t * p * e, z = g > 0.0f ? 1.0f - half : half;
    if constexpr (SLOPE) *slope = fmaf(g * 0.39894228040143268f, e, z);
    return g * z;
}

// ROW tiles of 64 or 128 bytes a row: place c ^ row_swap holds piece c.
template <int KS>
__device__ __forceinline__ int row_swap(int row)
{
    return KS == 32 ? (row >> 2) & 3 : (row >> 1) & 7;
}

// COL tiles: four neighbouring rows' 64 bytes lie in different banks, of which rows of 64 columns fill half.
template <int R>
__device__ __forceinline__ int col_swap(int row)
{
    return R == 64 ? (row & 2) << 1 : (row & 3) << 2;
}

// One operand's tile of R rows (ROW) or columns (COL) and KS k: this thread's loads of it.  Every wavefront makes the same number: where
// they do not divide, some load a piece that another one loads too.
template <bool COL, int R, int KS, int NW>
struct TileFeed {
    static constexpr int CS = COL ? R / 8 : KS / 8, N = R * KS / 512, PT = (N + NW - 1) / NW;
    static_assert(R % 32 == 0 && (!COL || R == 64 || R % 128 == 0), "whole wavefronts of loads; rows of COL tiles span all banks, or half");
    static __device__ __forceinline__ int swap(int row) { return COL ? col_swap<R>(row) : row_swap<KS>(row); }
    unsigned off[PT];
    static __device__ __forceinline__ int place(int wave, int i)
    {
        const int n = wave + NW * i;
        return N % NW != 0 && n >= N ? n % N : n;
    }
    // `exist` rows (ROW) or columns (COL) of the tile exist; FOLD: the tile's second half is those rows of another matrix.
    template <bool FOLD>
    __device__ __forceinline__ void init(int64_t ld, int exist)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < PT; ++i) {
            const int q = place(wave, i) * 64 + lane, line = q / CS, c = (q - line * CS) ^ swap(line), row = FOLD ? line % (R / 2) : line;
            const bool in = COL ? 8 * c < exist : row < exist;
            off[i] = in ? (unsigned)row * (unsigned)(2 * ld) + 16u * c : 0x80000000u;
        }
    }
    uint64_t base, step;        // bytes: of the step's tile, and to the next one
    unsigned full, row;         // bytes that may be read from base on; of a row of k (COL)
    // The first step of a pass: the tile's first element, and what there is from it on: `rows` rows of `cols` elements of k (ROW), or `cols`
    // columns (COL).
    __device__ __forceinline__ void start(const __bf16* p, int64_t ld, int rows, int cols)
    {
        base = reinterpret_cast<uint64_t>(p);
        step = COL ? (uint64_t)(2 * KS * ld) : 2 * KS;
        full = (unsigned)(2 * ((COL ? KS - 1 : rows - 1) * ld + cols));
        row = (unsigned)(2 * ld);
    }
    // Descriptor of the step's loads, `from` elements further (another plane, or the gates), of which `left` k are there; of nothing where not
    // `live`: then the loads write zeros.
    __device__ __forceinline__ v4i window(int left, bool live, int64_t from) const
    {
        const unsigned n = COL ? full - (unsigned)(KS - min(left, KS)) * row : full;
        return make_rsrc(reinterpret_cast<const void*>(base + 2 * from), live ? n : 0u);
    }
    // Load i; `lane_out`: this lane's piece of k is not there (ROW).
    __device__ __forceinline__ void load(const v4i& r, unsigned lds, bool lane_out, int i) const
    {
        dma16_free(r, !COL && lane_out ? 0x80000000u : off[i], lds + place(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i) * 1024);
    }
    __device__ __forceinline__ void advance()
    {
        base += step;
        if (!COL) full -= 2 * KS;
    }
};

// This lane's places in a tile for its 32 T rows or columns from `first` on.
template <bool COL, int R, int KS, int T>
struct TilePlaces {
    int at[COL ? T : KS / 16];        // bytes: COL per 32 columns; ROW per 16 k
    __device__ __forceinline__ void init(int first)
    {
        const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
        if constexpr (COL) {
            const int q = 8 * h + ((lane & 15) >> 2);
#pragma unroll
            for (int d = 0; d < T; ++d) {
                const int c = first / 8 + 4 * d + ((lane & 16) >> 3) + ((lane & 3) >> 1);
                at[d] = q * (2 * R) + 16 * (c ^ col_swap<R>(q)) + 8 * (lane & 1);
            }
        } else {
#pragma unroll
            for (int t = 0; t < KS / 16; ++t) at[t] = (first + r) * (2 * KS) + 16 * ((2 * t + h) ^ row_swap<KS>(r));
        }
    }
    // operand for 16 k from 16 t on
    __device__ __forceinline__ v8bf read(const char* tile, int u, int t) const
    {
        if constexpr (COL) {
            const char* p = tile + at[u] + t * 16 * (2 * R);
            const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(p));
            const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(p + 4 * (2 * R)));
            return __builtin_bit_cast(v8bf, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *reinterpret_cast<const v8bf*>(tile + at[t] + u * 32 * (2 * KS));
        }
    }
};

// The tile of a workgroup: neighbours in time on one XCD share rows of A and columns of B, in bands of `kBand` tiles along m.
struct MatmulPlace {
    int m, n, slice;
};
__device__ __forceinline__ MatmulPlace matmul_place(const MatmulArgs& p, int id)
{
    constexpr int kBand = 8;
    const int total = p.tiles_m * p.tiles_n * p.slices, per = total >> 3;
    if (id < per << 3) id = (id & 7) * per + (id >> 3);
    const int tiles = p.tiles_m * p.tiles_n;
    MatmulPlace r;
    r.slice = id / tiles;
    id -= r.slice * tiles;
    const int band = id / (kBand * p.tiles_n), first = band * kBand, high = min(kBand, p.tiles_m - first);
    id -= band * kBand * p.tiles_n;
    r.n = id / high;
    r.m = first + id - r.n * high;
    return r;
}

// Four neighbouring results of a row from column n on, as far as there are N.
typedef uint32_t piece8 __attribute__((ext_vector_type(2), aligned(2), may_alias));
__device__ __forceinline__ void put4(void* out, int64_t at, int f32, int n, int N, const float (&v)[4])
{
    const bool all = n + 4 <= N;
    if (f32) {
        float* const o = static_cast<float*>(out) + at;
        if (all) {
            *reinterpret_cast<piece16*>(o) = piece16{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (n + e < N) o[e] = v[e];
        }
    } else {
        __bf16* const o = static_cast<__bf16*>(out) + at;
        if (all) {
            *reinterpret_cast<piece8*>(o) = piece8{pair_bf16(v[0], v[1]), pair_bf16(v[2], v[3])};
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (n + e < N) o[e] = (__bf16)v[e];
        }
    }
}

// Rows of 32 results of a wavefront, on their way to memory through LDS in whole pieces of 16 bytes: as the matrix unit leaves them a
// lane has four of a row's results, and stores of 8 or 16 bytes a row cost the L2 a request each (of 84 MB as codes 8 bytes at a time:
// 40 us).  Lane (h, l32) puts the results 8 q + 4 h + {0..3} of row l32; then the 64 lanes store B bytes of each of the 32 rows.
template <int B>
struct RowStage {
    static constexpr int STRIDE = B + 16, LANES = B / 16;   // (an odd number of places of 16 bytes, or nearly: rows start in different banks)
    char* room;
    template <typename V>
    __device__ __forceinline__ void put(int q, V v) const
    {
        const int lane = threadIdx.x & 63;
        *reinterpret_cast<V*>(room + (lane & 31) * STRIDE + (2 * q + (lane >> 5)) * (int)sizeof(V)) = v;
    }
    // `rows` rows exist, and `bytes` of each, elements of type T
    template <typename T>
    __device__ __forceinline__ void flush(T* to, int64_t ld, int rows, int bytes) const
    {
        asm volatile("" ::: "memory");                   // (a wavefront's accesses of LDS are carried out in order)
        const int lane = threadIdx.x & 63;
        if (bytes % 16 == 0) {
#pragma unroll
            for (int i = 0; i < B / 32; ++i) {
                const int id = i * 64 + lane, r = id / LANES, at = id % LANES * 16;
                const uint4 v = *reinterpret_cast<const uint4*>(room + r * STRIDE + at);
                if (r < rows && at < bytes) *reinterpret_cast<piece16*>(to + r * ld + at / (int)sizeof(T)) = __builtin_bit_cast(piece16, v);
            }
        } else {                                         // (the last columns of a matrix: an element at a time)
            const int n = bytes / (int)sizeof(T);
#pragma unroll 1
            for (int r = lane >> 5; r < rows; r += 2)
                if ((lane & 31) < n) to[r * ld + (lane & 31)] = reinterpret_cast<const T*>(room + r * STRIDE)[lane & 31];
        }
        asm volatile("" ::: "memory");
    }
};

// Four results of each q = 0 .. 3 of 32 rows from column n on, in the type.
template <typename F>
__device__ __forceinline__ void put_rows(char* room, void* out, int64_t ld, int f32, int64_t m0, int rows, int n, int N, F&& value)
{
    const int left = min(N - n, 32);
    if (f32) {
        const RowStage<128> s{room};
#pragma unroll
        for (int q = 0; q < 4; ++q) s.put(q, make_float4(value(4 * q), value(4 * q + 1), value(4 * q + 2), value(4 * q + 3)));
        s.flush(static_cast<uint32_t*>(out) + m0 * ld + n, ld, rows, 4 * left);
    } else {
        const RowStage<64> s{room};
#pragma unroll
        for (int q = 0; q < 4; ++q) s.put(q, make_uint2(pair_bf16(value(4 * q), value(4 * q + 1)), pair_bf16(value(4 * q + 2), value(4 * q + 3))));
        s.flush(static_cast<uint16_t*>(out) + m0 * ld + n, ld, rows, 2 * left);
    }
}

// A block of 32 outputs of 32 rows: values a and gates g, 16 of a row in each of the lanes l and l + 32 (as the matrix unit leaves
// them: places 8 (i / 4) + 4 h + i % 4 from n0 on).  Writes h and what is kept; of blocks the codes, and the scales of a row, values' and gates', to
// scales[row][0], [row][SCALES].
template <int SCALES>
__device__ __forceinline__ void gated_block(const Gate& p, int f32, int64_t m0, int rows, int n0, int N, const float (&a)[16], const float (&g)[16], char* room,
                                            uint8_t* scales)
{
    const int lane = threadIdx.x & 63, h = lane >> 5, np = (N + 31) & ~31;
    if (n0 >= N) return;
    put_rows(room, p.h, p.ld_h, f32, m0, rows, n0, N, [&](int i) { return a[i] * gate_of<false>(p.act, g[i], nullptr); });
    if (!p.pre) return;
    if (!p.pre_scales) {
        put_rows(room, p.pre, p.ld_pre, f32, m0, rows, n0, N, [&](int i) { return a[i]; });
        put_rows(room, f32 ? static_cast<void*>(static_cast<float*>(p.pre) + N) : static_cast<void*>(static_cast<__bf16*>(p.pre) + N), p.ld_pre, f32, m0, rows, n0, N,
                 [&](int i) { return g[i]; });
        return;
    }
    // (columns behind the last are zeros)
    auto codes = [&](const float (&x)[16], uint8_t* to, uint8_t* scale) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
        const uint32_t s = block_scale8(top);
        const float r = inverse_scale(s);
        const RowStage<32> stage{room};
#pragma unroll
        for (int q = 0; q < 4; ++q) stage.put(q, codes8(x[4 * q] * r, x[4 * q + 1] * r, x[4 * q + 2] * r, x[4 * q + 3] * r));
        stage.flush(to, 2 * (int64_t)np, rows, 32);
        if (h == 0) scale[(lane & 31) * 2 * SCALES] = (uint8_t)s;
    };
    uint8_t* const to = static_cast<uint8_t*>(p.pre) + m0 * (2 * (int64_t)np) + n0;
    codes(a, to, scales);
    codes(g, to + np, scales + SCALES);
}

// All but the last COUNT loads of this wavefront have landed, its reads of LDS are done, and all wavefronts are here.
template <int COUNT>
__device__ __forceinline__ void stage_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(COUNT) : "memory");
}

// KS: k of a step; STAGES: of the ring; PL: planes of both operands in a stage, whose six products are made from one read of each, or 1: a
// pass over k for each.
template <bool COLA, bool COLB, int BM, int BN, int WM, int WN, int KS, int STAGES, int PL, int END>
__device__ __forceinline__ void matmul_tile(const MatmulArgs& p, int id)
{
    constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, G = END == kGated ? TN / 2 : TN;
    using FA = TileFeed<COLA, BM, KS, NW>;
    using FB = TileFeed<COLB, BN, KS, NW>;
    constexpr int TILE_A = BM * 2 * KS, TILE_B = BN * 2 * KS, STAGE = PL * (TILE_A + TILE_B), LOADS = PL * (FA::PT + FB::PT);
    static_assert(PL == 1 || PL == 3, "planes");
    static_assert(END != kGated || (!COLB && TN % 2 == 0), "gated: a wavefront has the values and the gates of the same outputs");
    extern __shared__ __align__(1024) char lds[];
    const MatmulPlace at = matmul_place(p, id);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, wm = wave / WN, wn = wave % WN;
    constexpr int CB = END == kGated ? BN / 2 : BN;             // columns of the result in a tile
    const int m0 = at.m * BM, n0 = at.n * CB;
    const int64_t lda = p.a.ld, ldb = p.b.ld;

    FA fa;
    FB fb;
    fa.template init<false>(lda, p.M - m0);
    fb.template init<END == kGated>(ldb, p.N - n0);
    const int64_t gates = (int64_t)p.N * ldb;                   // from a value's row to its gate's
    const int beg = (int)((int64_t)p.total * at.slice / p.slices), end = (int)((int64_t)p.total * (at.slice + 1) / p.slices);
    int pass = beg / p.steps, left = p.K - (beg - pass * p.steps) * KS, todo = end - beg;      // k of the pass and steps that are not loaded yet
    const unsigned base = lds_address(lds);
    unsigned to = base;
    // (of a step: this lane's piece of a ROW tile)
    const int k_lane = 8 * (KS == 32 ? (lane & 3) ^ ((lane >> 4) & 3) : (lane & 7) ^ ((lane >> 4 & 3) | (wave & 1) << 2));
    auto start = [&]() {
        const int k0 = p.K - left, left8 = (left + 7) & ~7;
        const __bf16* const pa = p.a.p + ((p.order_a >> (4 * min(pass, 7))) & 15) * p.a.plane;
        const __bf16* const pb = p.b.p + ((p.order_b >> (4 * min(pass, 7))) & 15) * p.b.plane;
        if constexpr (COLA) fa.start(pa + (int64_t)k0 * lda + m0, lda, 0, ((p.M + 7) & ~7) - m0);
        else fa.start(pa + (int64_t)m0 * lda + k0, lda, min(p.M - m0, BM), left8);
        if constexpr (COLB) fb.start(pb + (int64_t)k0 * ldb + n0, ldb, 0, ((p.N + 7) & ~7) - n0);
        else fb.start(pb + (int64_t)n0 * ldb + k0, ldb, min(p.N - n0, CB), left8);
    };
    v4i wa[PL], wb[PL], wg[PL];
    bool lane_out;
    // A step's loads: their descriptors, load i of LOADS, and the way to the next step.  Behind the last one they write zeros, so that every
    // step has the same number of loads on their way.
    auto windows = [&]() {
#pragma unroll
        for (int q = 0; q < PL; ++q) {
            wa[q] = fa.window(left, todo > 0, q * p.a.plane);
            wb[q] = fb.window(left, todo > 0, q * p.b.plane);
            if constexpr (END == kGated) wg[q] = fb.window(left, todo > 0, q * p.b.plane + gates);
        }
        lane_out = k_lane >= ((left + 7) & ~7);
    };
    auto load = [&](int i) {
        constexpr int EACH = FA::PT + FB::PT;
        const int q = i / EACH, j = i % EACH;
        if (j < FA::PT) fa.load(wa[q], to + q * TILE_A, lane_out, j);
        else if (END == kGated && FB::place(wave, j - FA::PT) >= FB::N / 2) fb.load(wg[q], to + PL * TILE_A + q * TILE_B, lane_out, j - FA::PT);
        else fb.load(wb[q], to + PL * TILE_A + q * TILE_B, lane_out, j - FA::PT);
    };
    auto loaded = [&]() {
        fa.advance();
        fb.advance();
        --todo;
        left -= KS;
        to = to + STAGE == base + STAGES * STAGE ? base : to + STAGE;
        if (left <= 0) {
            left = p.K;
            ++pass;
            start();
        }
    };

    TilePlaces<COLA, BM, KS, TM> ra;
    TilePlaces<COLB, BN, KS, G> rb;
    ra.init(wm * TM * 32);
    rb.init(wn * G * 32);
    v16f acc[TM][TN];
#pragma unroll
    for (int u = 0; u < TM; ++u)
#pragma unroll
        for (int v = 0; v < TN; ++v) acc[u][v] = zero16();
    float sums[TM] = {};                                        // kSums: of this lane's k

    struct Operands {
        v8bf a[PL][TM], b[PL][TN];
    };
    // Read i of the PL (TM + TN) of a step's half t, product i of its TM TN (PL == 3: six times that, small ones first).
    constexpr int MM = TM * TN * (PL == 3 ? 6 : 1), RD = PL * (TM + TN);
    auto read = [&](Operands& o, const char* ta, int t, int i) {
        const int q = i / (TM + TN), j = i % (TM + TN);
        if (j < TN) o.b[q][j] = rb.read(ta + PL * TILE_A + q * TILE_B + j / G * CB * 2 * KS, j % G, t);
        else o.a[q][j - TN] = ra.read(ta + q * TILE_A, j - TN, t);
    };
    auto multiply = [&](const Operands& o, int i) {
        constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
        const int c = i / (TM * TN), u = i % (TM * TN) / TN, v = i % TN;
        acc[u][v] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(o.b[PL == 3 ? pb[c] : 0][v], o.a[PL == 3 ? pa[c] : 0][u], acc[u][v], 0, 0, 0);
    };

    // The sums of A: its values times one, two at a time, by vector instructions that run beside the products.
    // Only the first tiles along n make them, in loops of their own, each wavefront of one of the operands that it shares with another.  What 16 steps
    // gave, 256 or 384 pairs a lane, is set aside, so that no sum's roundings grow with the length (4 M equal rows in fp32: off by 1e-7 for 0.0017).
    auto add = [&](const Operands& o, int i) {
        const v8bf a = o.a[i / TM][i % TM];
        const v2bf one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
        for (int k = 0; k < 4; ++k) sums[i % TM] = __builtin_amdgcn_fdot2_f32_bf16(v2bf{a[2 * k], a[2 * k + 1]}, one, sums[i % TM], false);
    };

    auto run = [&](auto with) {
        constexpr int SUMS = decltype(with)::value;             // of the operands u that this wavefront sums up: -1 none
        float aside = 0.0f;
        start();
        Operands even, odd;
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) {
            windows();
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load(i);
            loaded();
        }
        const char* tile = lds;
        // Products of one half, and between them the reads of the other and the loads of a step ahead, one at a time: they are issued
        // while the matrix unit is busy.
        auto half = [&](const Operands& now, Operands& next, int t, auto loads) {
#pragma unroll
            for (int i = 0; i < (MM > RD ? MM : RD); ++i) {
                if (i < MM) multiply(now, i);
                if (i < RD) read(next, tile, t, i);
                if constexpr (SUMS >= 0)
                    if (i < PL * TM && i % TM == SUMS) add(now, i);
                if constexpr (decltype(loads)::value) {
                    constexpr int EACH = (LOADS + MM - 1) / MM;
#pragma unroll
                    for (int j = 0; j < EACH; ++j)
                        if (i * EACH + j < LOADS) load(i * EACH + j);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto advance = [&]() { tile = tile + STAGE == lds + STAGES * STAGE ? lds : tile + STAGE; };
        stage_barrier<(STAGES - 2) * LOADS>();
#pragma unroll
        for (int i = 0; i < RD; ++i) read(even, tile, 0, i);
        windows();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(i);
        loaded();
        half(even, odd, 1, std::false_type());
        if constexpr (KS == 64) {
            half(odd, even, 2, std::false_type());
            half(even, odd, 3, std::false_type());
        }
        advance();
        for (int it = beg + 1; it < end; ++it) {
            stage_barrier<(STAGES - 2) * LOADS>();
            windows();
            __builtin_amdgcn_s_setprio(1);                  // (a wavefront that has loads to start goes first: two tiles of 128 rows a compute unit gain 5 %)
            half(odd, even, 0, std::true_type());
            __builtin_amdgcn_s_setprio(0);
            loaded();
            half(even, odd, 1, std::false_type());
            if constexpr (KS == 64) {
                half(odd, even, 2, std::false_type());
                half(even, odd, 3, std::false_type());
            }
            advance();
            if constexpr (SUMS >= 0)
                if (((it - beg) & 15) == 15) {
                    aside += sums[SUMS];
                    sums[SUMS] = 0.0f;
                }
        }
#pragma unroll
        for (int i = 0; i < MM; ++i) multiply(odd, i);
        if constexpr (SUMS >= 0) {
#pragma unroll
            for (int i = 0; i < PL * TM; ++i)
                if (i % TM == SUMS) add(odd, i);
            sums[SUMS] += aside;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    if constexpr (END == kSums) static_assert(TM <= WN && WN == 2, "wavefront n sums operand n");
    if (beg < end) {
        if (END != kSums || at.n || wn >= TM) run(std::integral_constant<int, -1>());
        else if (wn == 0) run(std::integral_constant<int, END == kSums ? 0 : -1>());
        else run(std::integral_constant<int, END == kSums ? TM - 1 : -1>());
    }

    const int h = lane >> 5;
    if constexpr (END == kSums) {
#pragma unroll
        for (int u = 0; u < TM; ++u) {
            const float all = sums[u] + __shfl_xor(sums[u], 32, 64);
            const int m = m0 + (wm * TM + u) * 32 + lane;
            if (at.n == 0 && wn == u && h == 0 && m < p.M) p.sums[(int64_t)at.slice * p.M + m] = all;
        }
    }
    if (p.slices > 1) {
        __syncthreads();                                        // the ring is free
        constexpr int ROOM = RowStage<128>::STRIDE * 32;
        static_assert(NW * ROOM <= STAGES * STAGE, "room for the results on their way");
        const int cols = END == kGated ? 2 * p.N : p.N;
        float* const part = static_cast<float*>(p.out) + (int64_t)at.slice * p.M * cols;
#pragma unroll
        for (int v = 0; v < TN; ++v) {
            const int nb = n0 + (wn * G + v % G) * 32;
            if (nb >= p.N) continue;
#pragma unroll
            for (int u = 0; u < TM; ++u) {
                const int m = m0 + (wm * TM + u) * 32;
                if (m >= p.M) break;
                put_rows(lds + wave * ROOM, part + (END == kGated ? v / G * p.N : 0), cols, 1, m, min(p.M - m, 32), nb, p.N,
                         [&](int i) { return acc[u][v][i]; });
            }
        }
        return;
    }
    if constexpr (END == kGated) {
        __syncthreads();                                        // the ring is free
        constexpr int SC = WN * G, ROOM = RowStage<128>::STRIDE * 32;
        static_assert(NW * ROOM + BM * 2 * SC <= STAGES * STAGE, "room for the results on their way");
        uint8_t* const scales = reinterpret_cast<uint8_t*>(lds) + NW * ROOM;     // [BM][values, gates][blocks of the tile]
#pragma unroll
        for (int v = 0; v < G; ++v) {
            const int nb = n0 + (wn * G + v) * 32;
            float ba[16], bg[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int n = nb + 8 * (i / 4) + 4 * h + i % 4;
                ba[i] = p.bias && n < p.N ? p.bias[n] : 0.0f;
                bg[i] = p.bias && n < p.N ? p.bias[p.N + n] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < TM; ++u) {
                const int row = (wm * TM + u) * 32, m = m0 + row;
                if (m >= p.M) break;
                float a[16], g[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    a[i] = acc[u][v][i] + ba[i];
                    g[i] = acc[u][G + v][i] + bg[i];
                }
                if (nb + 32 > p.N) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (nb + 8 * (i / 4) + 4 * h + i % 4 >= p.N) a[i] = g[i] = 0.0f;
                }
                gated_block<SC>(p.gate, p.out_f32, m, min(p.M - m, 32), nb, p.N, a, g, lds + wave * ROOM, scales + row * 2 * SC + wn * G + v);
            }
        }
        if (p.gate.pre_scales) {
            __syncthreads();
            // a row's scales of the tile lie together
            const int all = (p.N + 31) / 32, first = n0 / 32, here = min(all - first, SC);
            const bool words = SC == 4 && here == 4 && all % 4 == 0 && ((uintptr_t)p.gate.pre_scales & 3) == 0;
            for (int i = threadIdx.x; i < 2 * min(BM, p.M - m0); i += 64 * NW) {
                uint8_t* const to = p.gate.pre_scales + (int64_t)(m0 + i / 2) * (2 * all) + i % 2 * all + first;
                if (words) *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(scales + i * SC);
                else
                    for (int k = 0; k < here; ++k) to[k] = scales[i * SC + k];
            }
        }
    } else {
        __syncthreads();                                        // the ring is free
        constexpr int ROOM = RowStage<128>::STRIDE * 32;
        static_assert(NW * ROOM <= STAGES * STAGE, "room for the results on their way");
#pragma unroll
        for (int v = 0; v < TN; ++v) {
            const int nb = n0 + (wn * TN + v) * 32;
            if (nb >= p.N) continue;
            float b[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int n = nb + 8 * (i / 4) + 4 * h + i % 4;
                b[i] = p.bias && n < p.N ? p.bias[n] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < TM; ++u) {
                const int m = m0 + (wm * TM + u) * 32;
                if (m >= p.M) break;
                put_rows(lds + wave * ROOM, p.out, p.ld_out, p.out_f32, m, min(p.M - m, 32), nb, p.N, [&](int i) { return acc[u][v][i] + b[i]; });
            }
        }
    }
}

// (Two wavefronts per SIMD: one workgroup of eight, or two of four.)
template <bool COLA, bool COLB, int BM, int BN, int WM, int WN, int KS, int STAGES, int PL, int END>
__global__ __launch_bounds__(64 * WM * WN, 2) void matmul_kernel(MatmulArgs p)
{
    matmul_tile<COLA, COLB, BM, BN, WM, WN, KS, STAGES, PL, END>(p, blockIdx.x);
}

// d w and d^T x: those of the two whose workgroups take longer are the first `first`.
template <int BM, int BN, int WM, int WN, int KS, int STAGES, int PL, int END>
__global__ __launch_bounds__(64 * WM * WN, 2) void matmul_both_kernel(MatmulArgs x, MatmulArgs w, int first, int x_first)
{
    const bool front = (int)blockIdx.x < first;
    const int id = front ? blockIdx.x : blockIdx.x - first;
    if (front == (x_first != 0)) matmul_tile<false, true, BM, BN, WM, WN, KS, STAGES, PL, kStore>(x, id);
    else matmul_tile<true, true, BM, BN, WM, WN, KS, STAGES, PL, END>(w, id);
}

// A product as the callers give it: M, N, K, operands, `planes` of each, forms, and what becomes of it.
struct Product {
    Operand a, b;
    int64_t M, N, K;
    int planes_a, planes_b;
    bool col_a, col_b;
    void* out;
    int64_t ld_out;
    int out_f32;
    const float* bias;
    float* sums;                // of A over k (col_a; where plan_sums allows it), or null
    bool gated;
    Gate gate;
};
// How a product is made: its tile (matmul_tiles.h), in how many slices of k, and an estimate of its time.  By sizes and planes alone, so that the same
// plan gives the workspace's size and the launch.
struct ProductPlan {
    int tile, slices;
    double us;
};
ProductPlan plan_product(int64_t M, int64_t N, int64_t K, int planes_a, int planes_b, bool col_a, bool gated);
// Bytes of partial results (0 where it is made in one slice).
size_t product_part_bytes(const ProductPlan& plan, int64_t M, int64_t N, bool col_a, bool gated);
int launch_product(const Product& p, const ProductPlan& plan, void* part, hipStream_t s);

// Planes of what both gradients of a layer are made from: d [M, N], w [N, K], x [M, K].
struct Planes {
    int d, w, x;
};
// Both gradients of y = x w^T for d: each on its own, and together in one launch where that is faster (tile >= 0).  A call makes this once: it takes the host
// some microseconds.
struct GradientPlan {
    ProductPlan x, w;
    int tile, slices_x, slices_w;
};
GradientPlan plan_gradients(int64_t M, int64_t N, int64_t K, Planes planes);
// Bytes of partial results of whichever gradients are made.
size_t gradient_part_bytes(const GradientPlan& plan, int64_t M, int64_t N, int64_t K);
// Whether grad_w can give the sums of d in a launch of its own; together with grad_x it always can.
bool plan_sums(const GradientPlan& plan, int planes_x);
// x.M, N, K = M, K, N, by rows and by columns, w.M, N, K = N, K, M, both by columns.
int launch_products(const Product& x, const Product& w, const GradientPlan& plan, void* part, hipStream_t s);

}  // namespace fpq
