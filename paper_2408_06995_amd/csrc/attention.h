// Attention and its gradient: what the kernels share.
//
// Every product is a 32 x 32 x 16 step of the bf16 matrix instruction with fp32 sums.  An operand of type bf16 is one plane of
// its own values; an fp32 operand is split into three planes of 8 significant bits each (x = h + m + l, as in rounding.hip), of
// whose nine products the six largest are taken: what is left out is at most 2^-24 of a product, less than the rounding of an
// fp32 sum.
//
// Operand layout of the instruction, lane = 32 h + r: A holds row r, B column r, each the eight k-places (h, 0..7); C holds
// column r and rows 8 (i / 4) + 4 h + i % 4 of its 16 values i.  Any order of k will do if A and B agree.  So a C tile is used as
// an operand where it lies: values 8 s .. 8 s + 7 of a lane are the k-places (h, 0..7) of step s for the contraction over the
// tile's rows, and the other operand takes the rows 16 s + 4 h + {0..3} and 16 s + 8 + 4 h + {0..3} in that order.  Those come from
// a row-major tile in LDS by the transposing read, which gives a lane four rows of its column.  Scores and their gradients
// therefore never leave the registers, and one row-major copy of a tile serves both kinds of reads.
#pragma once
#include "fpq_dev.h"
#include "fpq_host.h"
#include "lds_dma.h"

namespace fpq {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4s* lds_v4s;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

template <typename T>
constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;

// Elements of a tile row in LDS for KS steps of 16 columns: 16 bytes more, which make the row an odd number of 16-byte places, so
// that the 16 rows of a quarter wave's read start in different banks.  Output tiles of 32 columns may reach past a row with an odd
// KS: those columns of the result are not used, and the tile has kSlack bytes behind it.
template <int KS>
constexpr int kRowStride = 16 * KS + 8;
constexpr int kSlack = 64;

template <int NP>
struct Frag {
    v8bf p[NP];
};

template <int NP>
__device__ __forceinline__ void mma(v16f& c, const Frag<NP>& a, const Frag<NP>& b)
{
    if constexpr (NP == 3) {                       // small products first
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[2], b.p[0], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[0], b.p[2], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[1], b.p[1], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[1], b.p[0], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[0], b.p[1], c, 0, 0, 0);
    }
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[0], b.p[0], c, 0, 0, 0);
}

__device__ __forceinline__ v16f zero16()
{
    v16f z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}

__device__ __forceinline__ uint32_t pair_bf16(float a, float b)
{
    const v2f v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, v2bf));      // round to nearest even
}

// The planes of two neighbouring values, each difference exact.
template <int NP>
__device__ __forceinline__ void planes_of_pair(float a, float b, uint32_t (&out)[NP])
{
    out[0] = pair_bf16(a, b);
    if constexpr (NP == 3) {
        const float ra = a - __uint_as_float(out[0] << 16), rb = b - __uint_as_float(out[0] & 0xffff0000u);
        out[1] = pair_bf16(ra, rb);
        out[2] = pair_bf16(ra - __uint_as_float(out[1] << 16), rb - __uint_as_float(out[1] & 0xffff0000u));
    }
}

template <int NP>
__device__ __forceinline__ Frag<NP> frag_of(const float* v)
{
    uint32_t w[NP][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        uint32_t o[NP];
        planes_of_pair<NP>(v[2 * t], v[2 * t + 1], o);
#pragma unroll
        for (int p = 0; p < NP; ++p) w[p][t] = o[p];
    }
    Frag<NP> f;
#pragma unroll
    for (int p = 0; p < NP; ++p) f.p[p] = __builtin_bit_cast(v8bf, make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]));
    return f;
}

// Eight columns from `col` on of a row in memory, zero from column `dim` on.  VEC: 16-byte aligned rows of a whole number of
// 16-byte pieces.
template <typename T, bool VEC>
__device__ __forceinline__ void row8(const T* row, int col, int dim, float (&v)[8])
{
    if constexpr (VEC && sizeof(T) == 4) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int c = col + 4 * t;
            const float4 x = *reinterpret_cast<const float4*>(row + min(c, dim - 4));
            const bool in = c < dim;
            v[4 * t] = in ? x.x : 0.0f;
            v[4 * t + 1] = in ? x.y : 0.0f;
            v[4 * t + 2] = in ? x.z : 0.0f;
            v[4 * t + 3] = in ? x.w : 0.0f;
        }
    } else if constexpr (VEC) {
        const uint4 x = *reinterpret_cast<const uint4*>(row + min(col, dim - 8));
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            v[2 * t] = col < dim ? __uint_as_float(w[t] << 16) : 0.0f;
            v[2 * t + 1] = col < dim ? __uint_as_float(w[t] & 0xffff0000u) : 0.0f;
        }
    } else {
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = col + t < dim ? (float)row[min(col + t, dim - 1)] : 0.0f;
    }
}

// Operand rows from LDS: lane r's row, eight columns.
template <int NP, int RS, int ROWS>
__device__ __forceinline__ Frag<NP> row_frag(const __bf16* tile, int row, int col)
{
    Frag<NP> f;
#pragma unroll
    for (int p = 0; p < NP; ++p) f.p[p] = *reinterpret_cast<const v8bf*>(tile + (p * ROWS + row) * RS + col);
    return f;
}

// Operand columns from LDS: lane (h, r) gets column c0 + r of rows r0 + 4 h + {0..3} and r0 + 8 + 4 h + {0..3}.  Of the 16 lanes
// that read a block of 4 rows x 16 columns, lane i names four columns of row i / 4 and receives column i.
template <int NP, int RS, int ROWS>
__device__ __forceinline__ Frag<NP> col_frag(const __bf16* tile, int r0, int c0, int lane)
{
    const __bf16* at = tile + (r0 + 4 * (lane >> 5) + ((lane & 15) >> 2)) * RS + c0 + (lane & 16) + (lane & 3) * 4;
    Frag<NP> f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(at + p * ROWS * RS));
        const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(at + (p * ROWS + 8) * RS));
        f.p[p] = __builtin_bit_cast(v8bf, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    return f;
}

// ROWS rows of a matrix in memory on their way to an LDS tile: load() a step ahead, store() when the tile is free.  Rows past
// `last` are not read; rows from `end` on and columns from `dim` on become zero, whatever memory holds there.
template <typename T, int KS, bool VEC, int ROWS, int NT>
struct Stage {
    static constexpr int E = 16 / sizeof(T), CH = 16 * KS / E, N = ROWS * CH, PT = (N + NT - 1) / NT, NP = kPlanes<T>;
    static constexpr int RS = kRowStride<KS>;
    uint4 reg[PT];
    __device__ __forceinline__ void load(const T* base, int64_t stride, int row0, int last, int dim, int tid)
    {
#pragma unroll
        for (int it = 0; it < PT; ++it) {
            const int id = it * NT + tid, row = id / CH, c = (id - row * CH) * E;
            const T* p = base + (int64_t)min(row0 + row, last) * stride;
            if constexpr (VEC) {
                reg[it] = *reinterpret_cast<const uint4*>(p + min(c, dim - E));
            } else {
                T v[E];
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = p[min(c + e, dim - 1)];
                __builtin_memcpy(&reg[it], v, 16);
            }
        }
    }
    __device__ __forceinline__ void store(__bf16* tile, int row0, int end, int dim, int tid)
    {
#pragma unroll
        for (int it = 0; it < PT; ++it) {
            const int id = it * NT + tid, row = id / CH, c = (id - row * CH) * E;
            if (N % NT != 0 && id >= N) continue;
            const bool in = row0 + row < end;
            uint4 w = reg[it];
            if constexpr (VEC) {
                if (!(in && c < dim)) w = make_uint4(0, 0, 0, 0);
            } else {
                T v[E];
                __builtin_memcpy(v, &w, 16);
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = in && c + e < dim ? v[e] : (T)0.0f;
                __builtin_memcpy(&w, v, 16);
            }
            if constexpr (NP == 1) {
                *reinterpret_cast<uint4*>(tile + row * RS + c) = w;
            } else {
                uint32_t lo[3], hi[3];
                planes_of_pair<3>(__uint_as_float(w.x), __uint_as_float(w.y), lo);
                planes_of_pair<3>(__uint_as_float(w.z), __uint_as_float(w.w), hi);
#pragma unroll
                for (int p = 0; p < 3; ++p) *reinterpret_cast<uint2*>(tile + (p * ROWS + row) * RS + c) = make_uint2(lo[p], hi[p]);
            }
        }
    }
};

// Two matrices on their way through LDS, tile by tile of ROWS rows from the same row on.  begin() starts a tile, ready()
// makes it readable for the whole workgroup.
//
// bf16 rows of whole 16-byte pieces go from memory to LDS directly, a tile ahead, into the other one of two buffers: no registers, no
// instructions per piece, one barrier per tile.  A descriptor per tile bounds the reads, so that rows past the last and columns past
// the dimension (whose offsets are out of range) become zeros; its base moves in 64 bits, offsets within a tile fit 32.
// Others pass through registers (fp32: split on the way).
template <typename T, int KS, bool VEC, int ROWS, int NW, bool DIRECT = (sizeof(T) == 2 && VEC)>
struct Feed {
    static constexpr int CHP = 2 * KS + 1, N = (ROWS * CHP + 63) / 64, PW = (N + NW - 1) / NW, TILE = N * 1024, RS = kRowStride<KS>;
    static constexpr int LDS = 4 * TILE + kSlack;
    static constexpr bool kDirect = true;
    unsigned off[2][PW];
    const T* base[2];
    int64_t stride[2];
    unsigned lds;
    int dim, buf, now;
    __device__ __forceinline__ void init(unsigned char* at, const T* a, int64_t sa, const T* b, int64_t sb, int dim_)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        base[0] = a;
        base[1] = b;
        stride[0] = sa;
        stride[1] = sb;
        dim = dim_;
        buf = 1;
        lds = lds_address(at);
#pragma unroll
        for (int i = 0; i < PW; ++i) {
            const int q = (wave + NW * i) * 64 + lane, row = q / CHP, c = q - row * CHP;
#pragma unroll
            for (int m = 0; m < 2; ++m) off[m][i] = row < ROWS && 8 * c < dim ? (unsigned)row * (unsigned)(2 * stride[m]) + 16u * c : 0x80000000u;
        }
    }
    // rows row0 .. end - 1 of the tile exist (at least one)
    __device__ __forceinline__ void begin(int row0, int end)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rows = min(ROWS, end - row0);
        buf ^= 1;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const v4i r = make_rsrc(base[m] + (int64_t)row0 * stride[m], 2u * ((unsigned)(rows - 1) * (unsigned)stride[m] + (unsigned)dim));
#pragma unroll
            for (int i = 0; i < PW; ++i)
                if (wave + NW * i < N) dma16(r, off[m][i], lds + (2 * buf + m) * TILE + (wave + NW * i) * 1024);
        }
    }
    __device__ __forceinline__ void ready(int, int)
    {
        dma_barrier();
        now = buf;
    }
    __device__ __forceinline__ int at(int m) const { return (2 * now + m) * (TILE / 2); }      // the readable tile, in elements
};

template <typename T, int KS, bool VEC, int ROWS, int NW>
struct Feed<T, KS, VEC, ROWS, NW, false> {
    static constexpr int NP = kPlanes<T>, RS = kRowStride<KS>, TILE = NP * ROWS * RS * 2;
    static constexpr int LDS = 2 * TILE + kSlack;
    static constexpr bool kDirect = false;
    Stage<T, KS, VEC, ROWS, 64 * NW> st[2];
    const T* base[2];
    int64_t stride[2];
    __bf16* tile;
    int dim;
    __device__ __forceinline__ void init(unsigned char* at, const T* a, int64_t sa, const T* b, int64_t sb, int dim_)
    {
        tile = reinterpret_cast<__bf16*>(at);
        base[0] = a;
        base[1] = b;
        stride[0] = sa;
        stride[1] = sb;
        dim = dim_;
    }
    __device__ __forceinline__ void begin(int row0, int end)
    {
#pragma unroll
        for (int m = 0; m < 2; ++m) st[m].load(base[m], stride[m], row0, end - 1, dim, threadIdx.x);
    }
    __device__ __forceinline__ void ready(int row0, int end)
    {
        __syncthreads();
#pragma unroll
        for (int m = 0; m < 2; ++m) st[m].store(tile + m * TILE / 2, row0, end, dim, threadIdx.x);
        __syncthreads();
    }
    __device__ __forceinline__ int at(int m) const { return m * (TILE / 2); }
};

// Four neighbouring values from column d on; `vec`: the row is aligned for one store.
__device__ __forceinline__ void store4(float* row, int d, int dim, bool vec, const float (&v)[4])
{
    if (vec) {
        if (d < dim) *reinterpret_cast<float4*>(row + d) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (d + e < dim) row[d + e] = v[e];
    }
}
__device__ __forceinline__ void store4(__bf16* row, int d, int dim, bool vec, const float (&v)[4])
{
    if (vec) {
        if (d < dim) *reinterpret_cast<uint2*>(row + d) = make_uint2(pair_bf16(v[0], v[1]), pair_bf16(v[2], v[3]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (d + e < dim) row[d + e] = (__bf16)v[e];
    }
}

// Strides in elements: sample, token, head.
struct Strides {
    int64_t b, t, h;
};

struct AttentionArgs {
    const void *q, *k, *v, *o, *go;
    void *out, *gq, *gk, *gv;
    float *lse, *stats;         // stats: per row its log-sum in base 2 (infinity for a row without keys) and its delta
    const int32_t* lens;
    Strides qs, ks, vs, os, gos, gqs, gks, gvs;
    int batch, kv_heads, group, q_len, kv_len, dim, causal;
    float scale;
    int blocks;                 // blocks of rows (or keys) per sample and key head
    int splits, per_split;      // parts of the other axis, and its keys (or tiles of queries) per part
    int vec_out;                // results may be stored four values at a time (bit 0: out / gq)
    float *part, *part_lse;     // splits > 1: results of the parts
};

// The part of the grid that a workgroup works on.  Workgroups go round-robin over the eight XCDs; each XCD takes a contiguous run
// of them, so that the blocks that read the same keys share an L2.  Under `causal` blocks differ in length by up to their number:
// the longest (number 0) of all heads of an XCD go first.
struct Place {
    int bh, split, block;
};
__device__ __forceinline__ Place place_of(const AttentionArgs& a)
{
    const int total = gridDim.x, per = total >> 3, bhs = a.batch * a.kv_heads;
    int id = blockIdx.x;
    Place p;
    if (a.causal) {
        const bool whole = (bhs & 7) == 0;
        const int local = whole ? bhs >> 3 : bhs;
        if (whole) id >>= 3;
        p.split = id % a.splits;
        id /= a.splits;
        p.bh = id % local + (whole ? (int)(blockIdx.x & 7) * local : 0);
        p.block = id / local;
        return p;
    }
    if (id < (per << 3)) id = (id & 7) * per + (id >> 3);
    p.block = id % a.blocks;
    id /= a.blocks;
    p.split = id % a.splits;
    p.bh = id / a.splits;
    return p;
}

__device__ __forceinline__ int keys_of(const AttentionArgs& a, int b)
{
    return a.lens ? min(max(a.lens[b], 0), a.kv_len) : a.kv_len;
}

// The queries of all heads of a group are the rows of one matrix (head by head): the group reads its keys once, and single
// tokens fill a tile together.
struct RowRange {
    int hi, lo;                 // keys from hi on are hidden from all rows of the block, keys below lo from none
};
__device__ __forceinline__ RowRange visible(const AttentionArgs& a, int n, int first, int last)
{
    RowRange v = {n, n};
    if (a.causal) {
        const int off = n - a.q_len, g0 = first / a.q_len, g1 = last / a.q_len;
        const bool one = g0 == g1;
        v.hi = one ? max(0, min(n, last - g1 * a.q_len + off + 1)) : n;
        v.lo = max(0, min(n, (one ? first - g0 * a.q_len : 0) + off + 1));
    }
    return v;
}

constexpr int KeysTile = 32;    // queries of a tile of the backward pass's keys kernel (host and device)

// How a call's kernels are chosen and cut (host): by sizes, type and alignment only, the same for the size of the workspace.
struct AttentionPlan {
    bool by_keys;               // forward: the wavefronts of a workgroup share 32 rows and divide the keys
    int blocks, splits, per_split;
    int q_blocks, q_splits, q_per_split;      // backward, gradient of the queries
    int k_blocks, k_splits, k_per_split;      // backward, gradient of the keys and values
};

int launch_attention(const AttentionArgs& a, int type, bool vec, const AttentionPlan& p, hipStream_t s);
int launch_attention_backward(const AttentionArgs& a, int type, bool vec, const AttentionPlan& p, float* part_q, float* part_kv, hipStream_t s);
AttentionPlan plan_attention(int64_t batch, int64_t kv_heads, int64_t group, int64_t q_len, int64_t kv_len);

}  // namespace fpq
