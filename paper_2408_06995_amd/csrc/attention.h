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
#include "attention_plan.h"
#include "fpq_dev.h"
#include "fpq_host.h"
#include "lds_dma.h"

namespace fpq {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4s* lds_v4s;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

template <typename T>
constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
// Planes of the probabilities and their gradients as operands.  Beside bf16 operands two, 16 significant bits.  One would round them by as
// much as the results are: errors of 1.4 times a result's own rounding (0.0024 of its norm for 0.0017), 1.5 in gradients of few rows and
// keys.  It would also be faster, 4 x 16 heads on 4 of 2048 x 128 forward 171 us for 221 and backward 501 for 654.
template <typename T>
constexpr int kPlanesP = sizeof(T) == 4 ? 3 : 2;

// Elements of a tile row in LDS for KS steps of 16 columns: 16 bytes more, which make the row an odd number of 16-byte places, so
// that the 16 rows of a quarter wave's read start in different banks.
template <int KS>
constexpr int kRowStride = 16 * KS + 8;

template <int NP>
struct Frag {
    v8bf p[NP];
};

template <int NA, int NB>
__device__ __forceinline__ void mma(v16f& c, const Frag<NA>& a, const Frag<NB>& b)
{
    static_assert(NA == NB || NA * NB == 2, "three planes with three, or one with one or two");
    if constexpr (NA == 1 && NB == 2) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[0], b.p[1], c, 0, 0, 0);
    if constexpr (NA == 2 && NB == 1) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[1], b.p[0], c, 0, 0, 0);
    if constexpr (NA == 3) {                       // small products first
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
    if constexpr (NP >= 2) {
        const float ra = a - __uint_as_float(out[0] << 16), rb = b - __uint_as_float(out[0] & 0xffff0000u);
        out[1] = pair_bf16(ra, rb);
        if constexpr (NP == 3) out[2] = pair_bf16(ra - __uint_as_float(out[1] << 16), rb - __uint_as_float(out[1] & 0xffff0000u));
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
        for (int t = 0; t < 8; ++t) {
            const float x = (float)row[min(col + t, dim - 1)];           // (loaded in any case: no branch)
            v[t] = col + t < dim ? x : 0.0f;
        }
    }
}

// A lane's part of a whole row: columns 16 s + 8 h .. + 7 of every step s.  All loads are under way before the first is waited for.
template <typename T, int KS>
__device__ __forceinline__ void row_all(const T* row, int h, int dim, int vec, float (&v)[KS][8])
{
    if (vec) {
#pragma unroll
        for (int s = 0; s < KS; ++s) row8<T, true>(row, 16 * s + 8 * h, dim, v[s]);
    } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) row8<T, false>(row, 16 * s + 8 * h, dim, v[s]);
    }
}
template <typename T, int KS, int NP>
__device__ __forceinline__ void row_frags(const T* row, int h, int dim, int vec, Frag<NP> (&f)[KS])
{
    float v[KS][8];
    row_all<T, KS>(row, h, dim, vec, v);
#pragma unroll
    for (int s = 0; s < KS; ++s) f[s] = frag_of<NP>(v[s]);
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

// A matrix as the feed reads it: NP planes of bf16 rows of whole 16-byte pieces.  bf16 tensors with such rows are read where they
// are; others are packed first (attention_pack.hip).
struct Source {
    const __bf16* p;
    Strides s;                  // in elements
    int64_t plane;              // from one plane to the next
};

// LDS tiles of the feed: a row has CS places of 16 bytes, and place c ^ swap(row) holds piece c, so that neither kind of read
// meets a bank twice: 16 rows of one piece (operand rows) start in the 16 different groups of four banks, and so do four rows of
// four pieces (transposed reads, half a wavefront at a time).
template <int KS>
struct Places {
    static constexpr int CS = KS <= 4 ? 8 : KS <= 6 ? 12 : KS <= 8 ? 16 : 20, RS = 8 * CS, DT = (KS + 1) / 2;
    static __device__ __forceinline__ int swap(int row)
    {
        if (CS == 8) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
        if (CS == 16) return (row & 3) << 2 | ((row >> 2) & 3);
        return (row >> 2) & 3;
    }
    int row[KS];                // of this lane, in elements: its row (lane % 32), step t
    int col[DT][2];             // its part of a transposed read: output columns 32 d, rows 0 .. 3 and 8 .. 11 (+ 4 h)
    __device__ __forceinline__ void init(int lane)
    {
        const int r = lane & 31, h = lane >> 5;
#pragma unroll
        for (int t = 0; t < KS; ++t) row[t] = r * RS + 8 * ((2 * t + h) ^ swap(r));
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int q = 4 * h + ((lane & 15) >> 2) + 8 * e, c = 4 * d + ((lane & 16) >> 3) + ((lane & 3) >> 1);
                col[d][e] = q * RS + 8 * (c ^ swap(q)) + 4 * (lane & 1);
            }
    }
};

// Operand rows 32 u + lane % 32, step t, and operand columns 32 d + lane % 32 of the rows r0 .. r0 + 15 (r0 a multiple of 16), of a
// tile whose planes are `plane` elements apart.
template <int NP, int KS>
__device__ __forceinline__ Frag<NP> rows_at(const __bf16* tile, int plane, const Places<KS>& at, int u, int t)
{
    Frag<NP> f;
#pragma unroll
    for (int p = 0; p < NP; ++p) f.p[p] = *reinterpret_cast<const v8bf*>(tile + p * plane + 32 * u * Places<KS>::RS + at.row[t]);
    return f;
}
template <int NP, int KS>
__device__ __forceinline__ Frag<NP> cols_at(const __bf16* tile, int plane, const Places<KS>& at, int r0, int d)
{
    Frag<NP> f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(tile + p * plane + r0 * Places<KS>::RS + at.col[d][0]));
        const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(tile + p * plane + r0 * Places<KS>::RS + at.col[d][1]));
        f.p[p] = __builtin_bit_cast(v8bf, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    return f;
}

// M matrices from memory to LDS, tile by tile of ROWS rows, a tile ahead, into the other one of two buffers: no registers, no
// instructions per piece, one barrier per tile.  A descriptor per tile bounds the reads, so that rows past the last and columns
// past the dimension (whose offsets are out of range) become zeros; its base moves in 64 bits, offsets within a tile fit 32.
// begin() starts a tile, ready() makes the one begun last readable for the whole workgroup.
template <int NP, int KS, int ROWS, int M, int NW>
struct Feed {
    static constexpr int CS = Places<KS>::CS, N = ROWS * CS / 64, PW = (N + NW - 1) / NW, PLANE = ROWS * CS * 16, TILE = NP * PLANE, LDS = 2 * M * TILE;
    unsigned off[M][PW];
    Source src[M];              // p: of row 0 of the head
    unsigned lds;
    int buf, now, cols;         // cols: columns that exist, in whole pieces
    __device__ __forceinline__ void init(unsigned lds_at, int dim)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        buf = 1;
        lds = lds_at;
        cols = (dim + 7) / 8 * 8;
#pragma unroll
        for (int i = 0; i < PW; ++i) {
            const int q = (wave + NW * i) * 64 + lane, row = q / CS, c = (q - row * CS) ^ Places<KS>::swap(row);
#pragma unroll
            for (int m = 0; m < M; ++m) off[m][i] = 8 * c < cols ? (unsigned)row * (unsigned)(2 * src[m].s.t) + 16u * c : 0x80000000u;
        }
    }
    // rows row0 .. end - 1 exist (at least one)
    __device__ __forceinline__ void begin(int row0, int end)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rows = min(ROWS, end - row0);
        buf ^= 1;
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const v4i r = make_rsrc(src[m].p + p * src[m].plane + (int64_t)row0 * src[m].s.t,
                                        2u * ((unsigned)(rows - 1) * (unsigned)src[m].s.t + (unsigned)cols));
#pragma unroll
                for (int i = 0; i < PW; ++i)
                    if (N % NW == 0 || wave + NW * i < N) dma16(r, off[m][i], lds + (M * buf + m) * TILE + p * PLANE + (wave + NW * i) * 1024);
            }
    }
    __device__ __forceinline__ void ready()
    {
        dma_barrier();
        now = buf;
    }
    __device__ __forceinline__ int at(int m) const { return (M * now + m) * (TILE / 2); }      // the readable tile, in elements
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

struct AttentionArgs {
    const void *q, *k, *v, *o, *go;
    void *out, *gq, *gk, *gv;
    float *lse, *stats;         // stats: two values per row, from the queries kernel for the keys kernel
    const int32_t* lens;
    Source fq, fk, fv, fgo;     // as the feed reads them
    int vec;                    // rows of the tensors may be read 16 bytes at a time
    Strides qs, ks, vs, os, gos, gqs, gks, gvs;
    int batch, kv_heads, group, q_len, kv_len, dim, causal;
    int q_pad;                  // rows form, gradient of the queries: a head's rows in the grid
    float scale;
    int blocks;                 // blocks of rows (or keys) per sample and key head
    int splits;                 // parts of the other axis
    int vec_out;                // results may be stored four values at a time (bit 0: out / gq)
    float *part, *part_lse;     // splits > 1: results of the parts
};

// The part of the grid that a workgroup works on.  Workgroups go round-robin over the eight XCDs; the blocks that read the same keys
// go to one of them, so that they share an L2.  Samples of different lengths (lens) go to all of them: heads one by one instead of
// runs of heads, which would be runs of samples.  Under `causal` blocks differ in length by up to their number: the longest (number
// 0) go first, or, where the whole grid runs at once, the longest next to the shortest; with lens too, an XCD then has blocks of
// every head, of which the resident ones that read the same keys are few but run side by side.
struct Place {
    int bh, split, block;
};
__device__ __forceinline__ Place place_of(const AttentionArgs& a)
{
    const int total = gridDim.x, per = total >> 3, bhs = a.batch * a.kv_heads;
    int id = blockIdx.x;
    Place p;
    if (a.causal) {
        if (a.lens) {
            p.split = id % a.splits;
            id /= a.splits;
            p.block = id / bhs;
            p.bh = (int)(((int64_t)id + p.block) % bhs);
        } else {
            const bool whole = (bhs & 7) == 0;
            const int local = whole ? bhs >> 3 : bhs;
            if (whole) id >>= 3;
            p.split = id % a.splits;
            id /= a.splits;
            p.bh = id % local + (whole ? (int)(blockIdx.x & 7) * local : 0);
            p.block = id / local;
        }
        // all resident at once, two per compute unit: a long one and a short one each
        if (total <= 512 && 2 * p.block >= a.blocks) p.block = a.blocks - 1 - (p.block - a.blocks / 2 - (a.blocks & 1));
        return p;
    }
    if (a.lens) {
        const int units = bhs * a.splits, whole = (units & ~7) * a.blocks;
        int unit;
        if (id < whole) {
            const int local = id >> 3, turn = local / a.blocks;
            unit = turn * 8 + (id & 7);
            p.block = local - turn * a.blocks;
        } else {
            id -= whole;
            unit = (units & ~7) + id / a.blocks;
            p.block = id % a.blocks;
        }
        p.split = unit / bhs;
        p.bh = unit - p.split * bhs;
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

// A part of what a workgroup has to go through (keys that its rows see, tiles of queries that see its keys), in whole units: equal
// parts of each workgroup's own, which differ under `causal` and between samples.
struct Part {
    int64_t beg, end;
};
__device__ __forceinline__ Part part_of(int64_t all, int unit, int split, int splits)
{
    const int64_t units = (all + unit - 1) / unit;
    auto upto = [&](int s) { return min((units * s + splits - 1) / splits * unit, all); };      // (the first part has the first unit)
    return {upto(split), upto(split + 1)};
}

// A block of 32 NW rows of the heads of a group, one head after the other, each with q_pad rows: q_len, or, where that costs little,
// whole blocks, so that a block has one head's rows.  Under `causal` the blocks of the most keys come first, of all heads.
struct RowBlock {
    RowRange range;
    int i, g, end;              // the lane's query and head of the group, and the keys that it sees; clamped to those that exist
    bool in;
};
template <int NW>
__device__ __forceinline__ RowBlock row_block(const AttentionArgs& a, int n, int number, int wave, int l32)
{
    RowBlock b;
    if (a.causal) {
        const int per = a.q_pad / (32 * NW);
        number = a.q_pad % (32 * NW) ? a.blocks - 1 - number : (number % a.group + 1) * per - 1 - number / a.group;
    }
    const int all = a.group * a.q_pad, first = number * 32 * NW, last = min(first + 32 * NW, all) - 1;
    auto real = [&](int r) {
        const int g = r / a.q_pad;
        return g * a.q_len + min(r - g * a.q_pad, a.q_len - 1);
    };
    b.range = visible(a, n, real(first), real(last));
    const int r = first + 32 * wave + l32, rc = min(r, all - 1);
    b.g = rc / a.q_pad;
    const int i = rc - b.g * a.q_pad;
    b.i = min(i, a.q_len - 1);
    b.in = r < all && i < a.q_len;
    b.end = a.causal ? max(0, min(n, b.i + n - a.q_len + 1)) : n;
    return b;
}

// A tensor and where its planes go: [plane][batch * heads][len][cols], cols = dim rounded up to 8.
struct Pack {
    const void* src;
    Strides s;
    __bf16* dst;
    int heads, len, by_lens;    // by_lens: rows past a sample's keys are not needed
};
struct PackArgs {
    Pack m[4];
    int count, batch, kv_len, dim;
    const int32_t* lens;
};
inline Source packed_source(const Pack& p, int64_t batch, int64_t dim)
{
    const Strides s = packed_strides(p.heads, p.len, dim);
    return Source{p.dst, s, batch * s.b};
}
int launch_pack(const PackArgs& a, int type, hipStream_t s);
int launch_attention(const AttentionArgs& a, int type, const AttentionPlan& p, hipStream_t s);
int launch_attention_backward(const AttentionArgs& a, int type, const AttentionPlan& p, float* part_q, float* part_kv, hipStream_t s);

}  // namespace fpq
