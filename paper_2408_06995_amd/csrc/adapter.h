// Low-rank adapters of many requests beside a shared projection, and their gradients: what the kernels share.
//
//   t_m = A_a x_m,  y_m = base_m + s_a B_a t_m          for the rows m of a request with adapter a
//   dt_m = s_a B_a^T dy_m,  dx_m = base_m + A_a^T dt_m,  dA_a = sum_m dt_m x_m^T,  dB_a = s_a sum_m dy_m t_m^T
//
// Products are 16 x 16 x 32 steps of the bf16 matrix instruction with fp32 sums on operands split into planes as in attention.h: x and
// the gradients of fp32 activations and fp32 weights three planes, bf16 ones their own, t and dt always three, so that nothing is
// rounded below 24 bits before a result.  Lane 16 g + r: A holds row r, B column r, each the k-places 8 g .. 8 g + 7; C holds
// column r and rows 4 g .. 4 g + 3.  The columns of y are tiles of the 32 x 32 x 16 instruction (attention.h).
//
// All of it is bound by the rows read and written (a rank of 16 makes 8 flops per byte, one of 64 in bf16 64); the adapters
// themselves come from the caches.  Rows are cut into tiles that end with their request, so that a workgroup sees one adapter;
// which tile a workgroup has it finds by a search among the requests' first rows, 64 at a time.
#pragma once
#include "attention.h"

namespace fpq {

constexpr int kMaxRank = 128, kPlainRank = 16;     // up to kPlainRank weights are read where they are, whatever their alignment

// Weights of one contraction: [adapters][rows][cols], the contraction along the columns; or packed in the order in which the matrix
// instructions take them, 64 lanes x 8 elements at a time, zeros outside the matrix:
//   W1, steps of 32 columns:  [adapter][plane][step][group of 16 ranks][lane]: rank 16 group + lane % 16, columns 32 step + 8 (lane / 16) ..
//   W2, blocks of 32 rows:    [adapter][plane][block][step of 16 ranks][lane]: row 32 block + lane % 32, ranks 16 step + 8 (lane / 32) ..
struct Weights {
    const void* p;
    int64_t each;                   // elements of an adapter
    int64_t plane;                  // packed: elements of a plane
    int ld;                         // from one row to the next
    int vec;                        // rows may be read 16 bytes at a time
};

// One call's map of rows through a rank: t = x W1^T, y = base + t W2^T.
struct AdapterArgs {
    const void *x, *base;
    void* y;                        // null: t only
    float* t;                       // [M, R], or null
    Weights w1, w2;                 // [R, L1], [L2, R]
    const float *scale1, *scale2;   // per adapter: of t, of what enters y; null: 1
    const int32_t *row_start, *adapter;
    int64_t ldx, ld_base, ldy;
    int M, L1, L2, R, requests, adapters;
    int parts;                      // of the columns of y: the workgroups of a tile
    int vec_x;                      // rows of x, 16 bytes at a time
};

// The gradients of the adapters: out[0][a][r][k] = sum dt_m[r] x_m[k], out[1][a][n][r] = scale sum dy_m[n] t_m[r].
struct OuterArgs {
    const void* rows[2];            // x, dy
    const float* t[2];              // dt, t
    float* out[2];                  // of a part: in `part` when there are several
    const float* scaling;
    const int32_t *row_start, *adapter;
    int64_t ld[2];
    int L[2], M, R, requests, adapters, splits;
    int vec_rows[2], vec_t;
};

// c += a b over the planes whose product counts: of x = sum_i x_i with x_i about 2^-8i of x, those with i + j <= 2.
template <int NA, int NB>
__device__ __forceinline__ void mma16(v4f& c, const Frag<NA>& a, const Frag<NB>& b)
{
#pragma unroll
    for (int sum = 2; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (sum - i >= 0 && sum - i < NB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[sum - i], c, 0, 0, 0);
}

template <int NA, int NB>
__device__ __forceinline__ void mma32(v16f& c, const Frag<NA>& a, const Frag<NB>& b)
{
#pragma unroll
    for (int sum = 2; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (sum - i >= 0 && sum - i < NB) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[i], b.p[sum - i], c, 0, 0, 0);
}

// Operand columns of a tile in LDS: lane (g, r) gets column c0 + r of rows r0 + 8 g .. + 7.
template <int NP>
__device__ __forceinline__ Frag<NP> col_frag16(const __bf16* tile, int rs, int plane, int r0, int c0, int lane)
{
    const __bf16* at = tile + (r0 + 8 * (lane >> 4) + ((lane & 15) >> 2)) * rs + c0 + (lane & 3) * 4;
    Frag<NP> f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(at + p * plane));
        const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(at + p * plane + 4 * rs));
        f.p[p] = __builtin_bit_cast(v8bf, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    return f;
}

// Rows [lo, hi) of request v - 1; 0 and requests + 1 are the rows ahead of the first request and behind the last.
struct Rows {
    int lo, hi, adapter;            // adapter < 0: none
};
template <typename Args>
__device__ __forceinline__ Rows rows_of(const Args& p, int v)
{
    Rows r = {0, 0, -1};
    if (v <= p.requests + 1) {
        const int lo = v > 0 ? p.row_start[v - 1] : 0, hi = v <= p.requests ? p.row_start[v] : p.M;
        if (v > 0 && v <= p.requests) r.adapter = p.adapter[v - 1];
        r.lo = min(max(lo, 0), p.M);
        r.hi = max(min(hi, p.M), r.lo);
        if (r.adapter >= p.adapters) r.adapter = -1;
    }
    return r;
}

__device__ __forceinline__ int scan64(int v)      // inclusive sum over the lanes
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int u = __shfl_up(v, off);
        if (lane >= off) v += u;
    }
    return v;
}

// Tile number `tile` (of TM rows) of all rows: its rows and adapter; lo == hi when there is no such tile.  The same for all lanes.
// Numbers have gaps: the tiles of run v of rows start at number lo / TM + v.  Up to the next run's that is room for them, since rows
// that start and end anywhere make at most one tile more than there are multiples of TM from lo to hi; and the run of a number is the last
// that does not start past it, found with 64 guesses at a time: four reads for 2^21 requests, one for 62.
template <int TM>
__device__ __forceinline__ Rows find_tile(const AdapterArgs& p, int tile)
{
    int v0 = 0, n = p.requests + 2;                  // v0 <= the run < v0 + n
    for (;;) {
        const int step = (n + 63) / 64, at = (int)(threadIdx.x & 63) * step;
        const Rows r = rows_of(p, at < n ? v0 + at : p.requests + 2);
        const int first = r.lo / TM + v0 + at;
        const int who = 63 - __builtin_clzll(__ballot(at < n && first <= tile) | 1);
        if (step == 1) {
            Rows f;
            const int number = __shfl(first, who);
            f.hi = __shfl(r.hi, who);
            f.lo = __shfl(r.lo, who) + (tile - number) * TM;
            f.hi = min(f.hi, f.lo + TM);
            f.adapter = __shfl(r.adapter, who);
            f.lo = __builtin_amdgcn_readfirstlane(f.lo);
            f.hi = __builtin_amdgcn_readfirstlane(f.hi);
            f.adapter = __builtin_amdgcn_readfirstlane(f.adapter);
            return f;
        }
        v0 += who * step;
        n = min(step, n - who * step);
    }
}

// Sizes only; the same for the workspace.
struct AdapterPlan {
    int waves;                      // of a workgroup of the map: 4, or 16 (as many as the rank lets)
    int parts_n, parts_k;           // of the columns of y and of dx
    int splits;                     // of an adapter's rows in the gradients
};
AdapterPlan plan_adapter(int64_t M, int64_t N, int64_t K, int64_t requests, int64_t adapters);

// Both weights of a call, packed: W1 from a [adapters][R][K] and W2 from b [adapters][N][R] in the forward call, W1 from b and W2
// from a in the backward one.
struct AdapterPack {
    const void *a, *b;
    __bf16 *w1, *w2;
    int N, K, R, adapters;
    bool forward;
};
static inline int rank_groups(int64_t R) { return R <= 16 ? 1 : R <= 32 ? 2 : R <= 64 ? 4 : 8; }
static inline int64_t packed_elements(int64_t len, int64_t R) { return (len + 63) / 64 * 2 * rank_groups(R) * 512; }     // of a plane: N or K

int launch_adapter_map(const AdapterArgs& a, int x_type, int w_type, bool packed, int waves, hipStream_t s);
int launch_adapter_pack(const AdapterPack& a, int w_type, hipStream_t s);
int launch_adapter_outer(const OuterArgs& a, int x_type, hipStream_t s);
int launch_adapter_sums(const float* part_a, const float* part_b, int splits, size_t na, size_t nb, float* ga, float* gb, hipStream_t s);

}  // namespace fpq
