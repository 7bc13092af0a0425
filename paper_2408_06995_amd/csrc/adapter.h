// Low-rank adapters of many requests beside a shared projection, and their gradients: what the kernels share.
//
//   t_m = A_a x_m,  y_m = base_m + s_a B_a t_m          for the rows m of a request with adapter a
//   dt_m = s_a B_a^T dy_m,  dx_m = base_m + A_a^T dt_m,  dA_a = sum_m dt_m x_m^T,  dB_a = s_a sum_m dy_m t_m^T
//
// Products are 16 x 16 x 32 steps of the bf16 matrix instruction with fp32 sums on operands split into planes as in attention.h: x and
// the gradients of fp32 activations and fp32 weights three planes, bf16 ones their own, t and dt always three, so that nothing is
// rounded below 24 bits before a result.  Lane 16 g + r: A holds row r, B column r, each the k-places 8 g .. 8 g + 7; C holds
// column r and rows 4 g .. 4 g + 3.
//
// All of it is bound by the rows read and written (32 rows of the largest listed shapes: 16 to 64 flops per byte); the adapters
// themselves come from the caches.  Rows are cut into tiles that end with their request, so that a workgroup sees one adapter;
// which tile a workgroup has it finds by a scan of the requests' lengths, 64 at a time.
#pragma once
#include "attention.h"

namespace fpq {

constexpr int kTile = 32;          // rows of a tile
constexpr int kMaxRank = 128;

struct AdapterArgs {
    const void *x, *a, *b, *base, *gy, *gx_base;
    void *y, *gx;
    const float *scaling;
    const int32_t *row_start, *adapter;
    float *t, *t_part;              // t_part: parts of t over K, or null
    const float *t_in;
    float *dt, *ga, *gb, *part_a, *part_b;
    int64_t ldx, ld_base, ldy, ld_gy, ld_gx_base, ld_gx;
    int M, N, K, R, requests, adapters;
    int parts, steps_per_part;      // of t over K
    int columns;                    // of a workgroup that writes rows
    int splits;                     // of the rows in the gradients of the adapters
    int vec_r;                      // rows along the rank may be read 16 bytes at a time (t and the weights)
    int vec_a;                      // the weights [rank, K] along K
    int vec_y;                      // rows of results and their bases, four values at a time
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

// Operand columns from a wavefront's view of a tile in LDS: lane (g, r) gets column c0 + r of rows r0 + 8 g .. + 7.
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
__device__ __forceinline__ Rows rows_of(const AdapterArgs& p, int v)
{
    Rows r = {0, 0, -1};
    if (v <= p.requests + 1) {
        const int lo = v > 0 ? p.row_start[v - 1] : 0, hi = v <= p.requests ? p.row_start[v] : p.M;
        r.lo = min(max(lo, 0), p.M);
        r.hi = max(min(hi, p.M), r.lo);
        if (v > 0 && v <= p.requests) r.adapter = p.adapter[v - 1];
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

// Tile number `tile` of all rows: its rows and adapter; lo == hi when there is no such tile.  The same for all lanes.
__device__ __forceinline__ Rows find_tile(const AdapterArgs& p, int tile)
{
    for (int v0 = 0; v0 < p.requests + 2; v0 += 64) {
        const Rows r = rows_of(p, v0 + (threadIdx.x & 63));
        const int tiles = (r.hi - r.lo + kTile - 1) / kTile, upto = scan64(tiles);
        const uint64_t past = __ballot(upto > tile);
        if (past) {
            const int who = __ffsll((unsigned long long)past) - 1;
            Rows f;
            const int first = __shfl(upto - tiles, who);
            f.hi = __shfl(r.hi, who);
            f.lo = __shfl(r.lo, who) + (tile - first) * kTile;
            f.hi = min(f.hi, f.lo + kTile);
            f.adapter = __shfl(r.adapter, who);
            f.lo = __builtin_amdgcn_readfirstlane(f.lo);
            f.hi = __builtin_amdgcn_readfirstlane(f.hi);
            f.adapter = __builtin_amdgcn_readfirstlane(f.adapter);
            return f;
        }
        tile -= __shfl(upto, 63);
    }
    return Rows{0, 0, -1};
}

static inline int64_t tiles_of(int64_t rows, int64_t requests) { return rows / kTile + requests + 2; }

// Sizes only; the same for the workspace.
struct AdapterPlan {
    int parts, steps_per_part;      // of t over K
    int columns_y, columns_x;       // columns of a workgroup that writes y, or dx
    int splits;
};
AdapterPlan plan_adapter(int64_t M, int64_t N, int64_t K, int64_t R, int64_t requests, int64_t adapters);

int launch_adapter_apply(const AdapterArgs& a, int x_type, int w_type, bool vec_k, const AdapterPlan& plan, hipStream_t s);
int launch_adapter_backward(const AdapterArgs& a, int x_type, int w_type, bool vec_n, bool vec_k, const AdapterPlan& plan, hipStream_t s);

}  // namespace fpq
