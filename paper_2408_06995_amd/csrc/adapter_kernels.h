// The adapters' kernels (see adapter.h).  Three shapes of work:
//   shrink   rows x weights over a long axis -> [rows, rank]:   t (weights [rank, K]), dt (weights [N, rank])
//   expand   [rows, rank] x weights -> rows of a long axis:     y (weights [N, rank]), dx (weights [rank, K])
//   outer    columns of rows x [rows, rank], over the rows:     dA, dB
// Weights whose contraction runs along their rows are read as operands from memory as they lie; the other two (dt, dx) pass through
// a wavefront's own LDS tile and the transposing read.
#pragma once
#include "adapter.h"

namespace fpq {

// Eight values along the rank, zero from R on; the branch is the same for all lanes of a launch.
template <typename T>
__device__ __forceinline__ void rank8(const T* row, int col, int R, int vec, float (&v)[8])
{
    if (vec)
        row8<T, true>(row, col, R, v);
    else
        row8<T, false>(row, col, R, v);
}

// This wavefront's tile of ROWS rows from a matrix in memory: rows from `rows` on and columns from `cols` on become zero.
template <typename T, int ROWS, int COLS, int RS>
__device__ __forceinline__ void stage_wave(__bf16* tile, const T* base, int64_t stride, int rows, int cols, bool vec, int lane)
{
    constexpr int NP = kPlanes<T>, CH = COLS / 8, N = ROWS * CH, PT = (N + 63) / 64;
    float v[PT][8];
#pragma unroll
    for (int it = 0; it < PT; ++it) {
        const int id = it * 64 + lane, row = id / CH, c = (id - row * CH) * 8;
        const T* at = base + (int64_t)min(row, rows - 1) * stride;
        if (vec)
            row8<T, true>(at, c, cols, v[it]);
        else
            row8<T, false>(at, c, cols, v[it]);
    }
#pragma unroll
    for (int it = 0; it < PT; ++it) {
        const int id = it * 64 + lane, row = id / CH, c = (id - row * CH) * 8;
        if (N % 64 != 0 && id >= N) continue;
        if (row >= rows) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[it][e] = 0.0f;
        }
        const Frag<NP> f = frag_of<NP>(v[it]);
#pragma unroll
        for (int p = 0; p < NP; ++p) *reinterpret_cast<v8bf*>(tile + (p * ROWS + row) * RS + c) = f.p[p];
    }
}

// A wavefront's own LDS writes ahead of its reads, and its reads ahead of the next writes.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// TRANS false: weights [adapters][R][L] (t from x, L = K); true: [adapters][L][R] (dt from dy, L = N, scaled).
// A workgroup takes one tile of rows and, of its part of L, its four wavefronts steps of 32 in turn.
template <typename TX, typename TW, int RT, bool VEC, bool TRANS>
__global__ __launch_bounds__(256) void adapter_shrink_kernel(AdapterArgs p)
{
    constexpr int NX = kPlanes<TX>, NW = kPlanes<TW>, RP = 16 * RT + 4, RS = 16 * RT + 8;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const Rows rows = find_tile(p, blockIdx.x);
    if (rows.lo >= rows.hi) return;
    const int L = TRANS ? p.N : p.K, R = p.R, count = rows.hi - rows.lo;
    const int64_t ld = TRANS ? p.ld_gy : p.ldx;
    float* const out = p.t_part ? p.t_part + (size_t)blockIdx.y * p.M * R : TRANS ? p.dt : p.t;
    if (rows.adapter < 0) {
        for (int id = threadIdx.x; id < count * R; id += 256) out[(size_t)rows.lo * R + id] = 0.0f;
        return;
    }
    const TX* const x = static_cast<const TX*>(TRANS ? p.gy : p.x) + (int64_t)rows.lo * ld;
    const TW* const w = static_cast<const TW*>(TRANS ? p.b : p.a) + (size_t)rows.adapter * R * L;
    __bf16* const tile = reinterpret_cast<__bf16*>(lds) + wave * NW * 32 * RS;      // TRANS
    v4f acc[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int m = 0; m < 2; ++m) acc[r][m] = v4f{0, 0, 0, 0};
    const int steps = (L + 31) / 32, beg = TRANS ? 0 : min((int)blockIdx.y * p.steps_per_part, steps), end = TRANS ? steps : min(beg + p.steps_per_part, steps);
    const TX* const x0 = x + (int64_t)min(r16, count - 1) * ld;
    const TX* const x1 = x + (int64_t)min(r16 + 16, count - 1) * ld;
    const bool both = count > 16;
    for (int s = beg + wave; s < end; s += 4) {
        const int col = 32 * s + 8 * g;
        float v[8];
        Frag<NX> xf[2];
        row8<TX, VEC>(x0, col, L, v);
        xf[0] = frag_of<NX>(v);
        if (both) {
            row8<TX, VEC>(x1, col, L, v);
            xf[1] = frag_of<NX>(v);
        }
        if (TRANS) {
            wave_sync();
            stage_wave<TW, 32, 16 * RT, RS>(tile, w + (size_t)32 * s * R, R, min(32, L - 32 * s), R, p.vec_r, lane);
            wave_sync();
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            Frag<NW> wf;
            if constexpr (TRANS) {
                wf = col_frag16<NW>(tile, RS, 32 * RS, 0, 16 * r, lane);
            } else {
                const int row = 16 * r + r16;
                row8<TW, VEC>(w + (size_t)min(row, R - 1) * L, col, L, v);
                wf = frag_of<NW>(v);
            }
            mma16<NW, NX>(acc[r][0], wf, xf[0]);
            if (both) mma16<NW, NX>(acc[r][1], wf, xf[1]);
        }
    }
    // the four sums of a value, in order: [wave][row][rank]
    float* const sums = reinterpret_cast<float*>(lds);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int m = 0; m < 2; ++m)
            *reinterpret_cast<v4f*>(sums + (wave * kTile + 16 * m + r16) * RP + 16 * r + 4 * g) = acc[r][m];
    __syncthreads();
    const float scale = TRANS ? p.scaling[rows.adapter] : 1.0f;
    for (int id = threadIdx.x; id < count * 16 * RT; id += 256) {
        const int m = id / (16 * RT), r = id - m * 16 * RT;
        if (r >= R) continue;
        const float* at = sums + m * RP + r;
        out[(size_t)(rows.lo + m) * R + r] = scale * (((at[0] + at[kTile * RP]) + at[2 * kTile * RP]) + at[3 * kTile * RP]);
    }
}

// TRANS false: weights [adapters][L][R] (y from t, scaled, L = N); true: [adapters][R][L] (dx from dt, L = K).
// A workgroup takes a tile of rows and p.columns columns, its wavefronts 32 columns at a time.
template <typename TX, typename TW, int RT, bool TRANS>
__global__ __launch_bounds__(256) void adapter_expand_kernel(AdapterArgs p)
{
    constexpr int NW = kPlanes<TW>, RK = (RT + 1) / 2, RS = 32 + 8, ROWS = 32 * RK;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const Rows rows = find_tile(p, blockIdx.x);
    if (rows.lo >= rows.hi) return;
    const int L = TRANS ? p.K : p.N, R = p.R, count = rows.hi - rows.lo;
    const int cbeg = blockIdx.y * p.columns, cend = min(cbeg + p.columns, L);
    const TX* const base = static_cast<const TX*>(TRANS ? p.gx_base : p.base);
    TX* const y = static_cast<TX*>(TRANS ? p.gx : p.y);
    const int64_t ldb = TRANS ? p.ld_gx_base : p.ld_base, ldy = TRANS ? p.ld_gx : p.ldy;
    __bf16* const tile = reinterpret_cast<__bf16*>(lds) + wave * NW * ROWS * RS;    // TRANS
    const bool some = rows.adapter >= 0, both = count > 16;

    Frag<3> tf[2][RK];
    const float scale = some && !TRANS ? p.scaling[rows.adapter] : 1.0f;
    if (some) {
        const float* const t = TRANS ? p.dt : p.t_part ? p.t_part : p.t;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int k = 0; k < RK; ++k) {
                const int row = min(16 * m + r16, count - 1);
                float v[8], u[8];
                rank8(t + (size_t)(rows.lo + row) * R, 32 * k + 8 * g, R, p.vec_r, v);
                if (!TRANS && p.t_part) {
                    for (int s = 1; s < p.parts; ++s) {
                        rank8(t + ((size_t)s * p.M + rows.lo + row) * R, 32 * k + 8 * g, R, p.vec_r, u);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += u[e];
                    }
                    if (blockIdx.y == 0 && wave == 0 && p.t && 16 * m + r16 < count) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (32 * k + 8 * g + e < R) p.t[(size_t)(rows.lo + row) * R + 32 * k + 8 * g + e] = v[e];
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= scale;
                tf[m][k] = frag_of<3>(v);
            }
    } else if (!TRANS && p.t_part && p.t && blockIdx.y == 0) {
        for (int id = threadIdx.x; id < count * R; id += 256) p.t[(size_t)rows.lo * R + id] = 0.0f;
    }
    const TW* const w = static_cast<const TW*>(TRANS ? p.a : p.b) + (size_t)max(rows.adapter, 0) * R * L;
    for (int c0 = cbeg + 32 * wave; c0 < cend; c0 += 128) {
        float have[2][2][4];       // of the base: [columns][rows]
        const bool left = c0 + 16 < cend;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int e = 0; e < 4; ++e) have[c][m][e] = 0.0f;
                const int row = min(16 * m + r16, count - 1), col = c0 + 16 * c + 4 * g;
                if (base && (m == 0 || both) && (c == 0 || left)) {
                    const TX* at = base + (int64_t)(rows.lo + row) * ldb;
                    if (p.vec_y) {
                        if (col < L) {
                            if constexpr (sizeof(TX) == 4) {
                                const float4 f = *reinterpret_cast<const float4*>(at + col);
                                have[c][m][0] = f.x; have[c][m][1] = f.y; have[c][m][2] = f.z; have[c][m][3] = f.w;
                            } else {
                                const uint2 f = *reinterpret_cast<const uint2*>(at + col);
                                have[c][m][0] = __uint_as_float(f.x << 16); have[c][m][1] = __uint_as_float(f.x & 0xffff0000u);
                                have[c][m][2] = __uint_as_float(f.y << 16); have[c][m][3] = __uint_as_float(f.y & 0xffff0000u);
                            }
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) have[c][m][e] = col + e < L ? (float)at[col + e] : 0.0f;
                    }
                }
            }
        v4f acc[2][2];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int m = 0; m < 2; ++m) acc[c][m] = v4f{0, 0, 0, 0};
        if (some) {
            if (TRANS) {
                wave_sync();
                stage_wave<TW, ROWS, 32, RS>(tile, w + c0, L, R, L - c0, p.vec_a, lane);
                wave_sync();
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (c == 1 && !left) continue;
#pragma unroll
                for (int k = 0; k < RK; ++k) {
                    Frag<NW> wf;
                    if constexpr (TRANS) {
                        wf = col_frag16<NW>(tile, RS, ROWS * RS, 32 * k, 16 * c, lane);
                    } else {
                        float v[8];
                        rank8(w + (size_t)min(c0 + 16 * c + r16, L - 1) * R, 32 * k + 8 * g, R, p.vec_r, v);
                        wf = frag_of<NW>(v);
                    }
                    mma16<NW, 3>(acc[c][0], wf, tf[0][k]);
                    if (both) mma16<NW, 3>(acc[c][1], wf, tf[1][k]);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int row = 16 * m + r16, col = c0 + 16 * c + 4 * g;
                if (row >= count || (c == 1 && !left)) continue;
                const float v[4] = {have[c][m][0] + acc[c][m][0], have[c][m][1] + acc[c][m][1], have[c][m][2] + acc[c][m][2],
                                    have[c][m][3] + acc[c][m][3]};
                store4(y + (int64_t)(rows.lo + row) * ldy, col, L, p.vec_y, v);
            }
    }
}

constexpr int kListed = 512;        // requests that a workgroup looks over at a time

// B false: dA[a][r][k] from dt and x; true: dB[a][n][r] from dy and t, scaled.
// A workgroup has 128 columns of one adapter's rows; of the adapter's tiles of 32 rows it takes its share of p.splits.
template <typename TX, int RT, bool VEC, bool B>
__global__ __launch_bounds__(256) void adapter_outer_kernel(AdapterArgs p)
{
    constexpr int NX = kPlanes<TX>, CS = kRowStride<8>, RS = kRowStride<RT>;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    __bf16* const xt = reinterpret_cast<__bf16*>(lds);                   // [NX][32][CS]
    __bf16* const tt = xt + NX * 32 * CS;                                // [3][32][RS]
    int* const upto = reinterpret_cast<int*>(tt + 3 * 32 * RS);          // [kListed + 1] tiles ahead of a request, [kListed] first rows
    int* const first = upto + kListed + 1;
    int* const wsum = first + kListed;                                   // [8]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, g = lane >> 4;
    const int L = B ? p.N : p.K, R = p.R, c0 = blockIdx.x * 128, adapter = blockIdx.y, split = blockIdx.z;
    const TX* const x = static_cast<const TX*>(B ? p.gy : p.x) + c0;
    const int64_t ld = B ? p.ld_gy : p.ldx;
    const float* const t = B ? p.t_in : p.dt;
    v4f acc[2][RT];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[c][r] = v4f{0, 0, 0, 0};
    Stage<TX, 8, VEC, 32, 256> sx;
    Stage<float, RT, true, 32, 256> sv;
    Stage<float, RT, false, 32, 256> ss;
    for (int q0 = 1; q0 <= p.requests; q0 += kListed) {
        __syncthreads();
        int before = 0;                              // tiles of this adapter in the requests listed so far
        for (int part = 0; part < kListed; part += 256) {
            const int v = q0 + part + tid;
            Rows r = {0, 0, -1};
            if (v <= p.requests) r = rows_of(p, v);
            const int tiles = r.adapter == adapter ? (r.hi - r.lo + kTile - 1) / kTile : 0, sum = scan64(tiles);
            if (lane == 63) wsum[wave] = sum;
            __syncthreads();
            int ahead = before + sum - tiles;
            for (int w = 0; w < 4; ++w) {
                if (w < wave) ahead += wsum[w];
                before += wsum[w];
            }
            upto[part + tid] = ahead;
            first[part + tid] = r.lo;
            __syncthreads();
        }
        if (tid == 0) upto[kListed] = before;
        __syncthreads();
        const int tbeg = (int)((int64_t)before * split / p.splits), tend = (int)((int64_t)before * (split + 1) / p.splits);
        int lo = 0, hi = 0;                          // of the tile last loaded
        auto load = [&](int tile) {
            int a = 0, b = kListed;                  // upto[a] <= tile < upto[b]
            while (b - a > 1) {
                const int m = (a + b) >> 1;
                if (upto[m] <= tile)
                    a = m;
                else
                    b = m;
            }
            const Rows r = rows_of(p, q0 + a);
            lo = first[a] + (tile - upto[a]) * kTile;
            hi = min(r.hi, lo + kTile);
            sx.load(x, ld, lo, hi - 1, L - c0, tid);
            if (p.vec_r)
                sv.load(t, R, lo, hi - 1, R, tid);
            else
                ss.load(t, R, lo, hi - 1, R, tid);
        };
        if (tbeg < tend) load(tbeg);
        for (int tile = tbeg; tile < tend; ++tile) {
            __syncthreads();
            sx.store(xt, lo, hi, L - c0, tid);
            if (p.vec_r)
                sv.store(tt, lo, hi, R, tid);
            else
                ss.store(tt, lo, hi, R, tid);
            __syncthreads();
            if (tile + 1 < tend) load(tile + 1);
            Frag<NX> xf[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) xf[c] = col_frag16<NX>(xt, CS, 32 * CS, 0, 32 * wave + 16 * c, lane);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const Frag<3> tf = col_frag16<3>(tt, RS, 32 * RS, 0, 16 * r, lane);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if constexpr (B)
                        mma16<NX, 3>(acc[c][r], xf[c], tf);              // lane: rank r16, columns 4 g + i
                    else
                        mma16<3, NX>(acc[c][r], tf, xf[c]);              // lane: column r16, ranks 4 g + i
                }
            }
        }
    }
    const float scale = B ? p.scaling[adapter] : 1.0f;
    const size_t each = (size_t)p.adapters * L * R;
    float* const out = (p.splits > 1 ? (B ? p.part_b : p.part_a) + split * each : B ? p.gb : p.ga) + (size_t)adapter * L * R;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int col = c0 + 32 * wave + 16 * c + (B ? 4 * g + e : r16), rank = 16 * r + (B ? r16 : 4 * g + e);
                if (col >= L || rank >= R) continue;
                out[B ? (size_t)col * R + rank : (size_t)rank * L + col] = scale * acc[c][r][e];
            }
}

template <typename TX, typename TW, int RT, bool VEC, bool TRANS>
int launch_shrink(const AdapterArgs& a, int parts, hipStream_t s)
{
    constexpr int tile = TRANS ? 4 * kPlanes<TW> * 32 * (16 * RT + 8) * 2 : 0, sums = 4 * kTile * (16 * RT + 4) * 4, lds = tile > sums ? tile : sums;
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&adapter_shrink_kernel<TX, TW, RT, VEC, TRANS>), lds, done)) return FPQ_ERR_LAUNCH;
    adapter_shrink_kernel<TX, TW, RT, VEC, TRANS><<<dim3((unsigned)tiles_of(a.M, a.requests), parts), dim3(256), lds, s>>>(a);
    return FPQ_OK;
}

template <typename TX, typename TW, int RT, bool TRANS>
int launch_expand(AdapterArgs a, int columns, hipStream_t s)
{
    constexpr int lds = TRANS ? 4 * kPlanes<TW> * 32 * ((RT + 1) / 2) * 40 * 2 : 0;
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&adapter_expand_kernel<TX, TW, RT, TRANS>), lds, done)) return FPQ_ERR_LAUNCH;
    a.columns = columns;
    const int L = TRANS ? a.K : a.N;
    adapter_expand_kernel<TX, TW, RT, TRANS><<<dim3((unsigned)tiles_of(a.M, a.requests), (L + columns - 1) / columns), dim3(256), lds, s>>>(a);
    return FPQ_OK;
}

template <typename TX, int RT, bool VEC, bool B>
int launch_outer(const AdapterArgs& a, hipStream_t s)
{
    constexpr int lds = kPlanes<TX> * 32 * kRowStride<8> * 2 + 3 * 32 * kRowStride<RT> * 2 + (2 * kListed + 16) * 4;
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&adapter_outer_kernel<TX, RT, VEC, B>), lds, done)) return FPQ_ERR_LAUNCH;
    const int L = B ? a.N : a.K;
    adapter_outer_kernel<TX, RT, VEC, B><<<dim3((L + 127) / 128, a.adapters, a.splits), dim3(256), lds, s>>>(a);
    return FPQ_OK;
}

template <typename TX, typename TW, int RT>
int apply_of_rank(const AdapterArgs& a, bool vec_k, const AdapterPlan& plan, hipStream_t s)
{
    const int st = vec_k ? launch_shrink<TX, TW, RT, true, false>(a, plan.parts, s) : launch_shrink<TX, TW, RT, false, false>(a, plan.parts, s);
    return st != FPQ_OK ? st : launch_expand<TX, TW, RT, false>(a, plan.columns_y, s);
}

template <typename TX, typename TW>
int launch_apply(const AdapterArgs& a, bool vec_k, const AdapterPlan& plan, hipStream_t s)
{
    const int st = a.R <= 16 ? apply_of_rank<TX, TW, 1>(a, vec_k, plan, s) : a.R <= 32 ? apply_of_rank<TX, TW, 2>(a, vec_k, plan, s)
                 : a.R <= 64 ? apply_of_rank<TX, TW, 4>(a, vec_k, plan, s) : apply_of_rank<TX, TW, 8>(a, vec_k, plan, s);
    return st != FPQ_OK ? st : hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

int launch_adapter_sums(const AdapterArgs& a, hipStream_t s);

template <typename TX, typename TW, int RT>
int backward_of_rank(const AdapterArgs& a, bool vec_n, bool vec_k, const AdapterPlan& plan, hipStream_t s)
{
    int st = vec_n ? launch_shrink<TX, TW, RT, true, true>(a, 1, s) : launch_shrink<TX, TW, RT, false, true>(a, 1, s);
    if (st == FPQ_OK && a.gx) st = launch_expand<TX, TW, RT, true>(a, plan.columns_x, s);
    if (st == FPQ_OK) st = vec_k ? launch_outer<TX, RT, true, false>(a, s) : launch_outer<TX, RT, false, false>(a, s);
    if (st == FPQ_OK) st = vec_n ? launch_outer<TX, RT, true, true>(a, s) : launch_outer<TX, RT, false, true>(a, s);
    return st;
}

template <typename TX, typename TW>
int launch_backward(const AdapterArgs& a, bool vec_n, bool vec_k, const AdapterPlan& plan, hipStream_t s)
{
    int st = a.R <= 16 ? backward_of_rank<TX, TW, 1>(a, vec_n, vec_k, plan, s) : a.R <= 32 ? backward_of_rank<TX, TW, 2>(a, vec_n, vec_k, plan, s)
           : a.R <= 64 ? backward_of_rank<TX, TW, 4>(a, vec_n, vec_k, plan, s) : backward_of_rank<TX, TW, 8>(a, vec_n, vec_k, plan, s);
    if (st == FPQ_OK && a.splits > 1) st = launch_adapter_sums(a, s);
    return st != FPQ_OK ? st : hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

}  // namespace fpq
