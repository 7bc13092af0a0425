// The tiles of a product's kernels, and their launch: what the instantiations share.
#pragma once
#include "matmul.h"

namespace fpq {

// Tiles: results of a workgroup.
enum MatmulTile : int { kTile256 = 0, kTile192 = 1, kTile128 = 2, kTile128Deep = 3, kTile32 = 4, kPlanes256 = 5, kPlanes128 = 6, kTile64 = 7 };
constexpr int kTileM[8] = {256, 192, 128, 128, 32, 256, 128, 64};
// (columns; of gated projections values and gates together)
constexpr int tile_n(int tile, bool gated) { return tile == kTile64 ? (gated ? 128 : 64) : tile <= kTile192 || tile == kTile32 ? 256 : 128; }

template <int KS, int PL>
void set_steps(MatmulArgs& p)
{
    p.steps = p.K ? (p.K + KS - 1) / KS : 1;
    if (PL == 3) p.passes = 1, p.order_a = p.order_b = 0;
    p.total = p.K ? p.steps * p.passes : 0;             // (nothing to sum over: zeros)
}

template <bool COLA, bool COLB, int BM, int BN, int WM, int WN, int KS, int STAGES, int PL, int END>
int launch_matmul_tile(MatmulArgs p, hipStream_t s)
{
    set_steps<KS, PL>(p);
    static std::atomic<uint64_t> done{0};
    constexpr int bytes = STAGES * PL * (BM + BN) * 2 * KS;
    const auto kernel = matmul_kernel<COLA, COLB, BM, BN, WM, WN, KS, STAGES, PL, END>;
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes, done)) return FPQ_ERR_LAUNCH;
    kernel<<<dim3((unsigned)((int64_t)p.tiles_m * p.tiles_n * p.slices)), dim3(64 * WM * WN), bytes, s>>>(p);
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

template <int BM, int BN, int WM, int WN, int KS, int STAGES, int PL, int END>
int launch_matmul_both_tile(MatmulArgs x, MatmulArgs w, hipStream_t s)
{
    set_steps<KS, PL>(x);
    set_steps<KS, PL>(w);
    static std::atomic<uint64_t> done{0};
    constexpr int bytes = STAGES * PL * (BM + BN) * 2 * KS;
    const auto kernel = matmul_both_kernel<BM, BN, WM, WN, KS, STAGES, PL, END>;
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes, done)) return FPQ_ERR_LAUNCH;
    const bool x_first = (int64_t)x.total * w.slices >= (int64_t)w.total * x.slices;
    const int nx = x.tiles_m * x.tiles_n * x.slices, nw = w.tiles_m * w.tiles_n * w.slices;
    kernel<<<dim3((unsigned)(nx + nw)), dim3(64 * WM * WN), bytes, s>>>(x, w, x_first ? nx : nw, x_first);
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

template <int END>
int launch_matmul_both_form(const MatmulArgs& x, const MatmulArgs& w, int tile, hipStream_t s)
{
    if (tile == kTile64) return launch_matmul_both_tile<64, 64, 2, 2, 64, 4, 1, END>(x, w, s);
    if (tile == kTile128Deep) return launch_matmul_both_tile<128, 128, 2, 2, 64, 4, 1, END>(x, w, s);
    if (tile == kPlanes128) return launch_matmul_both_tile<128, 128, 2, 2, 32, 3, 3, END>(x, w, s);
    return launch_matmul_both_tile<128, 128, 2, 2, 64, 2, 1, END>(x, w, s);
}

template <bool COLA, bool COLB, int END>
int launch_matmul_form(const MatmulArgs& p, int tile, hipStream_t s)
{
    // (both by rows and no gates: layers on 4-bit blocks, which have more than 64 rows here and weights of one plane)
    constexpr bool FEW_OR_PLANES = COLB || END == kGated;
    if constexpr (END != kSums)
        if (tile == kTile256) return launch_matmul_tile<COLA, COLB, 256, 256, 2, 4, 64, 2, 1, END>(p, s);
    if constexpr (!COLA) {
        if (tile == kTile192) return launch_matmul_tile<COLA, COLB, 192, 256, 2, 4, 64, 2, 1, END>(p, s);
        if constexpr (FEW_OR_PLANES)
            if (tile == kTile32) return launch_matmul_tile<COLA, COLB, 32, 256, 1, 4, 32, 4, 1, END>(p, s);
    }
    if (tile == kTile64) return launch_matmul_tile<COLA, COLB, 64, END == kGated ? 128 : 64, 2, 2, 64, 4, 1, END>(p, s);
    if (tile == kTile128Deep) return launch_matmul_tile<COLA, COLB, 128, 128, 2, 2, 64, 4, 1, END>(p, s);
    if constexpr (FEW_OR_PLANES) {
        if (tile == kPlanes256) return launch_matmul_tile<COLA, COLB, 256, 128, 4, 2, 32, 2, 3, END>(p, s);
        if (tile == kPlanes128) return launch_matmul_tile<COLA, COLB, 128, 128, 2, 2, 32, 3, 3, END>(p, s);
    }
    return launch_matmul_tile<COLA, COLB, 128, 128, 2, 2, 64, 2, 1, END>(p, s);
}

int launch_matmul_rows(const MatmulArgs& p, int tile, hipStream_t s);
int launch_matmul_gated(const MatmulArgs& p, int tile, hipStream_t s);
int launch_matmul_rows_cols(const MatmulArgs& p, int tile, hipStream_t s);
int launch_matmul_cols(const MatmulArgs& p, int tile, hipStream_t s);
int launch_matmul_cols_sums(const MatmulArgs& p, int tile, hipStream_t s);
int launch_matmul_both(const MatmulArgs& x, const MatmulArgs& w, int tile, hipStream_t s);
int launch_matmul_both_sums(const MatmulArgs& x, const MatmulArgs& w, int tile, hipStream_t s);

}  // namespace fpq
