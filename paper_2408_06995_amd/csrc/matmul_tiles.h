// The tiles of a product's kernels, and their launch: what the instantiations share.
#pragma once
#include "matmul.h"

namespace fpq {

// Tiles: results and wavefronts of a workgroup.
enum MatmulTile : int { kTile256 = 0, kTile128 = 1, kTile32 = 2 };
constexpr int kTileM[3] = {256, 128, 32}, kTileN[3] = {256, 128, 256};

template <bool COLA, bool COLB, int BM, int BN, int WM, int WN, int END>
int launch_matmul_tile(const MatmulArgs& p, hipStream_t s)
{
    static std::atomic<uint64_t> done{0};
    constexpr int bytes = 2 * (BM + BN) * 128;
    const auto kernel = matmul_kernel<COLA, COLB, BM, BN, WM, WN, END>;
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes, done)) return FPQ_ERR_LAUNCH;
    kernel<<<dim3((unsigned)((int64_t)p.tiles_m * p.tiles_n * p.slices)), dim3(64 * WM * WN), bytes, s>>>(p);
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

template <bool COLA, bool COLB, int END>
int launch_matmul_form(const MatmulArgs& p, int tile, hipStream_t s)
{
    if (tile == kTile256) return launch_matmul_tile<COLA, COLB, 256, 256, 2, 4, END>(p, s);
    if constexpr (!COLA)
        if (tile == kTile32) return launch_matmul_tile<COLA, COLB, 32, 256, 1, 4, END>(p, s);
    return launch_matmul_tile<COLA, COLB, 128, 128, 2, 2, END>(p, s);
}

int launch_matmul_rows(const MatmulArgs& p, int tile, hipStream_t s);
int launch_matmul_gated(const MatmulArgs& p, int tile, hipStream_t s);
int launch_matmul_rows_cols(const MatmulArgs& p, int tile, hipStream_t s);
int launch_matmul_cols(const MatmulArgs& p, int tile, hipStream_t s);

}  // namespace fpq
