// Layers on 4-bit blocks for single tokens: one or two rows in bf16, up to four in fp32.
//
// Bound by the codes' bytes: every code is read once, 1 KB of a row at a time (a lane has a block of 32 codes, 16 bytes, and its scale), and a
// wavefront's loads for four rows of weights go out together.  x is in LDS, in the order in which the lanes read it: piece i of 16 bytes of
// all lanes' blocks lie side by side.  bf16: codes become pairs of bf16 in the conversion instruction and are summed by the two-element dot
// product; fp32: pairs of fp32 and fused multiply-adds.  The conversion takes the scale too: a block's sum without it could leave the range where
// the products do not.  5120 -> 20480: one row 12.3 us in bf16 (4.5 TB/s
// with the launch), on the matrix unit 22.9; two rows 18.3 and 23.3, three 20.5 and 24.1 (but 5120 -> 5120 9.5 and 8.6); in fp32 one row 16.5 and 31.2, four the same.
#include "rows.h"

namespace fpq {

namespace {

constexpr int kTokenRows = 4;           // rows of weights of a wavefront

template <typename T, int M>
__global__ __launch_bounds__(256) void token_blocks_kernel(RowsArgs a)
{
    constexpr int P = 4 * (int)sizeof(T) / 2, E = 16 / (int)sizeof(T), R = kTokenRows;      // pieces of a block, elements of a piece
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int blocks = (a.K + 31) / 32, chunks = (blocks + 63) / 64;
    uint4* const room = reinterpret_cast<uint4*>(lds);
    const int n0 = (blockIdx.x * 4 + wave) * R;

    const uint8_t *w[R], *sc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t n = min(n0 + r, a.N - 1);
        w[r] = static_cast<const uint8_t*>(a.w) + n * a.ld_w;
        sc[r] = a.scales + n * a.ld_s;
    }
    uint4 code[R];
    uint32_t scale[R];
    auto load = [&](int c) {
        const int b = min(c * 64 + lane, blocks - 1);                 // (x is zero behind the row)
#pragma unroll
        for (int r = 0; r < R; ++r) code[r] = *reinterpret_cast<const uint4*>(w[r] + 16 * b);
#pragma unroll
        for (int r = 0; r < R; ++r) scale[r] = sc[r][b];
    };
    load(0);

    // x to LDS: [m][chunk][piece][lane]
    const int pieces = chunks * 64 * P;
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const T* const x = static_cast<const T*>(a.x) + m * a.ld_x;
        for (int i = threadIdx.x; i < pieces; i += 256) {
            const int k = i * E, b = i / P, c = b >> 6, l = b & 63;
            uint4 v;
            if (k + E <= a.K) {
                v = __builtin_bit_cast(uint4, *reinterpret_cast<const piece16*>(x + k));
            } else {
                T e[E];
#pragma unroll
                for (int j = 0; j < E; ++j) e[j] = k + j < a.K ? x[k + j] : (T)0.0f;
                __builtin_memcpy(&v, e, 16);
            }
            room[((m * chunks + c) * P + i % P) * 64 + l] = v;
        }
    }
    __syncthreads();

    float acc[R][M];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m) acc[r][m] = 0.0f;
    for (int c = 0; c < chunks; ++c) {
        uint4 now[R];
        float f[R];
        const bool in = c * 64 + lane < blocks;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            now[r] = code[r];
            f[r] = in ? scale_of(scale[r]) : 1.0f;
        }
        if (c + 1 < chunks) load(c + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {                                 // eight codes of the block
            uint4 x[M][P / 4];
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int j = 0; j < P / 4; ++j) x[m][j] = room[((m * chunks + c) * P + i * (P / 4) + j) * 64 + lane];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const uint32_t q = i == 0 ? now[r].x : i == 1 ? now[r].y : i == 2 ? now[r].z : now[r].w;
                auto pair = [&](auto byte) {
                    constexpr int B = decltype(byte)::value;
                    if constexpr (sizeof(T) == 2) {
                        const v2bf v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, f[r], B);
#pragma unroll
                        for (int m = 0; m < M; ++m) {
                            const uint32_t u = B == 0 ? x[m][0].x : B == 1 ? x[m][0].y : B == 2 ? x[m][0].z : x[m][0].w;
                            acc[r][m] = __builtin_amdgcn_fdot2_f32_bf16(v, __builtin_bit_cast(v2bf, u), acc[r][m], false);
                        }
                    } else {
                        const v2f v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, f[r], B);
#pragma unroll
                        for (int m = 0; m < M; ++m) {
                            const uint4 u = x[m][B / 2];
                            acc[r][m] = fmaf(v.x, __uint_as_float(B % 2 ? u.z : u.x), acc[r][m]);
                            acc[r][m] = fmaf(v.y, __uint_as_float(B % 2 ? u.w : u.y), acc[r][m]);
                        }
                    }
                };
                pair(std::integral_constant<int, 0>());
                pair(std::integral_constant<int, 1>());
                pair(std::integral_constant<int, 2>());
                pair(std::integral_constant<int, 3>());
            }
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int m = 0; m < M; ++m) acc[r][m] += __shfl_xor(acc[r][m], off, 64);
    // lane r + R m stores result (m, n0 + r)
    float v = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m) v = lane == r + R * m ? acc[r][m] : v;
    const int n = n0 + (lane & (R - 1)), m = lane / R;
    if (lane < R * M && n < a.N) static_cast<T*>(a.out)[m * a.ld_out + n] = (T)(v + (a.bias ? a.bias[n] : 0.0f));
}

template <typename T, int M>
int launch(const RowsArgs& a, hipStream_t s)
{
    const int bytes = (int)token_blocks_lds(M, a.K, a.f32);
    token_blocks_kernel<T, M><<<dim3((unsigned)((a.N + 4 * kTokenRows - 1) / (4 * kTokenRows))), dim3(256), bytes, s>>>(a);
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

}  // namespace

int launch_token_blocks(const RowsArgs& a, hipStream_t s)
{
    if (!a.f32) return a.M == 1 ? launch<__bf16, 1>(a, s) : launch<__bf16, 2>(a, s);
    switch (a.M) {
    case 1: return launch<float, 1>(a, s);
    case 2: return launch<float, 2>(a, s);
    case 3: return launch<float, 3>(a, s);
    default: return launch<float, 4>(a, s);
    }
}

}  // namespace fpq
