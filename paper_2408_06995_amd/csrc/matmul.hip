// Matrix products: the choice of tile and slices, and the sum of the slices.
#include "matmul_tiles.h"

namespace fpq {

namespace {

struct Plan {
    int tile, slices;
};

// Passes of the planes: the largest products of two operands, small ones first.
int passes(int planes_a, int planes_b) { return planes_a * planes_b == 9 ? 6 : planes_a * planes_b; }

Plan plan_product(int64_t M, int64_t N, int64_t K, int planes_a, int planes_b, bool col_a, bool gated)
{
    auto tiles = [&](int t) { return ((M + kTileM[t] - 1) / kTileM[t]) * ((N + kTileN[t] / (gated ? 2 : 1) - 1) / (kTileN[t] / (gated ? 2 : 1))); };
    const int64_t total = passes(planes_a, planes_b) * ((K + kStep - 1) / kStep);
    Plan p{kTile128, 1};
    if (tiles(kTile256) >= 200) p.tile = kTile256;
    else if (!col_a && M <= 32) p.tile = kTile32;
    const int64_t wanted = p.tile == kTile256 ? 256 : 512, n = tiles(p.tile);
    // parts of no fewer than eight steps, and no more than 16 of them
    int64_t most = total / 8 < 16 ? total / 8 : 16;
    if (n * 2 <= wanted && most > 1) p.slices = (int)(wanted / n < most ? wanted / n : most);
    return p;
}

struct SumArgs {
    const float* part;
    int64_t M, N;
    int slices;
    void* out;
    int64_t ld_out;
    int out_f32;
    const float* bias;
    Gate gate;
};

// Four columns of a row per thread.
__global__ __launch_bounds__(256) void matmul_sum_kernel(SumArgs p)
{
    const int64_t per = (p.N + 3) / 4, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= p.M * per) return;
    const int64_t m = id / per;
    const int n = (int)(id - m * per) * 4;
    const bool vec = (p.N & 3) == 0;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < p.slices; ++s) {
        const float* const x = p.part + (s * p.M + m) * p.N + n;
        if (vec) {
            const float4 t = *reinterpret_cast<const float4*>(x);
            v[0] += t.x;
            v[1] += t.y;
            v[2] += t.z;
            v[3] += t.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < p.N) v[e] += x[e];
        }
    }
    if (p.bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < p.N) v[e] += p.bias[n + e];
    }
    put4(p.out, m * p.ld_out + n, p.out_f32, n, (int)p.N, vec && (p.ld_out & 3) == 0 && ((uintptr_t)p.out & 15) == 0, v);
}

// A wavefront per 32 rows and 32 outputs, as the product's kernel leaves them.
__global__ __launch_bounds__(256) void matmul_sum_gated_kernel(SumArgs p)
{
    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int64_t blocks = (p.N + 31) / 32, id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), row = id / blocks, m = row * 32 + (lane & 31);
    if (row * 32 >= p.M) return;
    const int n0 = (int)(id - row * blocks) * 32, N = (int)p.N;
    const bool in = m < p.M;
    float a[16], g[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int n = n0 + 8 * (i / 4) + 4 * h + i % 4;
        a[i] = p.bias && n < N ? p.bias[n] : 0.0f;
        g[i] = p.bias && n < N ? p.bias[N + n] : 0.0f;
    }
    for (int s = 0; s < p.slices; ++s) {
        const float* const x = p.part + (s * p.M + (in ? m : 0)) * 2 * N;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int n = n0 + 8 * (i / 4) + 4 * h + i % 4;
            a[i] += n < N ? x[n] : 0.0f;
            g[i] += n < N ? x[N + n] : 0.0f;
        }
    }
    gated_block(p.gate, p.out_f32, m, n0, N, in, h, a, g);
}

}  // namespace

size_t product_part_bytes(int64_t M, int64_t N, int64_t K, int planes_a, int planes_b, bool col_a, bool gated)
{
    if (M == 0 || N == 0) return 0;
    const Plan p = plan_product(M, N, K, planes_a, planes_b, col_a, gated);
    return p.slices > 1 ? (size_t)p.slices * M * N * (gated ? 2 : 1) * 4 : 0;
}

int launch_product(const Product& q, void* part, hipStream_t s)
{
    if (q.M == 0 || q.N == 0) return FPQ_OK;
    const Plan plan = plan_product(q.M, q.N, q.K, q.planes_a, q.planes_b, q.col_a, q.gated);
    MatmulArgs p{};
    p.a = q.a;
    p.b = q.b;
    p.M = (int)q.M;
    p.N = (int)q.N;
    p.K = (int)q.K;
    p.steps = q.K ? (int)((q.K + kStep - 1) / kStep) : 1;
    if (q.planes_a == 3 && q.planes_b == 3) p.order_a = 0x001102, p.order_b = 0x010120;
    else if (q.planes_a == 3) p.order_a = 0x012;
    else if (q.planes_b == 3) p.order_b = 0x012;
    p.total = q.K ? p.steps * passes(q.planes_a, q.planes_b) : 0;      // (no rows to sum over: zeros)
    p.slices = plan.slices;
    const int cols = kTileN[plan.tile] / (q.gated ? 2 : 1);
    p.tiles_m = (int)((q.M + kTileM[plan.tile] - 1) / kTileM[plan.tile]);
    p.tiles_n = (int)((q.N + cols - 1) / cols);
    p.out = plan.slices > 1 ? part : q.out;
    p.ld_out = q.ld_out;
    p.out_f32 = q.out_f32;
    p.bias = q.bias;
    p.gate = q.gate;
    int st = q.gated ? launch_matmul_gated(p, plan.tile, s)
             : q.col_a ? launch_matmul_cols(p, plan.tile, s)
             : q.col_b ? launch_matmul_rows_cols(p, plan.tile, s)
                       : launch_matmul_rows(p, plan.tile, s);
    if (st != FPQ_OK || plan.slices == 1) return st;
    const SumArgs r{static_cast<const float*>(part), q.M, q.N, plan.slices, q.out, q.ld_out, q.out_f32, q.bias, q.gate};
    if (q.gated) {
        const int64_t waves = ((q.M + 31) / 32) * ((q.N + 31) / 32);
        matmul_sum_gated_kernel<<<dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s>>>(r);
    } else {
        const int64_t threads = q.M * ((q.N + 3) / 4);
        matmul_sum_kernel<<<dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s>>>(r);
    }
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

}  // namespace fpq
