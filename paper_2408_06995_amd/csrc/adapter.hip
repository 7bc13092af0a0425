// The adapters' plan of a call, the choice of its types, the packing of weights and the sums of partial gradients.
#include "adapter.h"

namespace fpq {

int launch_map_f32(const AdapterArgs& a, int waves, hipStream_t s);
int launch_map_f32_bf16(const AdapterArgs& a, int waves, hipStream_t s);
int launch_map_f32_packed(const AdapterArgs& a, int waves, hipStream_t s);
int launch_map_bf16(const AdapterArgs& a, int waves, hipStream_t s);
int launch_map_f32_bf16_packed(const AdapterArgs& a, int waves, hipStream_t s);
int launch_map_bf16_packed(const AdapterArgs& a, int waves, hipStream_t s);

// The map: four wavefronts per tile of 32 rows where the tiles fill the compute units (32768 rows of 320: 24 us; with eight 28, with
// 16 42); else 16, which divide the columns (64 rows of 1280 9.3 us; with eight 10.0, with four 13.4). Where the tiles leave most compute units
// idle, each has several workgroups, with a part of the columns and all of t each (259 rows of 1728 -> 5056 at rank 123: 58 us, with
// one 95; training step of 1000 rows of 1280 -> 1280 at rank 32 in bf16: 35 us, with one 41); with more tiles t's repetition costs more
// than it gives (5003 rows of 1280 -> 5120: 55 us, in two parts 64).
// Weights whose rows do not start at 16 bytes are packed for ranks above 16 (the same rows: read as they are 257 us); packing others
// ahead costs what it saves.
// The gradients' rows are cut until there are about four workgroups per compute unit, with no fewer than eight tiles each; but with
// 400 of them not at all (5003 rows, 450 workgroups: 29 us; the sums of two parts alone take 25).
AdapterPlan plan_adapter(int64_t M, int64_t N, int64_t K, int64_t requests, int64_t adapters)
{
    auto clamp = [](int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; };
    AdapterPlan p;
    p.waves = M / 32 + (requests < M / 32 ? requests : M / 32) >= 512 ? 4 : 16;
    const int64_t most = M / 32 + requests + 2;
    p.parts_n = (int)clamp(256 / most, 1, clamp(N / 256, 1, 8));
    p.parts_k = (int)clamp(256 / most, 1, clamp(K / 256, 1, 8));
    const int64_t blocks = adapters * ((K + 127) / 128 + (N + 127) / 128);
    p.splits = blocks >= 400 ? 1 : (int)clamp(1024 / blocks, 1, clamp(M / 256, 1, 64));
    return p;
}

namespace {

// A lane of an operand (see Weights) per thread: blockIdx.y = 2 adapter + which.
template <typename T>
__global__ __launch_bounds__(256) void adapter_pack_kernel(AdapterPack p, int groups, int64_t n1, int64_t n2)
{
    constexpr int NP = kPlanes<T>;
    const bool second = blockIdx.y & 1;
    const int adapter = blockIdx.y >> 1, lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), n = second ? n2 : n1;                // an operand of 64 lanes
    if (unit * 512 >= n) return;
    const int64_t outer = unit / groups;
    const int q = (int)(unit - outer * groups);
    const bool from_b = second == p.forward;                     // [L, R]; a is [R, L]
    const int L = from_b ? p.N : p.K;
    const T* const src = static_cast<const T*>(from_b ? p.b : p.a) + (size_t)adapter * p.R * L;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        // (rank, place along L) of the element
        const int rank = second ? 16 * q + 8 * (lane >> 5) + e : 16 * q + (lane & 15);
        const int64_t at = second ? 32 * outer + (lane & 31) : 32 * outer + 8 * (lane >> 4) + e;
        const int rc = min(rank, p.R - 1);
        const int64_t ac = min(at, (int64_t)L - 1);
        const float x = (float)src[from_b ? ac * p.R + rc : rc * (int64_t)L + ac];
        v[e] = rank < p.R && at < L ? x : 0.0f;
    }
    const Frag<NP> f = frag_of<NP>(v);
    __bf16* const dst = (second ? p.w2 : p.w1) + (size_t)adapter * NP * n + unit * 512 + lane * 8;
#pragma unroll
    for (int i = 0; i < NP; ++i) *reinterpret_cast<v8bf*>(dst + i * n) = f.p[i];
}

// 64 results per workgroup; its four wavefronts have a quarter of the parts each.
__global__ __launch_bounds__(256) void adapter_sums_kernel(const float* part_a, const float* part_b, int splits, size_t na, size_t nb, float* ga, float* gb)
{
    __shared__ float sums[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const size_t i = (size_t)blockIdx.x * 64 + lane;
    const bool b = i >= na, in = i < na + nb;
    const size_t e = b ? i - na : i, n = b ? nb : na;
    const float* const part = (b ? part_b : part_a) + (in ? e : 0);
    const int each = (splits + 3) / 4, s0 = wave * each, s1 = min(s0 + each, splits);
    float v = 0.0f;
    for (int s = s0; s < s1; s += 4) {
        float x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = part[min(s + u, s1 - 1) * n];
#pragma unroll
        for (int u = 0; u < 4; ++u) v += s + u < s1 ? x[u] : 0.0f;
    }
    sums[wave][lane] = v;
    __syncthreads();
    if (wave == 0 && in) (b ? gb : ga)[e] = ((sums[0][lane] + sums[1][lane]) + sums[2][lane]) + sums[3][lane];
}

}  // namespace

int launch_adapter_pack(const AdapterPack& a, int w_type, hipStream_t s)
{
    const int64_t n1 = packed_elements(a.forward ? a.K : a.N, a.R), n2 = packed_elements(a.forward ? a.N : a.K, a.R), most = n1 > n2 ? n1 : n2;
    const dim3 grid((unsigned)((most + 2047) / 2048), 2 * a.adapters);
    const int groups = rank_groups(a.R);
    if (w_type == FPQ_TYPE_FP32)
        adapter_pack_kernel<float><<<grid, dim3(256), 0, s>>>(a, groups, n1, n2);
    else
        adapter_pack_kernel<__bf16><<<grid, dim3(256), 0, s>>>(a, groups, n1, n2);
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

int launch_adapter_sums(const float* part_a, const float* part_b, int splits, size_t na, size_t nb, float* ga, float* gb, hipStream_t s)
{
    adapter_sums_kernel<<<dim3((unsigned)((na + nb + 63) / 64)), dim3(256), 0, s>>>(part_a, part_b, splits, na, nb, ga, gb);
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

int launch_adapter_map(const AdapterArgs& a, int x_type, int w_type, bool packed, int waves, hipStream_t s)
{
    if (x_type == FPQ_TYPE_BF16) return packed ? launch_map_bf16_packed(a, waves, s) : launch_map_bf16(a, waves, s);
    if (w_type == FPQ_TYPE_BF16) return packed ? launch_map_f32_bf16_packed(a, waves, s) : launch_map_f32_bf16(a, waves, s);
    return packed ? launch_map_f32_packed(a, waves, s) : launch_map_f32(a, waves, s);
}

}  // namespace fpq
