// The adapters' plan of a call, the choice of its types, and the sums of partial gradients.
#include "adapter.h"

namespace fpq {

int launch_apply_f32(const AdapterArgs& a, bool vec_k, const AdapterPlan& plan, hipStream_t s);
int launch_apply_mixed(const AdapterArgs& a, bool vec_k, const AdapterPlan& plan, hipStream_t s);
int launch_apply_bf16(const AdapterArgs& a, bool vec_k, const AdapterPlan& plan, hipStream_t s);
int launch_backward_f32(const AdapterArgs& a, bool vec_n, bool vec_k, const AdapterPlan& plan, hipStream_t s);
int launch_backward_mixed(const AdapterArgs& a, bool vec_n, bool vec_k, const AdapterPlan& plan, hipStream_t s);
int launch_backward_bf16(const AdapterArgs& a, bool vec_n, bool vec_k, const AdapterPlan& plan, hipStream_t s);

// Few tiles of rows: the sums over K are cut into parts and the columns of a result go to more workgroups, until about two (four)
// workgroups per compute unit; a part keeps two steps of 32 for each of a workgroup's wavefronts.
AdapterPlan plan_adapter(int64_t M, int64_t N, int64_t K, int64_t R, int64_t requests, int64_t adapters)
{
    auto clamp = [](int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; };
    const int64_t tiles = clamp(M / kTile + (requests < M ? requests : M), 1, (int64_t)1 << 31), steps = (K + 31) / 32;
    AdapterPlan p;
    p.parts = (int)clamp(512 / tiles, 1, clamp(steps / 8, 1, 16));
    p.steps_per_part = (int)((steps + p.parts - 1) / p.parts);
    p.parts = (int)((steps + p.steps_per_part - 1) / p.steps_per_part);
    auto columns = [&](int64_t L) {
        const int64_t blocks = (L + 127) / 128, chunks = clamp(1024 / tiles, 1, blocks);
        return (int)((blocks + chunks - 1) / chunks * 128);
    };
    p.columns_y = columns(N);
    p.columns_x = columns(K);
    const int64_t blocks = adapters * ((K + 127) / 128 + (N + 127) / 128);
    p.splits = (int)clamp(1024 / (blocks > 0 ? blocks : 1), 1, clamp(M / (8 * kTile), 1, 64));
    (void)R;
    return p;
}

namespace {

__global__ __launch_bounds__(256) void adapter_sums_kernel(AdapterArgs p, size_t na, size_t nb)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < na + nb; i += (size_t)gridDim.x * 256) {
        const bool b = i >= na;
        const size_t e = b ? i - na : i, n = b ? nb : na;
        const float* const part = b ? p.part_b : p.part_a;
        float v = part[e];
        for (int s = 1; s < p.splits; ++s) v += part[s * n + e];
        (b ? p.gb : p.ga)[e] = v;
    }
}

}  // namespace

int launch_adapter_sums(const AdapterArgs& a, hipStream_t s)
{
    const size_t na = (size_t)a.adapters * a.R * a.K, nb = (size_t)a.adapters * a.R * a.N, want = (na + nb + 255) / 256;
    adapter_sums_kernel<<<dim3((unsigned)(want < 4096 ? want : 4096)), dim3(256), 0, s>>>(a, na, nb);
    return FPQ_OK;
}

int launch_adapter_apply(const AdapterArgs& a, int x_type, int w_type, bool vec_k, const AdapterPlan& plan, hipStream_t s)
{
    return x_type == FPQ_TYPE_BF16   ? launch_apply_bf16(a, vec_k, plan, s)
           : w_type == FPQ_TYPE_BF16 ? launch_apply_mixed(a, vec_k, plan, s)
                                     : launch_apply_f32(a, vec_k, plan, s);
}

int launch_adapter_backward(const AdapterArgs& a, int x_type, int w_type, bool vec_n, bool vec_k, const AdapterPlan& plan, hipStream_t s)
{
    return x_type == FPQ_TYPE_BF16   ? launch_backward_bf16(a, vec_n, vec_k, plan, s)
           : w_type == FPQ_TYPE_BF16 ? launch_backward_mixed(a, vec_n, vec_k, plan, s)
                                     : launch_backward_f32(a, vec_n, vec_k, plan, s);
}

}  // namespace fpq
