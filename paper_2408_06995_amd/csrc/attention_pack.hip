// Tensors whose rows the feed of the attention kernels cannot read as they are, packed into rows of whole 16-byte pieces: fp32 ones as
// three bf16 planes (once, instead of by every workgroup that reads them), bf16 ones of other alignments as they are.  Bound by
// memory: an fp32 element is read once (4 bytes) and written once (6).
#include "attention.h"

namespace fpq {

namespace {

template <typename T>
__global__ __launch_bounds__(256) void attention_pack_kernel(PackArgs a)
{
    constexpr int NP = kPlanes<T>;
    const Pack& m = a.m[blockIdx.y];
    const int pieces = (a.dim + 7) / 8;
    const int64_t heads = m.heads, n = a.batch * heads * m.len * pieces, plane = n * 8;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < n; id += (int64_t)gridDim.x * 256) {
        // in the order of the tensors that are usual here: heads of a token are neighbours
        const int64_t at = id / pieces, tok = at / heads, head = at - tok * heads, b = tok / m.len, t = tok - b * m.len;
        const int c = (int)(id - at * pieces) * 8;
        if (m.by_lens && a.lens && t >= a.lens[b]) continue;
        const T* const row = static_cast<const T*>(m.src) + b * m.s.b + t * m.s.t + head * m.s.h;
        float v[8];
        if (reinterpret_cast<uintptr_t>(row + c) % 16 == 0 && c + 8 <= a.dim) {
            row8<T, true>(row, c, c + 8, v);
        } else {
            row8<T, false>(row, c, a.dim, v);
        }
        const Frag<NP> f = frag_of<NP>(v);
#pragma unroll
        for (int p = 0; p < NP; ++p) *reinterpret_cast<v8bf*>(m.dst + p * plane + ((b * heads + head) * m.len + t) * pieces * 8 + c) = f.p[p];
    }
}

}  // namespace

int launch_pack(const PackArgs& a, int type, hipStream_t s)
{
    int64_t most = 0;
    for (int i = 0; i < a.count; ++i) {
        const int64_t n = (int64_t)a.batch * a.m[i].heads * a.m[i].len * ((a.dim + 7) / 8);
        if (n > most) most = n;
    }
    if (!most) return FPQ_OK;
    const int64_t want = (most + 255) / 256;
    const dim3 grid((unsigned)(want < 8192 ? want : 8192), a.count);
    if (type == FPQ_TYPE_FP32)
        attention_pack_kernel<float><<<grid, dim3(256), 0, s>>>(a);
    else
        attention_pack_kernel<__bf16><<<grid, dim3(256), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

}  // namespace fpq
