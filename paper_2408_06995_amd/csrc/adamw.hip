// AdamW over many tensors in one launch: the adapters of a whole network, or the rounding parameters of its layers.
//
//   g = grad * grad_scale,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every operation is one rounded fp32 operation in the order written (no fused multiply-add), so that the 8-bit codes, which are
// choices between neighbours, are the same wherever the formula is evaluated in fp32.
//
// 8-bit states: m and the root of v (whose range is half that of v in the logarithm) as E4M3 codes, 256 neighbouring elements of a
// tensor sharing a scale of their largest magnitude / 448.  A positive root never becomes code 0: it would divide the next step by
// eps alone.  One wavefront owns a block of 256, four elements per lane.
//
// The work is memory traffic (28 bytes per element with 32-bit states, 16.06 with 8 bits): a workgroup takes a piece of 2048 elements
// of one tensor, all its loads ahead of the arithmetic.  Which piece is in a table that the plan writes once, so that a step is one
// launch with two dependent loads ahead of the data, whatever the number of tensors.  59.7 M elements, 8-bit states: 178 us, 5.4 TB/s;
// 256 tensors of up to 20480 elements, 32-bit states and a copy in bf16 (34 MB): 9.6 us, 3.6 TB/s, of which about 3 are the launch.
#include <math.h>

#include "adamw.h"
#include "fpq_dev.h"

#pragma clang fp contract(off)

namespace fpq {

namespace {

constexpr int kGroups = kAdamwPiece / 1024;            // of four elements per thread
constexpr float kMaxE4M3 = 448.0f;

struct Step {
    float b1, c1, b2, c2;                              // beta, 1 - beta
    float root, eps, decay, size;                      // (1 - b2^t)^-1/2, eps, 1 - lr wd, lr / (1 - b1^t)
    const float* grad_scale;
};

struct Four {
    float v[4];
};

template <bool VEC>
__device__ __forceinline__ Four get(const float* p, int64_t i, int64_t n)
{
    Four r;
    if (VEC) {
        const float4 a = *reinterpret_cast<const float4*>(p + i);
        r.v[0] = a.x; r.v[1] = a.y; r.v[2] = a.z; r.v[3] = a.w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) r.v[e] = i + e < n ? p[i + e] : 0.0f;
    }
    return r;
}
template <bool VEC>
__device__ __forceinline__ Four get(const __bf16* p, int64_t i, int64_t n)
{
    Four r;
    if (VEC) {
        const uint2 a = *reinterpret_cast<const uint2*>(p + i);
        r.v[0] = __uint_as_float(a.x << 16); r.v[1] = __uint_as_float(a.x & 0xffff0000u);
        r.v[2] = __uint_as_float(a.y << 16); r.v[3] = __uint_as_float(a.y & 0xffff0000u);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) r.v[e] = i + e < n ? (float)p[i + e] : 0.0f;
    }
    return r;
}
template <bool VEC>
__device__ __forceinline__ uint32_t get(const uint8_t* p, int64_t i, int64_t n)
{
    if (VEC) return *reinterpret_cast<const uint32_t*>(p + i);
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) r |= i + e < n ? (uint32_t)p[i + e] << (8 * e) : 0u;
    return r;
}

template <bool VEC>
__device__ __forceinline__ void put(float* p, int64_t i, int64_t n, const Four& x)
{
    if (VEC) {
        *reinterpret_cast<float4*>(p + i) = make_float4(x.v[0], x.v[1], x.v[2], x.v[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) p[i + e] = x.v[e];
    }
}
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef float v2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t two(float a, float b)
{
    const v2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, v2b));
}
template <bool VEC>
__device__ __forceinline__ void put(__bf16* p, int64_t i, int64_t n, const Four& x)
{
    if (VEC) {
        *reinterpret_cast<uint2*>(p + i) = make_uint2(two(x.v[0], x.v[1]), two(x.v[2], x.v[3]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) p[i + e] = (__bf16)x.v[e];
    }
}
template <bool VEC>
__device__ __forceinline__ void put(uint8_t* p, int64_t i, int64_t n, uint32_t x)
{
    if (VEC) {
        *reinterpret_cast<uint32_t*>(p + i) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) p[i + e] = (uint8_t)(x >> (8 * e));
    }
}

__device__ __forceinline__ Four decode(uint32_t codes, float scale)
{
    const v2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    return Four{{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale}};
}

// Codes of the four values of each lane; the wavefront's largest magnitude makes the scale.  Compared as bits, which orders
// magnitudes and puts what is no number above infinity: it makes the scale one too.
template <bool ROOT>
__device__ __forceinline__ uint32_t encode(const Four& x, float& scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(x.v[e]) & 0x7fffffffu);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off));
    // (a scale below the smallest normal number has no reciprocal)
    scale = top == 0 ? 1.0f : __uint_as_float(top) * (1.0f / kMaxE4M3);
    if (scale < 1.17549435e-38f) scale = 1.17549435e-38f;
    const float r = 1.0f / scale;
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        y[e] = fminf(fmaxf(x.v[e] * r, -kMaxE4M3), kMaxE4M3);
        if (ROOT && x.v[e] > 0.0f) y[e] = fmaxf(y[e], 0x1p-9f);
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
}

template <typename P, typename G, bool EIGHT, bool VEC>
__device__ __forceinline__ void piece(const AdamwEntry& t, int64_t first, const Step& s, float gs)
{
    const int64_t n = t.n;
    typename std::conditional<EIGHT, uint32_t, Four>::type mr[kGroups], vr[kGroups];
    typedef typename std::conditional<EIGHT, uint8_t, float>::type S;
    Four p[kGroups], g[kGroups];
    float ms[kGroups], vs[kGroups];
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
        const int64_t i = first + 1024 * u + 4 * threadIdx.x;
        if (i >= n) continue;
        g[u] = get<VEC>(static_cast<const G*>(t.grad), i, n);
        mr[u] = get<VEC>(static_cast<const S*>(t.m), i, n);
        vr[u] = get<VEC>(static_cast<const S*>(t.v), i, n);
        p[u] = get<VEC>(static_cast<const P*>(t.param), i, n);
        if (EIGHT) {
            ms[u] = t.m_scale[i >> 8];
            vs[u] = t.v_scale[i >> 8];
        }
    }
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
        const int64_t i = first + 1024 * u + 4 * threadIdx.x;
        if (first + 1024 * u + 256 * (int64_t)(threadIdx.x >> 6) >= n) continue;         // no element of the wavefront's block
        const bool in = i < n;
        Four m, v, root;
        if constexpr (EIGHT) {
            m = decode(in ? mr[u] : 0u, in ? ms[u] : 1.0f);
            root = decode(in ? vr[u] : 0u, in ? vs[u] : 1.0f);
#pragma unroll
            for (int e = 0; e < 4; ++e) v.v[e] = root.v[e] * root.v[e];
        } else {
            m = mr[u];
            v = vr[u];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = g[u].v[e] * gs;
            m.v[e] = m.v[e] * s.b1 + x * s.c1;
            v.v[e] = v.v[e] * s.b2 + x * s.c2 * x;
            root.v[e] = sqrtf(v.v[e]);
            p[u].v[e] = p[u].v[e] * s.decay - m.v[e] / (root.v[e] * s.root + s.eps) * s.size;
            if (i + e >= n) m.v[e] = root.v[e] = 0.0f;                                       // (they take part in the scale)
        }
        if (in) {
            put<VEC>(static_cast<P*>(t.param), i, n, p[u]);
            if (t.copy) put<VEC>(static_cast<__bf16*>(t.copy), i, n, p[u]);
        }
        if constexpr (EIGHT) {
            float m_scale, v_scale;
            const uint32_t mc = encode<false>(m, m_scale), vc = encode<true>(root, v_scale);
            if (in) {
                put<VEC>(static_cast<uint8_t*>(t.m), i, n, mc);
                put<VEC>(static_cast<uint8_t*>(t.v), i, n, vc);
            }
            if ((threadIdx.x & 63) == 0) {
                t.m_scale[i >> 8] = m_scale;
                t.v_scale[i >> 8] = v_scale;
            }
        } else if (in) {
            put<VEC>(static_cast<float*>(t.m), i, n, m);
            put<VEC>(static_cast<float*>(t.v), i, n, v);
        }
    }
}

template <typename P, typename G>
__device__ __forceinline__ void piece(const AdamwEntry& t, int64_t first, const Step& s, float gs)
{
    const bool vec = t.vec && first + kAdamwPiece <= t.n;
    if (t.eight)
        vec ? piece<P, G, true, true>(t, first, s, gs) : piece<P, G, true, false>(t, first, s, gs);
    else
        vec ? piece<P, G, false, true>(t, first, s, gs) : piece<P, G, false, false>(t, first, s, gs);
}

__global__ __launch_bounds__(256) void adamw_kernel(const unsigned char* __restrict__ plan, Step s)
{
    const uint2 which = reinterpret_cast<const uint2*>(plan)[blockIdx.x];              // tensor, piece of it
    const AdamwEntry t = *reinterpret_cast<const AdamwEntry*>(plan + adamw_entries_at(gridDim.x) + (size_t)which.x * sizeof(AdamwEntry));
    const int64_t first = (int64_t)which.y * kAdamwPiece;
    const float gs = s.grad_scale ? s.grad_scale[0] : 1.0f;
    if (t.param_type == FPQ_TYPE_FP32)
        t.grad_type == FPQ_TYPE_FP32 ? piece<float, float>(t, first, s, gs) : piece<float, __bf16>(t, first, s, gs);
    else
        t.grad_type == FPQ_TYPE_FP32 ? piece<__bf16, float>(t, first, s, gs) : piece<__bf16, __bf16>(t, first, s, gs);
}

constexpr int kBatch = 32;
struct Batch {
    AdamwEntry entry[kBatch];
    int64_t first[kBatch];         // of its pieces
};

// One workgroup per tensor: its entry and its pieces.
__global__ __launch_bounds__(256) void adamw_plan_kernel(unsigned char* plan, Batch b, int tensor0, int64_t pieces)
{
    const int k = blockIdx.x;
    AdamwEntry* at = reinterpret_cast<AdamwEntry*>(plan + adamw_entries_at(pieces)) + tensor0 + k;
    if (threadIdx.x == 0) *at = b.entry[k];
    const int64_t n = (b.entry[k].n + kAdamwPiece - 1) / kAdamwPiece;
    for (int64_t i = threadIdx.x; i < n; i += 256) reinterpret_cast<uint2*>(plan)[b.first[k] + i] = make_uint2(tensor0 + k, (uint32_t)i);
}

}  // namespace

// The arrays of a tensor aligned for four elements at a time.
static bool four_at_a_time(const fpq_adamw_tensor_t& t)
{
    auto ok = [](const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; };
    const size_t state = t.state_bits == 8 ? 4 : 16;
    return ok(t.param, t.param_type == FPQ_TYPE_FP32 ? 16 : 8) && ok(t.grad, t.grad_type == FPQ_TYPE_FP32 ? 16 : 8) && ok(t.m, state) &&
           ok(t.v, state) && ok(t.copy, 8);
}

int launch_adamw_plan(const fpq_adamw_tensor_t* tensors, int count, int64_t pieces, void* plan, hipStream_t s)
{
    int64_t first = 0;
    for (int t = 0; t < count; t += kBatch) {
        Batch b{};
        const int n = count - t < kBatch ? count - t : kBatch;
        for (int k = 0; k < n; ++k) {
            const fpq_adamw_tensor_t& x = tensors[t + k];
            b.entry[k] = AdamwEntry{x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.n, x.param_type, x.grad_type, x.state_bits == 8,
                                    four_at_a_time(x)};
            b.first[k] = first;
            first += (x.n + kAdamwPiece - 1) / kAdamwPiece;
        }
        adamw_plan_kernel<<<dim3(n), dim3(256), 0, s>>>(static_cast<unsigned char*>(plan), b, t, pieces);
    }
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

int launch_adamw(const void* plan, int64_t pieces, double lr, double beta1, double beta2, double eps, double weight_decay, int64_t step,
                 const float* grad_scale, hipStream_t s)
{
    Step k;
    k.b1 = (float)beta1;
    k.c1 = (float)(1.0 - beta1);
    k.b2 = (float)beta2;
    k.c2 = (float)(1.0 - beta2);
    k.root = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
    k.eps = (float)eps;
    k.decay = (float)(1.0 - lr * weight_decay);
    k.size = (float)(lr / (1.0 - pow(beta1, (double)step)));
    k.grad_scale = grad_scale;
    adamw_kernel<<<dim3((unsigned)pieces), dim3(256), 0, s>>>(static_cast<const unsigned char*>(plan), k);
    return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

}  // namespace fpq
