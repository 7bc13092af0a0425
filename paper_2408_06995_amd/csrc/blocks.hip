// Blocks of codes with a power of two as their scale, and the elementwise passes around the products: planes of operands, column sums,
// the gated projections' gradient before the products.  All are bound by memory: a lane takes eight neighbouring elements, 16 bytes or
// twice as many at any address, and two such pieces, so that there are enough loads on their way.  Read and written together: planes of 10240 x 4096 in fp32 6.3
// TB/s (66 us), blocks back to bf16 6.1 (5003 x 5120: 12.8 us), to blocks 4.7 (16.5 us), the gated gradient of 8192 x 5120 from
// blocks 5.6 (90 us), column sums of 32768 x 960 in bf16 4.5 (13.9 us).
#include "blocks.h"

namespace fpq {

namespace {

// Eight elements from column k on; zeros from `cols` on.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int64_t k, int64_t cols, float (&v)[8])
{
    if (k + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            const piece16 a = *reinterpret_cast<const piece16*>(row + k), b = *reinterpret_cast<const piece16*>(row + k + 4);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                v[t] = __uint_as_float(a[t]);
                v[4 + t] = __uint_as_float(b[t]);
            }
        } else {
            const piece16 w = *reinterpret_cast<const piece16*>(row + k);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                v[2 * t] = __uint_as_float(w[t] << 16);
                v[2 * t + 1] = __uint_as_float(w[t] & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k + e < cols ? (float)row[k + e] : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* row, int64_t k, int64_t cols, const float (&v)[8])
{
    if (k + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int t = 0; t < 8; t += 4)
                *reinterpret_cast<piece16*>(row + k + t) =
                    piece16{__float_as_uint(v[t]), __float_as_uint(v[t + 1]), __float_as_uint(v[t + 2]), __float_as_uint(v[t + 3])};
        } else {
            *reinterpret_cast<piece16*>(row + k) = piece16{pair_bf16(v[0], v[1]), pair_bf16(v[2], v[3]), pair_bf16(v[4], v[5]), pair_bf16(v[6], v[7])};
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (k + e < cols) row[k + e] = (T)v[e];
    }
}

// Eight values in NP planes; of fewer than eight the first `some`.
template <int NP>
__device__ __forceinline__ void store_planes(__bf16* dst, int64_t plane, const float (&v)[8], int64_t some = 8)
{
    const Frag<NP> f = frag_of<NP>(v);
    if (some >= 8) {
#pragma unroll
        for (int p = 0; p < NP; ++p) *reinterpret_cast<piece16*>(dst + p * plane) = __builtin_bit_cast(piece16, f.p[p]);
    } else {
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < some) dst[p * plane + e] = f.p[p][e];
    }
}

// Eight codes of a block.
template <bool EIGHT>
__device__ __forceinline__ void decode8(const uint8_t* codes, int64_t at, float s, float (&v)[8])
{
    if constexpr (EIGHT) {
        const uint2 w = *reinterpret_cast<const uint2*>(codes + at);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t x = t ? w.y : w.x;
            const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
            v[4 * t] = a.x * s;
            v[4 * t + 1] = a.y * s;
            v[4 * t + 2] = b.x * s;
            v[4 * t + 3] = b.y * s;
        }
    } else {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + at / 2);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // 1 + e + m = 4 bits in a half's place: exponent bias 1 there against 15
            const uint32_t c = w >> (4 * e), bits = (c & 8) << 28 | (c & 7) << 22;
            v[e] = __uint_as_float(bits) * 0x1p126f * s;
        }
    }
}

constexpr int kEach = 2;                // pieces of eight elements per thread

template <int KIND>
__device__ __forceinline__ void pack_pieces(const PackItem& q, int64_t id0)
{
    const int64_t per = q.pieces.per, n = q.rows * per;
    constexpr int NP = KIND == FPQ_TYPE_FP32 ? 3 : 1;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t id = id0 + 256 * i;
        if (id >= n) return;
        const int64_t r = row_at(q.pieces, id), k = (id - r * per) * 8;
        float v[8];
        if constexpr (KIND == FPQ_TYPE_FP32) load8(static_cast<const float*>(q.src) + r * q.ld, k, q.cols, v);
        else if constexpr (KIND == FPQ_TYPE_BF16) load8(static_cast<const __bf16*>(q.src) + r * q.ld, k, q.cols, v);
        else decode8<KIND == 8>(static_cast<const uint8_t*>(q.src), id * 8, scale_of(q.scales[id / 4]), v);
        store_planes<NP>(q.dst + r * q.ld_dst + k, q.plane, v);
    }
}

__global__ __launch_bounds__(256) void pack_kernel(PackList p)
{
    const int which = p.count > 2 && blockIdx.x >= p.m[2].first ? 2 : p.count > 1 && blockIdx.x >= p.m[1].first ? 1 : 0;
    const PackItem q = which == 2 ? p.m[2] : which == 1 ? p.m[1] : p.m[0];
    const int64_t id0 = (int64_t)(blockIdx.x - q.first) * (256 * kEach) + threadIdx.x;
    if (q.kind == FPQ_TYPE_FP32) pack_pieces<FPQ_TYPE_FP32>(q, id0);
    else if (q.kind == FPQ_TYPE_BF16) pack_pieces<FPQ_TYPE_BF16>(q, id0);
    else if (q.kind == 8) pack_pieces<8>(q, id0);
    else pack_pieces<4>(q, id0);
}

template <bool EIGHT, typename T>
__global__ __launch_bounds__(256) void decode_kernel(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, RowOf pieces, T* dst, int64_t ld_dst)
{
    const int64_t n = rows * pieces.per, id0 = (int64_t)blockIdx.x * (256 * kEach) + threadIdx.x;
    float v[kEach][8];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t id = min(id0 + 256 * i, n - 1);
        decode8<EIGHT>(codes, id * 8, scale_of(scales[id / 4]), v[i]);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t id = id0 + 256 * i;
        if (id >= n) return;
        const int64_t r = row_at(pieces, id);
        store8(dst + r * ld_dst, (id - r * pieces.per) * 8, cols, v[i]);
    }
}

template <bool EIGHT, typename T>
__global__ __launch_bounds__(256) void block_quantize_kernel(const T* x, int64_t rows, int64_t cols, RowOf pieces, int64_t ld, const uint8_t* mask, uint8_t* codes,
                                                             uint8_t* scales)
{
    const int64_t n = rows * pieces.per, id0 = (int64_t)blockIdx.x * (256 * kEach) + threadIdx.x;
    float all[kEach][8];
    int64_t row[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t id = min(id0 + 256 * i, n - 1);                // (n is a multiple of four: a block's lanes stay together)
        row[i] = row_at(pieces, id);
        load8(x + row[i] * ld, (id - row[i] * pieces.per) * 8, cols, all[i]);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t id = id0 + 256 * i, k = (id - row[i] * pieces.per) * 8;
        const float (&v)[8] = all[i];
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
        if (id >= n) continue;
        const uint32_t s = EIGHT ? block_scale8(top) : block_scale4(top);
        const float r = inverse_scale(s);
        if ((threadIdx.x & 3) == 0) scales[id / 4] = (uint8_t)s;
        if constexpr (EIGHT) {
            *reinterpret_cast<uint2*>(codes + id * 8) = make_uint2(codes8(v[0] * r, v[1] * r, v[2] * r, v[3] * r), codes8(v[4] * r, v[5] * r, v[6] * r, v[7] * r));
        } else {
            const QParams q{1, 1, 3, 6.0f};
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (k + e >= cols) break;
                const uint32_t c = mask ? quantize_mask(v[e], r, mask[row[i] * cols + k + e], q) : quantize_nearest(v[e], r, q);
                w |= c << (4 * e);
            }
            *reinterpret_cast<uint32_t*>(codes + id * 4) = s == 255 ? 0u : w;
        }
    }
}

// ---- sums over rows: 64 lanes of eight columns, four wavefronts over the rows of a part

constexpr int kStripColumns = 512;

// A lane's sums of eight neighbouring columns, over the four wavefronts.
__device__ __forceinline__ void strip_sum(float (&sum)[8], int64_t first, int64_t cols, float* part)
{
    __shared__ float room[3][64 * 8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();
    if (wave) {
#pragma unroll
        for (int e = 0; e < 8; ++e) room[wave - 1][e * 64 + lane] = sum[e];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = (sum[e] + room[0][e * 64 + lane]) + (room[1][e * 64 + lane] + room[2][e * 64 + lane]);
        const int64_t k = first + 8 * lane + e;
        if (k < cols) part[k] = t;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void column_sums_kernel(const T* x, int64_t M, int64_t N, int64_t ld, int64_t rows, float* part)
{
    const int64_t k = ((int64_t)blockIdx.x * 64 + (threadIdx.x & 63)) * 8, m1 = min(M, (int64_t)(blockIdx.y + 1) * rows);
    float sum[8] = {};
    int64_t m = (int64_t)blockIdx.y * rows + (threadIdx.x >> 6);
    if (k < N) {
        for (; m + 12 < m1; m += 16) {                               // four rows' loads at once
            float v[4][8];
#pragma unroll
            for (int i = 0; i < 4; ++i) load8(x + (m + 4 * i) * ld, k, N, v[i]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += v[i][e];
        }
        for (; m < m1; m += 4) {
            float v[8];
            load8(x + m * ld, k, N, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[e];
        }
    }
    strip_sum(sum, (int64_t)blockIdx.x * kStripColumns, N, part + (int64_t)blockIdx.y * N);
}

// 64 columns, 16 wavefronts over the parts
__global__ __launch_bounds__(1024) void part_sums_kernel(const float* part, int parts, int64_t cols, float* out)
{
    __shared__ float room[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t k = (int64_t)blockIdx.x * 64 + lane;
    float sum = 0.0f;
    if (k < cols) {
        int p = wave;
        for (; p + 112 < parts; p += 128) {                          // eight loads at once
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = part[(int64_t)(p + 16 * i) * cols + k];
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[i];
        }
        for (; p < parts; p += 16) sum += part[(int64_t)p * cols + k];
    }
    room[wave][lane] = sum;
    __syncthreads();
    if (wave || k >= cols) return;
    for (int w = 1; w < 16; ++w) sum += room[w][lane];
    out[k] = sum;
}

// da = gh act(g), dg = gh a act'(g), in the planes that the products read, and their column sums.  A strip of 512 columns and a part of the rows per workgroup: the
// sums stay in registers, and what the products read is written in whole lines.  KEPT: 0 the type, 1 blocks.
template <typename T, int KEPT>
__global__ __launch_bounds__(256) void gate_backward_kernel(GateBackward p, int64_t rows)
{
    const int64_t first = (int64_t)blockIdx.x * kStripColumns, m1 = min(p.M, (int64_t)(blockIdx.y + 1) * rows), N = p.N;
    const int64_t k = first + 8 * (threadIdx.x & 63), np = (N + 31) / 32 * 32;
    constexpr int NP = sizeof(T) == 4 ? 3 : 2;                         // gate_planes
    float sum_a[8] = {}, sum_g[8] = {};
    if (k < N)
        for (int64_t m = (int64_t)blockIdx.y * rows + (threadIdx.x >> 6); m < m1; m += 4) {
            float a[8], g[8], gh[8], da[8], dg[8];
            load8(static_cast<const T*>(p.gh) + m * p.ld_gh, k, N, gh);
            if constexpr (KEPT) {
                const uint8_t* const s = p.pre_scales + m * (np / 16) + k / 32;
                const uint8_t* const c = static_cast<const uint8_t*>(p.pre) + m * 2 * np;
                decode8<true>(c, k, scale_of(s[0]), a);
                decode8<true>(c + np, k, scale_of(s[np / 32]), g);
            } else {
                const T* const row = static_cast<const T*>(p.pre) + m * 2 * N;
                load8(row, k, N, a);
                load8(row + N, k, N, g);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float slope;
                da[e] = gh[e] * gate_of<true>(p.act, g[e], &slope);
                dg[e] = gh[e] * a[e] * slope;
                sum_a[e] += da[e];
                sum_g[e] += dg[e];
            }
            if (!p.d) continue;
            __bf16* const d = p.d + m * p.ld_d + k;
            store_planes<NP>(d, p.plane, da, N - k);
            const int64_t left = p.ld_d - N - k;
            if (N - k < 8) {                                          // the row's end, and up to six zeros behind it
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k + e >= N) dg[e] = 0.0f;
                for (int64_t e = 8; e < left; ++e)
#pragma unroll
                    for (int q = 0; q < NP; ++q) d[q * p.plane + N + e] = (__bf16)0.0f;
            }
            store_planes<NP>(d + N, p.plane, dg, left);
        }
    if (!p.part) return;
    float* const part = p.part + (int64_t)blockIdx.y * 2 * N;
    strip_sum(sum_a, first, N, part);
    strip_sum(sum_g, first, N, part + N);
}

unsigned grid_of(int64_t pieces) { return (unsigned)((pieces + 256 * kEach - 1) / (256 * kEach)); }
int launched() { return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH; }

}  // namespace

// One launch, of fewer than 2^24 workgroups (2^32 threads) whatever the operands: they are [M, N], [N, K] and [M, K] with M <= 2^28, N, K <= 2^20 and fewer than 2^34
// elements each.  Rows filled up to multiples of 8, or 32 as blocks, make at most 2^34 72 / 65 and 2^34 96 / 65 elements of 4096 a workgroup, together 10.8 M
// workgroups; [N, K] adds at most 2.1 M while it has no more than 2^33, and with more all columns are 2^13 and up, the filling below 1 / 250, and the three
// 12.7 M.
int launch_packs(PackList& p, hipStream_t s)
{
    int64_t at = 0;
    for (int i = 0; i < p.count; ++i) {
        PackItem& q = p.m[i];
        q.first = at;
        q.pieces = row_of(q.rows, q.ld_dst / 8);
        at += grid_of(q.rows * (q.ld_dst / 8));
    }
    if (!at) return FPQ_OK;
    pack_kernel<<<dim3((unsigned)at), dim3(256), 0, s>>>(p);
    return launched();
}

int launch_decode(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, bool eight, void* dst, int f32, int64_t ld_dst, hipStream_t s)
{
    const int64_t padded = block_padded(cols);
    const unsigned grid = grid_of(rows * (padded / 8));
    if (!grid) return FPQ_OK;
    auto run = [&](auto kernel, auto* to) { kernel<<<dim3(grid), dim3(256), 0, s>>>(codes, scales, rows, cols, row_of(rows, padded / 8), to, ld_dst); };
    if (f32) eight ? run(decode_kernel<true, float>, static_cast<float*>(dst)) : run(decode_kernel<false, float>, static_cast<float*>(dst));
    else eight ? run(decode_kernel<true, __bf16>, static_cast<__bf16*>(dst)) : run(decode_kernel<false, __bf16>, static_cast<__bf16*>(dst));
    return launched();
}

int launch_block_quantize(const void* x, int type, int64_t M, int64_t K, int64_t ld, bool eight, const uint8_t* mask, uint8_t* codes, uint8_t* scales,
                          hipStream_t s)
{
    const int64_t padded = block_padded(K);
    const unsigned grid = grid_of(M * (padded / 8));
    if (!grid) return FPQ_OK;
    auto run = [&](auto kernel, auto* from) { kernel<<<dim3(grid), dim3(256), 0, s>>>(from, M, K, row_of(M, padded / 8), ld, mask, codes, scales); };
    if (type == FPQ_TYPE_FP32) eight ? run(block_quantize_kernel<true, float>, static_cast<const float*>(x)) : run(block_quantize_kernel<false, float>, static_cast<const float*>(x));
    else eight ? run(block_quantize_kernel<true, __bf16>, static_cast<const __bf16*>(x)) : run(block_quantize_kernel<false, __bf16>, static_cast<const __bf16*>(x));
    return launched();
}

// About 1024 workgroups, of no fewer than four rows (300 x 320 -> 1280 with its gradient in bf16: 30.7 us,
// 31.4 with eight), and no more parts than their sum is
// quick with; but parts of no more than some 8192 rows, 2048 a lane, so that no sum's roundings grow with the number of rows (2^26 rows of ones and tenths: off by
// 3e-4 with 512 parts).
RowParts row_parts(int64_t M, int64_t cols)
{
    const int64_t strips = (cols + kStripColumns - 1) / kStripColumns;
    int64_t parts = 1024 / strips < 512 ? 1024 / strips : 512, most = (M + 3) / 4;
    if (parts < M / 8192) parts = M / 8192;
    parts = parts < 1 ? 1 : parts > most ? most : parts;
    if (parts < 1) parts = 1;
    const int64_t rows = (M + parts - 1) / parts;
    return RowParts{rows < 1 ? 1 : rows, (int)(rows < 1 ? 1 : (M + rows - 1) / rows)};
}
size_t row_parts_bytes(int64_t M, int64_t cols) { return (size_t)row_parts(M, cols).parts * cols * 4; }

int launch_part_sums(const float* part, int parts, int64_t cols, float* out, hipStream_t s)
{
    part_sums_kernel<<<dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0, s>>>(part, parts, cols, out);
    return launched();
}

int launch_column_sums(const void* x, int type, int64_t M, int64_t N, int64_t ld, float* out, float* part, hipStream_t s)
{
    const RowParts r = row_parts(M, N);
    const dim3 grid((unsigned)((N + kStripColumns - 1) / kStripColumns), (unsigned)r.parts);
    if (type == FPQ_TYPE_FP32) column_sums_kernel<<<grid, dim3(256), 0, s>>>(static_cast<const float*>(x), M, N, ld, r.rows, part);
    else column_sums_kernel<<<grid, dim3(256), 0, s>>>(static_cast<const __bf16*>(x), M, N, ld, r.rows, part);
    const int st = launched();
    return st == FPQ_OK ? launch_part_sums(part, r.parts, N, out, s) : st;
}

int launch_gate_backward(const GateBackward& p, hipStream_t s)
{
    const RowParts r = row_parts(p.M, p.N);
    const dim3 grid((unsigned)((p.N + kStripColumns - 1) / kStripColumns), (unsigned)r.parts);
    GateBackward q = p;
    if (!p.grad_bias) q.part = nullptr;
    auto run = [&](auto kernel) { kernel<<<grid, dim3(256), 0, s>>>(q, r.rows); };
    if (p.type == FPQ_TYPE_FP32) p.pre_scales ? run(gate_backward_kernel<float, 1>) : run(gate_backward_kernel<float, 0>);
    else p.pre_scales ? run(gate_backward_kernel<__bf16, 1>) : run(gate_backward_kernel<__bf16, 0>);
    const int st = launched();
    return st == FPQ_OK && q.part ? launch_part_sums(q.part, r.parts, 2 * p.N, p.grad_bias, s) : st;
}

}  // namespace fpq
