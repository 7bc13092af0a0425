// Root-mean-square norm on the residual stream, and its gradient.
//
// A row is read once: 8 to 256 threads hold it in registers, in pieces of 16 bytes, while its mean square (or the gradient's
// projection on it) is summed; bound by memory.  Rows too long for that are read a second time, which the caches serve.
// 8192 x 5120 in bf16: forward with the residual 62 us (5.4 TB/s), backward 65 with the weights' gradient (5.2); 32768 x 320 with codes 15.2 (4.9).
#include "blocks.h"

#include <iterator>
#include <utility>

namespace fpq {

namespace {

template <typename T>
constexpr int kPiece = 16 / (int)sizeof(T);

// Elements k .. of a row as they lie in memory, zeros from K on; and as numbers.  VEC: rows are whole pieces.
template <typename T, bool VEC>
__device__ __forceinline__ uint4 raw_piece(const T* row, int64_t k, int64_t K)
{
    constexpr int E = kPiece<T>;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (VEC ? k < K : k + E <= K) {
        x = __builtin_bit_cast(uint4, *reinterpret_cast<const piece16*>(row + k));
    } else if constexpr (!VEC) {
        T v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = k + e < K ? row[k + e] : (T)0.0f;
        __builtin_memcpy(&x, v, 16);
    }
    return x;
}
template <typename T>
__device__ __forceinline__ void numbers(const uint4& x, float (&v)[kPiece<T>])
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if constexpr (sizeof(T) == 4) {
            v[t] = __uint_as_float(w[t]);
        } else {
            v[2 * t] = __uint_as_float(w[t] << 16);
            v[2 * t + 1] = __uint_as_float(w[t] & 0xffff0000u);
        }
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void piece(const T* row, int64_t k, int64_t K, float (&v)[kPiece<T>])
{
    numbers<T>(raw_piece<T, VEC>(row, k, K), v);
}

// `past`: results that the L2 cannot hold go past it (kPast).
template <typename T, bool VEC>
__device__ __forceinline__ void put(T* row, int64_t k, int64_t K, const float (&v)[kPiece<T>], int past)
{
    constexpr int E = kPiece<T>;
    if (VEC ? k < K : k + E <= K) {
        piece16 o;
        if constexpr (E == 4) o = piece16{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        else o = piece16{pair_bf16(v[0], v[1]), pair_bf16(v[2], v[3]), pair_bf16(v[4], v[5]), pair_bf16(v[6], v[7])};
        if (past) {
            asm volatile("");                                         // (keeps the two stores from being made one, the ordinary)
            __builtin_nontemporal_store(o, reinterpret_cast<piece16*>(row + k));
            asm volatile("");
        } else {
            *reinterpret_cast<piece16*>(row + k) = o;
        }
    } else if constexpr (!VEC) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (k + e < K) row[k + e] = (T)v[e];
    }
}

template <typename T>
__device__ __forceinline__ void weights(const float* w, int64_t k, int64_t K, float (&v)[kPiece<T>])
{
    constexpr int E = kPiece<T>;
    if (!w) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = 1.0f;
    } else if (k + E <= K) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            const piece16 x = *reinterpret_cast<const piece16*>(w + k + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[e + i] = __uint_as_float(x[i]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = k + e < K ? w[k + e] : 0.0f;
    }
}

// The sum over a row's TPR threads: neighbours in a wavefront, or two or four wavefronts (`room`: four values of this call's own).
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* room)
{
#pragma unroll
    for (int off = (TPR < 64 ? TPR : 64) / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if constexpr (TPR <= 64) return v;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) room[wave] = v;
    __syncthreads();
    if constexpr (TPR == 128) return room[wave & 2] + room[wave | 1];
    return (room[0] + room[1]) + (room[2] + room[3]);
}

// CH pieces of a row per thread; CH == 0: any number, in two passes.
template <typename T, bool VEC, int TPR, int CH>
__global__ __launch_bounds__(256) void norm_kernel(NormArgs p)
{
    constexpr int E = kPiece<T>, RPB = 256 / TPR;
    __shared__ float room[4];
    const int t = threadIdx.x % TPR;
    const int64_t row = p.first + (int64_t)blockIdx.x * RPB + threadIdx.x / TPR, m = min(row, p.M - 1), K = p.K;
    const bool in = row < p.M;                                        // (others take part in sums, and store nothing)
    const T* const x = static_cast<const T*>(p.x) + m * p.ld_x;
    const T* const res = p.residual ? static_cast<const T*>(p.residual) + m * p.ld_residual : nullptr;
    T* const sum = p.sum && in ? static_cast<T*>(p.sum) + m * p.ld_sum : nullptr;
    // columns that are written: codes go on behind the row
    const int64_t span = p.codes ? (p.code_scales ? (K + 31) / 32 * 32 : (K + 15) / 16 * 16) : K;

    auto stream = [&](int64_t k, float (&v)[E]) {
        piece<T, VEC>(x, k, K, v);
        if (res) {
            float u[E];
            piece<T, VEC>(res, k, K, u);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = (float)(T)(v[e] + u[e]);
        }
    };
    float c = 1.0f;
    if (p.codes && !p.code_scales) c = inv_scale(p.scale, p.scale_dev);
    auto finish = [&](int64_t k, const float (&v)[E], float rstd) {
        float w[E], y[E];
        weights<T>(p.w, k, K, w);
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = v[e] * rstd * w[e];
        if (p.y && in) put<T, VEC>(static_cast<T*>(p.y) + m * p.ld_y, k, K, y, p.past);
        if (!p.codes) return;
        uint32_t q[E / 4];
        if (p.code_scales) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (k + e >= K) y[e] = 0.0f;
                top = max(top, __float_as_uint(y[e]) & 0x7fffffffu);
            }
#pragma unroll
            for (int off = 1; off < 32 / E; off <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, 64));
            if (k >= span || !in) return;
            const uint32_t s = block_scale8(top);
            const float i = inverse_scale(s);
            if (k % 32 == 0) p.code_scales[m * (span / 32) + k / 32] = (uint8_t)s;
#pragma unroll
            for (int e = 0; e < E; e += 4) q[e / 4] = codes8(y[e] * i, y[e + 1] * i, y[e + 2] * i, y[e + 3] * i);
        } else {
            if (k >= span || !in) return;
            auto bound = [&](int e) {                                 // (NaN keeps its sign, as in fpq_quantize)
                const float v = __fmul_rn(y[e], c);
                return k + e < K ? copysignf(fminf(fabsf(v), 448.0f), v) : 0.0f;
            };
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                if (p.hardware) {
                    q[e / 4] = codes8(bound(e), bound(e + 1), bound(e + 2), bound(e + 3));
                } else {
                    q[e / 4] = 0;
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        if (k + e + b < K) q[e / 4] |= quantize_nearest(y[e + b], c, p.f) << (8 * b);
                }
            }
        }
        uint8_t* const to = p.codes + m * span + k;
        if constexpr (E == 4) *reinterpret_cast<uint32_t*>(to) = q[0];
        else *reinterpret_cast<uint2*>(to) = make_uint2(q[0], q[1]);
    };

    float ss = 0.0f;
    if constexpr (CH > 0) {
        float v[CH][E];
#pragma unroll
        for (int i = 0; i < CH; ++i) stream((int64_t)(t + TPR * i) * E, v[i]);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
#pragma unroll
            for (int e = 0; e < E; ++e) ss = fmaf(v[i][e], v[i][e], ss);
            if (sum) put<T, VEC>(sum, (int64_t)(t + TPR * i) * E, K, v[i], p.past);
        }
        const float rstd = 1.0f / sqrtf(row_sum<TPR>(ss, room) / (float)K + p.eps);
        if (p.rstd && in && t == 0) p.rstd[m] = rstd;
#pragma unroll
        for (int i = 0; i < CH; ++i) finish((int64_t)(t + TPR * i) * E, v[i], rstd);
    } else {
        const int64_t pieces = (span + E - 1) / E, rounds = (pieces + TPR - 1) / TPR;      // (all lanes take part in every round)
        float v[E];
        for (int64_t i = 0; i < rounds; ++i) {
            const int64_t k = (t + TPR * i) * E;
            stream(k, v);
#pragma unroll
            for (int e = 0; e < E; ++e) ss = fmaf(v[e], v[e], ss);
            if (sum) put<T, VEC>(sum, k, K, v, p.past);
        }
        const float rstd = 1.0f / sqrtf(row_sum<TPR>(ss, room) / (float)K + p.eps);
        if (p.rstd && in && t == 0) p.rstd[m] = rstd;
        for (int64_t i = 0; i < rounds; ++i) {
            const int64_t k = (t + TPR * i) * E;
            if (sum) piece<T, VEC>(sum, k, K, v);
            else stream(k, v);
            finish(k, v, rstd);
        }
    }
}

// Rows blockIdx, blockIdx + gridDim, ... (of 256 / TPR at a time); the columns' sums for the weights' gradient stay with the thread.
template <typename T, bool VEC, int TPR, int CH>
__global__ __launch_bounds__(256) void norm_backward_kernel(NormBackward p, int own_sums)
{
    constexpr int E = kPiece<T>, RPB = 256 / TPR;
    __shared__ float room[2][4];
    __shared__ float all[CH > 0 && RPB > 1 ? 256 * CH * E : 1];
    const int t = threadIdx.x % TPR;
    const int64_t K = p.K;
    const float over = 1.0f / (float)K;
    constexpr int C = CH > 0 ? CH : 1;
    float w[C][E], gw[C][E];
    if constexpr (CH > 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            weights<T>(p.w, (int64_t)(t + TPR * i) * E, K, w[i]);
#pragma unroll
            for (int e = 0; e < E; ++e) gw[i][e] = 0.0f;
        }
    }
    // A row's pieces as they come from memory, a row ahead.
    uint4 rv[C], rg[C], ru[C];
    auto load = [&](int64_t first) {
        const int64_t m = min(first + threadIdx.x / TPR, p.M - 1);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int64_t k = (int64_t)(t + TPR * i) * E;
            rv[i] = raw_piece<T, VEC>(static_cast<const T*>(p.sum) + m * p.ld_sum, k, K);
            rg[i] = raw_piece<T, VEC>(static_cast<const T*>(p.gy) + m * p.ld_gy, k, K);
            ru[i] = p.gs ? raw_piece<T, VEC>(static_cast<const T*>(p.gs) + m * p.ld_gs, k, K) : make_uint4(0, 0, 0, 0);
        }
    };
    const int64_t begin = (int64_t)blockIdx.x * RPB, stride = (int64_t)gridDim.x * RPB;
    if constexpr (CH > 0) load(begin);
    int flip = 0;
    for (int64_t first = begin; first < p.M; first += stride) {
        const int64_t row = first + threadIdx.x / TPR, m = min(row, p.M - 1);
        const bool in = row < p.M;                                    // (others take part in sums, and give nothing)
        const T* const r = static_cast<const T*>(p.sum) + m * p.ld_sum;
        const T* const gy = static_cast<const T*>(p.gy) + m * p.ld_gy;
        const T* const gs = p.gs ? static_cast<const T*>(p.gs) + m * p.ld_gs : nullptr;
        T* const gx = p.gx && in ? static_cast<T*>(p.gx) + m * p.ld_gx : nullptr;
        const float rstd = p.rstd[m];
        auto finish = [&](int64_t k, const float (&g)[E], const float (&v)[E], const float (&u)[E], float c) {
            float o[E];
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(rstd, fmaf(-v[e], c, g[e]), u[e]);
            put<T, VEC>(gx, k, K, o, p.past);
        };
        if constexpr (CH > 0) {
            uint4 nv[C], ng[C], nu[C];
#pragma unroll
            for (int i = 0; i < C; ++i) nv[i] = rv[i], ng[i] = rg[i], nu[i] = ru[i];
            if (first + stride < p.M) load(first + stride);
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                float v[E], g[E];
                numbers<T>(nv[i], v);
                numbers<T>(ng[i], g);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (in) gw[i][e] = fmaf(g[e] * v[e], rstd, gw[i][e]);
                    dot = fmaf(g[e] * w[i][e], v[e], dot);
                }
            }
            const float c = row_sum<TPR>(dot, room[flip]) * over * rstd * rstd;
            flip ^= 1;
            if (gx)
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    float v[E], g[E], u[E];
                    numbers<T>(nv[i], v);
                    numbers<T>(ng[i], g);
                    numbers<T>(nu[i], u);
#pragma unroll
                    for (int e = 0; e < E; ++e) g[e] *= w[i][e];
                    finish((int64_t)(t + TPR * i) * E, g, v, u, c);
                }
        } else {
            const int64_t pieces = (K + E - 1) / E;
            float v[E], g[E], u[E], y[E], dot = 0.0f;
            for (int64_t i = t; i < pieces; i += TPR) {
                piece<T, VEC>(r, i * E, K, v);
                piece<T, VEC>(gy, i * E, K, g);
                weights<T>(p.w, i * E, K, y);
#pragma unroll
                for (int e = 0; e < E; ++e) dot = fmaf(g[e] * y[e], v[e], dot);
            }
            const float c = row_sum<TPR>(dot, room[flip]) * over * rstd * rstd;
            flip ^= 1;
            if (gx)
                for (int64_t i = t; i < pieces; i += TPR) {
                    piece<T, VEC>(r, i * E, K, v);
                    piece<T, VEC>(gy, i * E, K, g);
                    weights<T>(p.w, i * E, K, y);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        g[e] *= y[e];
                        u[e] = 0.0f;
                    }
                    if (gs) piece<T, VEC>(gs, i * E, K, u);
                    finish(i * E, g, v, u, c);
                }
        }
    }
    if constexpr (CH > 0) {
        if (!own_sums) return;
        float* const part = p.part + (int64_t)blockIdx.x * K;
        if constexpr (RPB == 1) {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int64_t k = (int64_t)(t + TPR * i) * E;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (k + e < K) part[k + e] = gw[i][e];
            }
        } else {
            // the workgroup's rows, one after the other: [row][column]
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) all[threadIdx.x / TPR * (TPR * CH * E) + (t + TPR * i) * E + e] = gw[i][e];
            __syncthreads();
            for (int k = threadIdx.x; k < K; k += 256) {
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < RPB; ++r) sum += all[r * (TPR * CH * E) + k];
                part[k] = sum;
            }
        }
    }
}

// The weights' gradient of rows too long for registers: 256 columns per workgroup, a part of the rows.
template <typename T>
__global__ __launch_bounds__(256) void norm_weights_kernel(NormBackward p, int64_t rows)
{
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x, m1 = min(p.M, (int64_t)(blockIdx.y + 1) * rows);
    if (k >= p.K) return;
    float sum = 0.0f;
    for (int64_t m = (int64_t)blockIdx.y * rows; m < m1; ++m)
        sum = fmaf((float)static_cast<const T*>(p.gy)[m * p.ld_gy + k] * (float)static_cast<const T*>(p.sum)[m * p.ld_sum + k], p.rstd[m], sum);
    p.part[(int64_t)blockIdx.y * p.K + k] = sum;
}

// Results larger than the L2 (8 x 4 MB) leave no line of theirs there for a reader, and push the rows that are read out: stored past it, 32768 rows of 320 in
// bf16 take 15.6 us for 19.7, 8192 of 5120 with their gradient 131 for 144.
constexpr int64_t kPast = (int64_t)32 << 20;
constexpr int64_t kMostRowsAtOnce = (int64_t)1 << 23;

// Threads per row and pieces per thread (0: two passes).
struct Shape {
    int tpr, ch;
};
// Widths of 320 2^n and of powers of two leave no thread of a group without a piece: five or four of them each; few rows are spread over more
// threads.  (32768 rows of 320 in bf16: 22.5 us with one piece for 40 of 64 threads, 19.7 with five for eight.)
constexpr Shape kShapes[] = {{8, 4}, {8, 5}, {16, 4}, {16, 5}, {32, 4}, {32, 5}, {64, 4}, {64, 5}, {128, 4}, {128, 5}, {256, 4}, {256, 5}};
constexpr Shape kFewShapes[] = {{64, 1}, {256, 1}, {256, 2}, {256, 4}, {256, 5}};
constexpr Shape kPlainShapes[] = {{64, 1}, {64, 4}, {256, 4}};           // rows that are no whole pieces
constexpr Shape kTwoPasses{256, 0};                                       // rows longer than those
// (the backward kernel holds three tensors' pieces, those of the next row and two rows of sums and weights: no more than three pieces if they suffice)
constexpr Shape kBackwardShapes[] = {{16, 3}, {32, 2}, {32, 3}, {64, 2}, {64, 3}, {128, 2}, {128, 3}, {256, 2}, {256, 3}, {256, 4}, {256, 5}};
Shape shape_of(int64_t M, int64_t span, int piece, bool vec, bool back)
{
    const int64_t pieces = (span + piece - 1) / piece;
    auto first = [&](const auto& list) {
        for (const Shape& s : list)
            if ((int64_t)s.tpr * s.ch >= pieces) return s;
        return kTwoPasses;
    };
    return !vec ? first(kPlainShapes) : M * pieces < 65536 ? first(kFewShapes) : back ? first(kBackwardShapes) : first(kShapes);
}

// Workgroups of the backward kernel, each of which leaves a row of partial sums: of no more than some 2048 rows a thread, as in row_parts.
int64_t backward_blocks(int64_t M, Shape s)
{
    const int64_t rows = 256 / s.tpr, all = (M + rows - 1) / rows, most = all / 2048 > 512 ? all / 2048 : 512;
    return all < most ? all : most;
}

// Runs `run` with the shape's numbers as constants: those of shape_of's own lists, so that each has its kernel.
template <const auto& LIST, int I = 0, typename F>
bool among(Shape s, F&& run)
{
    if constexpr (I < (int)std::size(LIST)) {
        constexpr Shape c = LIST[I];
        if (s.tpr != c.tpr || s.ch != c.ch) return among<LIST, I + 1>(s, run);
        run(std::pair<std::integral_constant<int, c.tpr>, std::integral_constant<int, c.ch>>());
        return true;
    }
    return false;
}
template <bool BACK, bool VEC, typename F>
void with_shape(Shape s, F&& run)
{
    bool found;
    if constexpr (!VEC) found = among<kPlainShapes>(s, run);
    else if constexpr (BACK) found = among<kFewShapes>(s, run) || among<kBackwardShapes>(s, run);
    else found = among<kFewShapes>(s, run) || among<kShapes>(s, run);
    if (!found) run(std::pair<std::integral_constant<int, kTwoPasses.tpr>, std::integral_constant<int, kTwoPasses.ch>>());
}

template <typename T, bool VEC>
int forward(const NormArgs& p, hipStream_t s)
{
    const int64_t span = p.codes ? (p.code_scales ? block_padded(p.K) : padded_channels(p.K)) : p.K;
    const Shape shape = shape_of(p.M, span, kPiece<T>, VEC, false);
    const int64_t rows = 256 / shape.tpr;
    // (a launch has fewer than 2^32 threads)
    for (int64_t first = 0; first < p.M; first += kMostRowsAtOnce) {
        NormArgs q = p;
        q.first = first;
        q.past = p.M * p.K * (int64_t)sizeof(T) * ((p.sum != nullptr) + (p.y != nullptr)) > kPast;
        const dim3 grid((unsigned)(((p.M - first < kMostRowsAtOnce ? p.M - first : kMostRowsAtOnce) + rows - 1) / rows));
        with_shape<false, VEC>(shape, [&](auto c) {
            norm_kernel<T, VEC, decltype(c.first)::value, decltype(c.second)::value><<<grid, dim3(256), 0, s>>>(q);
        });
        if (hipGetLastError() != hipSuccess) return FPQ_ERR_LAUNCH;
    }
    return FPQ_OK;
}

template <typename T, bool VEC>
int backward(const NormBackward& p, hipStream_t s)
{
    if (p.M == 0) return p.gw ? launch_part_sums(p.part, 0, p.K, p.gw, s) : FPQ_OK;
    const Shape shape = shape_of(p.M, p.K, kPiece<T>, VEC, true);
    const int64_t blocks = backward_blocks(p.M, shape);
    const bool own = p.gw && shape.ch;
    const RowParts r = row_parts(p.M, p.K);
    if (p.gw && !own) {                                               // (first: grad_x may be written over gy)
        norm_weights_kernel<T><<<dim3((unsigned)((p.K + 255) / 256), (unsigned)r.parts), dim3(256), 0, s>>>(p, r.rows);
        if (hipGetLastError() != hipSuccess) return FPQ_ERR_LAUNCH;
    }
    if (p.gx || own)
        with_shape<true, VEC>(shape, [&](auto c) {
            NormBackward q = p;
            q.past = p.M * p.K * (int64_t)sizeof(T) > kPast;
            norm_backward_kernel<T, VEC, decltype(c.first)::value, decltype(c.second)::value><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(q, own);
        });
    if (hipGetLastError() != hipSuccess) return FPQ_ERR_LAUNCH;
    return p.gw ? launch_part_sums(p.part, own ? (int)blocks : r.parts, p.K, p.gw, s) : FPQ_OK;
}

}  // namespace

size_t norm_part_bytes(int64_t M, int64_t K)
{
    size_t most = row_parts_bytes(M, K);
    for (int piece : {4, 8})
        for (bool vec : {false, true}) {
            const Shape s = shape_of(M, K, piece, vec, true);
            const size_t n = (size_t)backward_blocks(M, s) * K * 4;
            if (s.ch && n > most) most = n;
        }
    return most;
}

int launch_norm(const NormArgs& p, int type, hipStream_t s)
{
    if (type == FPQ_TYPE_FP32) return p.K % 4 == 0 ? forward<float, true>(p, s) : forward<float, false>(p, s);
    return p.K % 8 == 0 ? forward<__bf16, true>(p, s) : forward<__bf16, false>(p, s);
}

int launch_norm_backward(const NormBackward& p, int type, hipStream_t s)
{
    if (type == FPQ_TYPE_FP32) return p.K % 4 == 0 ? backward<float, true>(p, s) : backward<float, false>(p, s);
    return p.K % 8 == 0 ? backward<__bf16, true>(p, s) : backward<__bf16, false>(p, s);
}

}  // namespace fpq
