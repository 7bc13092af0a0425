// Matrix products: the choice of tile and slices, and the sum of the slices.
#include "matmul_tiles.h"
#include <math.h>

namespace fpq {

namespace {

// Passes of the planes: the largest products of two operands, small ones first.
int passes(int planes_a, int planes_b) { return planes_a * planes_b == 9 ? 6 : planes_a * planes_b; }

// What a call takes, in microseconds: rounds of as many workgroups as run at once, each of steps / slices and what a workgroup needs
// at its start and end.  A step of 64 k takes `full` where the chip is full (1.2 PFLOP/s) and no less than `alone`; a round that is not full, its
// share.  Workgroups of 256 and 192 rows have their compute unit alone; two of 128 rows share one and hide one's waits behind the other, or one with
// a ring of four stages has it alone.  Slices cost the partial results' way to memory and back and a launch.  (Measured: 2048 x 4096 with 64
// steps 1.07 of 192 rows; 1280 x 1280 with 192 steps 1.09 of 256 rows, 0.66 of 128 and 0.43 deep;
// 512 x 1280 with 20 steps 9.0 us in tiles of 64 for 14.4 of 128.)  Operands of three planes each are read
// once for their six products: 4096 x 4096 x 2048 in fp32, both gradients, 666 us for 727.
struct Kind {
    int tile, at_once;
    double full, alone, ends;
};
constexpr Kind kKinds[] = {{kTile256, 256, 1.8, 1.2, 4}, {kTile192, 256, 1.35, 1.05, 4}, {kTile128, 512, 1.08, 0.66, 2}, {kTile128Deep, 256, 0.56, 0.43, 3},
                           {kPlanes256, 256, 0.84, 0.62, 3}, {kPlanes128, 256, 0.5, 0.38, 3}, {kTile64, 512, 0.5, 0.2, 5}};
constexpr Kind kGated64{kTile64, 256, 0.5, 0.24, 5};
constexpr double kLaunch = 4;

int64_t tiles_of(int t, int64_t M, int64_t N, bool gated)
{
    const int64_t columns = tile_n(t, gated) / (gated ? 2 : 1);
    return ((M + kTileM[t] - 1) / kTileM[t]) * ((N + columns - 1) / columns);
}
double steps_of(int64_t K, int planes_a, int planes_b) { return passes(planes_a, planes_b) * (double)((K + 63) / 64); }
bool takes_planes(int t) { return t == kPlanes256 || t == kPlanes128; }
// slices that are tried
int next_slices(int s) { return s < 4 ? s + 1 : s + s / 4; }
double sums_us(int s, int64_t M, int64_t N, bool gated) { return s > 1 ? (double)s * M * N * (gated ? 2 : 1) * 8 / 4.5e6 : 0.0; }

// Workgroups of two lengths (in steps), the long ones first, each where there is room next.  As many as run at once: the short ones share their
// compute units until they end.  More: steps take `full` as long as all units are busy, then `alone`.
double both_us(const Kind& k, int64_t na, double a, int64_t nb, double b)
{
    const int64_t nl = a >= b ? na : nb, ns = a >= b ? nb : na, slots = k.at_once;
    const double l = a >= b ? a : b, s = a >= b ? b : a, share = k.full * (nl + ns) / slots, busy = (nl * l + ns * s) / slots;
    if (nl + ns <= slots) {
        const double us = s * (share > k.alone ? share : k.alone) + (l - s) * k.alone;
        return us > busy * k.full ? us : busy * k.full;
    }
    const int64_t more = nl % slots;                // slots with one long workgroup more than the others
    const double low = (double)(nl / slots) * l, high = low + (more ? l : 0);
    double end = busy > high ? busy : high;
    for (int i = 0; i < 6; ++i) {                   // the next time at which enough short ones have ended
        const double ql = end > low ? floor((end - low) / s + 1e-9) : 0, qh = end > high ? floor((end - high) / s + 1e-9) : 0;
        if ((slots - more) * ql + more * qh >= ns) break;
        const double el = low + (ql + 1) * s, eh = high + (qh + 1) * s;
        end = el < eh || !more ? el : eh;
    }
    return busy * k.full + (end - busy) * k.alone;
}

struct SumArgs {
    const float* part;
    int64_t M, N;
    int slices;
    void* out;
    int64_t ld_out;
    int out_f32;
    const float* bias;
    const float* sums;          // [slice][M], to be added up into sums_out, or null
    float* sums_out;
    Gate gate;
    RowOf rows;                 // of the threads
};

// Four columns of a row per thread; behind them a thread for each row's sum of A.
__device__ __forceinline__ void sum_piece(const SumArgs& p, int64_t id)
{
    const int64_t per = p.rows.per;
    if (id >= p.M * per) {
        const int64_t r = id - p.M * per;
        if (!p.sums || r >= p.M) return;
        float t = 0.0f;
        for (int s = 0; s < p.slices; ++s) t += p.sums[s * p.M + r];
        p.sums_out[r] = t;
        return;
    }
    const int64_t m = row_at(p.rows, id);
    const int n = (int)(id - m * per) * 4;
    const bool all = n + 4 <= p.N;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < p.slices; ++s) {
        const float* const x = p.part + (s * p.M + m) * p.N + n;
        if (all) {
            const piece16 t = *reinterpret_cast<const piece16*>(x);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += __uint_as_float(t[e]);
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
    put4(p.out, m * p.ld_out + n, p.out_f32, n, (int)p.N, v);
}
__global__ __launch_bounds__(256) void matmul_sum_kernel(SumArgs p) { sum_piece(p, (int64_t)blockIdx.x * 256 + threadIdx.x); }
// The first `first` workgroups' and the others'
__global__ __launch_bounds__(256) void matmul_sum_both_kernel(SumArgs x, SumArgs w, unsigned first)
{
    if (blockIdx.x < first) sum_piece(x, (int64_t)blockIdx.x * 256 + threadIdx.x);
    else sum_piece(w, (int64_t)(blockIdx.x - first) * 256 + threadIdx.x);
}

// Four outputs of a row per thread, eight threads a block of 32.
__global__ __launch_bounds__(256) void matmul_sum_gated_kernel(SumArgs p)
{
    const int64_t per = p.rows.per, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const bool in = id < p.M * per;                                  // (whole blocks of lanes)
    const int64_t m = in ? row_at(p.rows, id) : 0;
    const int n = in ? (int)(id - m * per) * 4 : 0, N = (int)p.N;
    float a[4], g[4], v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        a[e] = p.bias && n + e < N ? p.bias[n + e] : 0.0f;
        g[e] = p.bias && n + e < N ? p.bias[N + n + e] : 0.0f;
    }
    const bool all = n + 4 <= N;
    for (int s = 0; s < p.slices; ++s) {
        const float* const x = p.part + (s * p.M + m) * 2 * N + n;
        if (all) {
            const piece16 t = *reinterpret_cast<const piece16*>(x), u = *reinterpret_cast<const piece16*>(x + N);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] += __uint_as_float(t[e]);
                g[e] += __uint_as_float(u[e]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < N) {
                    a[e] += x[e];
                    g[e] += x[N + e];
                }
        }
    }
    const Gate& q = p.gate;
    if (q.pre_scales) {
        uint32_t ta = 0, tg = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= N) a[e] = g[e] = 0.0f;
            ta = max(ta, __float_as_uint(a[e]) & 0x7fffffffu);
            tg = max(tg, __float_as_uint(g[e]) & 0x7fffffffu);
        }
#pragma unroll
        for (int off = 1; off < 8; off <<= 1) {
            ta = max(ta, (uint32_t)__shfl_xor((int)ta, off, 64));
            tg = max(tg, (uint32_t)__shfl_xor((int)tg, off, 64));
        }
        if (in) {
            const uint32_t ea = block_scale8(ta), eg = block_scale8(tg);
            const float ia = inverse_scale(ea), ig = inverse_scale(eg);
            const int np = (N + 31) & ~31;
            uint8_t* const c = static_cast<uint8_t*>(q.pre) + m * (2 * (int64_t)np) + n;
            *reinterpret_cast<uint32_t*>(c) = codes8(a[0] * ia, a[1] * ia, a[2] * ia, a[3] * ia);
            *reinterpret_cast<uint32_t*>(c + np) = codes8(g[0] * ig, g[1] * ig, g[2] * ig, g[3] * ig);
            if (n % 32 == 0) {
                uint8_t* const s = q.pre_scales + m * (2 * (np / 32)) + n / 32;
                s[0] = (uint8_t)ea;
                s[np / 32] = (uint8_t)eg;
            }
        }
    }
    if (!in || n >= N) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = a[e] * gate_of<false>(q.act, g[e], nullptr);
    put4(q.h, m * q.ld_h + n, p.out_f32, n, N, v);
    if (q.pre && !q.pre_scales) {
        put4(q.pre, m * q.ld_pre + n, p.out_f32, n, N, a);
        put4(q.pre, m * q.ld_pre + N + n, p.out_f32, n, N, g);
    }
}

size_t part_bytes(int slices, int64_t M, int64_t N, bool col_a, bool gated)
{
    return slices > 1 ? (size_t)slices * M * (N * (gated ? 2 : 1) + (col_a ? 1 : 0)) * 4 : 0;
}

MatmulArgs args_of(const Product& q, int tile, int slices, void* part)
{
    MatmulArgs p{};
    p.a = q.a;
    p.b = q.b;
    p.M = (int)q.M;
    p.N = (int)q.N;
    p.K = (int)q.K;
    // (small products first)
    if (q.planes_a == 3 && q.planes_b == 3) p.order_a = 0x001102, p.order_b = 0x010120;
    else if (q.planes_a == 3) p.order_a = 0x012;
    else if (q.planes_a == 2) p.order_a = 0x01;
    p.passes = passes(q.planes_a, q.planes_b);
    p.slices = slices;
    const int cols = tile_n(tile, q.gated) / (q.gated ? 2 : 1);
    p.tiles_m = (int)((q.M + kTileM[tile] - 1) / kTileM[tile]);
    p.tiles_n = (int)((q.N + cols - 1) / cols);
    p.out = slices > 1 ? part : q.out;
    p.ld_out = q.ld_out;
    p.out_f32 = q.out_f32;
    p.bias = q.bias;
    // (the partial sums lie behind the partial results)
    p.sums = slices > 1 ? static_cast<float*>(part) + (size_t)slices * q.M * q.N : q.sums;
    p.gate = q.gate;
    return p;
}
SumArgs sum_args_of(const Product& q, int slices, const void* part)
{
    const float* const from = static_cast<const float*>(part);
    return SumArgs{from, q.M, q.N, slices, q.out, q.ld_out, q.out_f32, q.bias, q.sums ? from + (size_t)slices * q.M * q.N : nullptr, q.sums, q.gate,
                   row_of(q.M, q.gated ? (q.N + 31) / 32 * 8 : (q.N + 3) / 4)};
}
unsigned sum_grid(const Product& q)
{
    const int64_t threads = q.gated ? q.M * ((q.N + 31) / 32 * 8) : q.M * ((q.N + 3) / 4) + (q.sums ? q.M : 0);
    return (unsigned)((threads + 255) / 256);
}
int launched() { return hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH; }

}  // namespace

ProductPlan plan_product(int64_t M, int64_t N, int64_t K, int planes_a, int planes_b, bool col_a, bool gated)
{
    const double steps = steps_of(K, planes_a, planes_b);
    if (!col_a && M <= 32) {
        // bound by B's bytes: parts of no fewer than eight steps until two workgroups per compute unit have work
        const int64_t n = tiles_of(kTile32, M, N, gated);
        int64_t most = (int64_t)(steps / 8 < 16 ? steps / 8 : 16), slices = 512 / n < most ? 512 / n : most;
        if (slices < 1) slices = 1;
        const double rounds = (double)(n * slices) / 512;
        return ProductPlan{kTile32, (int)slices, (rounds > 1 ? rounds : 1) * 0.3 * (steps / slices + 5) + (slices > 1 ? kLaunch : 0)};
    }
    ProductPlan best{kTile128, 1, 1e30};
    for (Kind k : kKinds) {
        if (k.tile == kTile192 && col_a) continue;
        if (takes_planes(k.tile) && planes_a * planes_b != 9) continue;
        if (k.tile == kTile64 && gated) k = kGated64;
        for (int s = 1; s <= 32; s = next_slices(s)) {
            if (s > 1 && steps / s < 8) break;
            const int64_t n = tiles_of(k.tile, M, N, gated) * s, rest = n % k.at_once;
            const double part = k.full * rest / k.at_once;
            double us = ((double)(n / k.at_once) * k.full + (rest ? (part > k.alone ? part : k.alone) : 0.0)) * (steps / s + k.ends);
            if (s > 1) us += kLaunch + sums_us(s, M, N, gated);
            if (us < best.us) best = ProductPlan{k.tile, s, us};
        }
    }
    return best;
}

// Both gradients in one launch: their workgroups fill the chip together where neither does alone, and there is a launch less, or two.  (Linear layers in
// bf16 with the blocks made, one after the other and together: 300 x 320 -> 960 18.2 and 14.8 us, 2048 x 1280 -> 1280 38.2 and 33.9, 8192 x 640 -> 640 41.6 and 33.8, 32768 x
// 320 -> 960 98 and 82; gated ones in bf16 without the bias's, 300 x 320 -> 1280 22.6 and 18.2, 2048 x 1280 -> 1280 85 and 72, 2928 x 64 -> 799 36 and 28; with the forward call 999 x
// 333 -> 1283 in fp32 98.7 and 87.5.)
GradientPlan plan_gradients(int64_t M, int64_t N, int64_t K, Planes p)
{
    GradientPlan best{M ? plan_product(M, K, N, p.d, p.w, false, false) : ProductPlan{}, plan_product(N, K, M, p.d, p.x, true, false), -1, 1, 1};
    if (M == 0) return best;
    const double steps_x = steps_of(N, p.d, p.w), steps_w = steps_of(M, p.d, p.x);
    double least = (best.x.us + best.w.us + kLaunch);
    for (const Kind& k : kKinds) {
        if (k.tile != kTile64 && k.tile != kTile128 && k.tile != kTile128Deep && k.tile != kPlanes128) continue;
        if (takes_planes(k.tile) != (p.d * p.x == 9)) continue;
        const int64_t tx = tiles_of(k.tile, M, K, false), tw = tiles_of(k.tile, N, K, false), most = 3 * k.at_once;      // (more parts gain nothing)
        for (int a = 1; a <= 32; a = next_slices(a)) {
            if (a > 1 && (steps_x / a < 8 || tx * a > most)) break;
            for (int b = 1; b <= 32; b = next_slices(b)) {
                if (b > 1 && (steps_w / b < 8 || tx * a + tw * b > most)) break;
                double us = both_us(k, tx * a, steps_x / a + k.ends, tw * b, steps_w / b + k.ends);
                if (a > 1 || b > 1) us += kLaunch + sums_us(a, M, K, false) + sums_us(b, N, K, false);
                if (us < least) {
                    least = us;
                    best.tile = k.tile, best.slices_x = a, best.slices_w = b;
                }
            }
        }
    }
    return best;
}

size_t product_part_bytes(const ProductPlan& plan, int64_t M, int64_t N, bool col_a, bool gated) { return part_bytes(plan.slices, M, N, col_a, gated); }

size_t gradient_part_bytes(const GradientPlan& plan, int64_t M, int64_t N, int64_t K)
{
    const size_t x = part_bytes(plan.x.slices, M, K, false, false), w = part_bytes(plan.w.slices, N, K, true, false);
    const size_t both = plan.tile < 0 ? 0 : part_bytes(plan.slices_x, M, K, false, false) + part_bytes(plan.slices_w, N, K, true, false);
    const size_t one = x > w ? x : w;
    return one > both ? one : both;
}

// Several passes over k read a plane of A more than once, unless there is but one plane of B or a tile takes all in one pass.  And the wavefronts that
// make the sums are slower: in tiles of 256 x 256, of which large products are one round, that is more than a pass for the sums (8192 x 4096 -> 4096
// with both gradients: 500 us, 481 with a pass); elsewhere it is less (5003 x 5120 -> 1280: 176 for 178, 32768 x 320 -> 960 99 for 107, 300 x 320 -> 960 18 for 25).
bool plan_sums(const GradientPlan& plan, int planes_x)
{
    const int tile = plan.w.tile;
    return tile != kTile256 && (planes_x == 1 || tile == kPlanes256 || tile == kPlanes128);
}

int launch_product(const Product& q, const ProductPlan& plan, void* part, hipStream_t s)
{
    if (q.M == 0 || q.N == 0) return FPQ_OK;
    const MatmulArgs p = args_of(q, plan.tile, plan.slices, part);
    const int st = q.gated ? launch_matmul_gated(p, plan.tile, s)
                   : q.col_a ? (q.sums ? launch_matmul_cols_sums(p, plan.tile, s) : launch_matmul_cols(p, plan.tile, s))
                   : q.col_b ? launch_matmul_rows_cols(p, plan.tile, s)
                             : launch_matmul_rows(p, plan.tile, s);
    if (st != FPQ_OK || plan.slices == 1) return st;
    const SumArgs r = sum_args_of(q, plan.slices, part);
    if (q.gated) matmul_sum_gated_kernel<<<dim3(sum_grid(q)), dim3(256), 0, s>>>(r);
    else matmul_sum_kernel<<<dim3(sum_grid(q)), dim3(256), 0, s>>>(r);
    return launched();
}

int launch_products(const Product& x, const Product& w, const GradientPlan& plan, void* part, hipStream_t s)
{
    if (plan.tile < 0) {
        const int st = launch_product(x, plan.x, part, s);
        return st == FPQ_OK ? launch_product(w, plan.w, part, s) : st;
    }
    char* const part_w = static_cast<char*>(part) + part_bytes(plan.slices_x, x.M, x.N, false, false);
    const MatmulArgs ax = args_of(x, plan.tile, plan.slices_x, part), aw = args_of(w, plan.tile, plan.slices_w, part_w);
    const int st = w.sums ? launch_matmul_both_sums(ax, aw, plan.tile, s) : launch_matmul_both(ax, aw, plan.tile, s);
    if (st != FPQ_OK || (plan.slices_x == 1 && plan.slices_w == 1)) return st;
    const unsigned first = plan.slices_x > 1 ? sum_grid(x) : 0, rest = plan.slices_w > 1 ? sum_grid(w) : 0;
    matmul_sum_both_kernel<<<dim3(first + rest), dim3(256), 0, s>>>(sum_args_of(x, plan.slices_x, part), sum_args_of(w, plan.slices_w, part_w), first);
    return launched();
}

}  // namespace fpq
