// The adapters' kernels (see adapter.h).
#pragma once
#include "adapter.h"

namespace fpq {

// ROWS rows of COLS neighbouring columns on their way from memory to a wavefront's own LDS: neighbouring lanes read neighbouring
// pieces of a row (an operand's lanes read different rows: loaded as operands, every lane's piece is a memory access of its own, and
// their number, not the bytes, is what bounds such a kernel).  LDS rows are 16 bytes longer than whole 64 bytes, so that 16 rows
// start in different banks.
template <typename T, int ROWS, int COLS, bool VEC>
struct WaveTile {
    static constexpr int E = 16 / (int)sizeof(T), CH = COLS / E, N = ROWS * CH, PT = (N + 63) / 64, RS = COLS + E;      // RS: elements of an LDS row
    static constexpr int BYTES = ROWS * RS * (int)sizeof(T);
    v4i reg[PT];
    // row r of the tile is at base + r ld; columns from `dim` on and rows from `rows` on are not read (they hold others' values)
    __device__ __forceinline__ void load(const T* base, unsigned ld, int rows, int col, int dim, int lane)
    {
#pragma unroll
        for (int i = 0; i < PT; ++i) {
            const int id = i * 64 + lane, row = id / CH, c = col + (id - row * CH) * E;
            const unsigned at = (unsigned)min(row, rows - 1) * ld;
            if constexpr (VEC) {
                reg[i] = *reinterpret_cast<const v4i*>(base + (at + (unsigned)min(c, dim - E)));
            } else {
                T v[E];
                v4i w;
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = base[at + (unsigned)min(c + e, dim - 1)];
                __builtin_memcpy(&w, v, 16);
                reg[i] = w;
            }
        }
    }
    __device__ __forceinline__ void store(unsigned char* lds, int lane) const
    {
#pragma unroll
        for (int i = 0; i < PT; ++i) {
            const int id = i * 64 + lane, row = id / CH;
            if (N % 64 != 0 && id >= N) continue;
            *reinterpret_cast<v4i*>(lds + (row * RS + (id - row * CH) * E) * (int)sizeof(T)) = reg[i];
        }
    }
    // Eight columns of a row as an operand; the first `left` of them, the others zero.
    static __device__ __forceinline__ Frag<kPlanes<T>> frag(const unsigned char* lds, int row, int col, int left)
    {
        const uint4* const at = reinterpret_cast<const uint4*>(lds + (row * RS + col) * (int)sizeof(T));
        if constexpr (sizeof(T) == 2) {
            const uint4 w = at[0];
            uint32_t v[4] = {w.x, w.y, w.z, w.w};
            if (left < 8) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = 2 * e + 1 < left ? v[e] : 2 * e < left ? v[e] & 0xffffu : 0u;
            }
            Frag<1> f;
            f.p[0] = __builtin_bit_cast(v8bf, make_uint4(v[0], v[1], v[2], v[3]));
            return f;
        } else {
            const uint4 a = at[0], b = at[1];
            const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(u[e]);
            if (left < 8) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = e < left ? v[e] : 0.0f;
            }
            return frag_of<3>(v);
        }
    }
};

// A wavefront's LDS writes ahead of its reads, and its reads ahead of the next writes (the LDS itself keeps their order).
__device__ __forceinline__ void wave_order() { __builtin_amdgcn_wave_barrier(); }

template <int W>
struct WeightType {
    typedef __bf16 T;
};
template <>
struct WeightType<0> {
    typedef float T;
};

// LDS of a wavefront: a tile of x and one of weights, or the weights of 32 columns of y.
template <typename TX, int W, int RT>
struct MapShape {
    typedef typename WeightType<W>::T TW;
    static constexpr int SC = 128 / (int)sizeof(TX), RC = RT < 4 ? RT : 4;              // columns of a step; groups of 16 ranks staged at once
    typedef WaveTile<TX, 32, SC, true> XT;
    typedef WaveTile<TW, 16 * RC, SC, true> W1T;
    typedef WaveTile<TW, 32, 16 * RC, true> W2T;
    static constexpr int FIRST = XT::BYTES + (W == 3 || W == 2 ? 0 : W1T::BYTES), SECOND = W == 3 || W == 2 ? 0 : W2T::BYTES;
    static constexpr int WAVE = FIRST > SECOND ? FIRST : SECOND;
    static constexpr int RP = 16 * RT + 4;
    static int bytes(int waves)
    {
        const int work = waves * WAVE, sums = (waves + 1) * 32 * RP * 4;                // the sums reuse it; t is behind them
        return work > sums ? work : sums;
    }
};

// Rows through a rank: t = scale1 x W1^T, y = base + scale2 t W2^T, in one pass.  A workgroup takes a tile of 32 rows of one request:
// its wavefronts divide the columns of x in steps of 128 bytes, their sums meet in LDS, and they divide the columns of y, 32 at a
// time, in tiles of the 32 x 32 instruction whose lanes hold neighbouring columns.  t never leaves the workgroup unless it is
// asked for.  Bound by the bytes of the rows, if enough of them are under way: hence two tiles of the base ahead (one: 29 us for 24),
// and nothing loaded behind the stores, which it would wait for.
//   32768 x 320 -> 320, rank 16, fp32 with bf16 weights: 24 us, 5.2 TB/s;  16384 x 320 -> 960, fp32: 35 us, 4.2 TB/s (its gradient
//   24 us);  5003 ragged rows of 1280 -> 5120, rank 64, bf16: 55 us (its gradient 30): 195 workgroups, bound by the latency of a
//   wavefront's tiles and the weights' way through LDS;  64 rows of 1280, an adapter each: 9 us, a launch and three latencies.
// W: 0 fp32 weights, split where they are read; 1 bf16; 2, 3 packed in the order of the operands, bf16 and three
// planes of fp32.
template <typename TX, int W, int RT, int NWV, bool VEC, bool WVEC>
__global__ __launch_bounds__(64 * NWV, NWV == 4 ? 2 : NWV / 4) void adapter_map_kernel(AdapterArgs p)
{
    typedef MapShape<TX, W, RT> Sh;
    typedef typename Sh::TW TW;
    constexpr int NX = kPlanes<TX>, NW = W == 1 || W == 2 ? 1 : 3, SC = Sh::SC, RC = Sh::RC, RP = Sh::RP;
    constexpr bool PACKED = W >= 2;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4, l32 = lane & 31, h = lane >> 5;
    unsigned char* const mine = lds + wave * Sh::WAVE;
    const Rows rows = find_tile<32>(p, blockIdx.x);
    if (rows.lo >= rows.hi) return;
    const int count = rows.hi - rows.lo, R = p.R;
    const bool some = rows.adapter >= 0;
    const size_t adapter = some ? rows.adapter : 0;

    // Element e of a lane in a 32 x 32 tile of y is in row 8 (e / 4) + 4 h + e % 4.  (The row's offset is made where it is used: kept,
    // it would take 32 registers.)
    auto row_at = [&](int e, int ld) {
        asm volatile("" : "+s"(ld));
        return (unsigned)min(8 * (e / 4) + 4 * h + e % 4, count - 1) * (unsigned)ld;
    };
    const TX* const base = p.base ? static_cast<const TX*>(p.base) + (int64_t)rows.lo * p.ld_base : nullptr;
    TX* const y = static_cast<TX*>(p.y) + (int64_t)rows.lo * p.ldy;
    // (kept as they come: a conversion here would be a wait for them)
    struct Base {
        TX v[16];
    } have[2];
    auto load_base = [&](Base& to, int c0) {
        const unsigned col = (unsigned)min(c0 + l32, p.L2 - 1);
        if (base) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (8 * q < count) {
#pragma unroll
                    for (int e = 4 * q; e < 4 * q + 4; ++e) to.v[e] = base[row_at(e, (int)p.ld_base) + col];
                }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) to.v[e] = (TX)0.0f;
        }
    };
    const int part = blockIdx.y, per = ((p.L2 + 31) / 32 + p.parts - 1) / p.parts * 32, end = p.y ? min(p.L2, (part + 1) * per) : 0;
    int c0 = part * per + 32 * wave;
    const int last = end - 1;                                             // (loads behind it are of its column, for nothing)
    if (c0 < end) {
        load_base(have[0], c0);
        load_base(have[1], min(c0 + 32 * NWV, last));
    }

    Frag<3> tf[RT];
    if (some) {
        const TX* const x = static_cast<const TX*>(p.x) + (int64_t)rows.lo * p.ldx;
        const TW* const w1 = static_cast<const TW*>(p.w1.p) + adapter * p.w1.each;
        v4f acc[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int m = 0; m < 2; ++m) acc[r][m] = v4f{0, 0, 0, 0};
        const int steps = (p.L1 + SC - 1) / SC;
        const bool both = count > 16;
        WaveTile<TX, 32, SC, VEC> xt;
        WaveTile<TW, 16 * RC, SC, WVEC> wt;
        auto load_w = [&](int q, int s) {
            if constexpr (!PACKED)
                wt.load(w1 + (size_t)min(16 * RC * q, R - 1) * p.w1.ld, (unsigned)p.w1.ld, max(R - 16 * RC * q, 1), s * SC, p.L1, lane);
        };
        Frag<NW> wp[PACKED ? SC / 32 : 1][PACKED && RT <= 4 ? RT : 1];
        auto load_p = [&](int s) {
            if constexpr (PACKED && RT <= 4) {
#pragma unroll
                for (int k = 0; k < SC / 32; ++k)
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int q = 0; q < NW; ++q)
                            wp[k][r].p[q] = (reinterpret_cast<const v8bf*>(w1) + ((size_t)(s * (SC / 32) + k) * RT + r) * 64 + lane)[q * (p.w1.plane / 8)];
            }
        };
        if (wave < steps) {
            load_p(wave);
            xt.load(x, (unsigned)p.ldx, count, wave * SC, p.L1, lane);
            load_w(0, wave);
        }
        for (int s = wave; s < steps; s += NWV) {
            const int next = min(s + NWV, steps - 1);                     // (loaded for nothing behind the last)
            wave_order();
            xt.store(mine, lane);
            if constexpr (!PACKED) wt.store(mine + Sh::XT::BYTES, lane);
            wave_order();
            xt.load(x, (unsigned)p.ldx, count, next * SC, p.L1, lane);
            load_w(RT > RC ? 1 : 0, RT > RC ? s : next);
            Frag<NX> xf[SC / 32][2];
#pragma unroll
            for (int k = 0; k < SC / 32; ++k)
#pragma unroll
                for (int m = 0; m < 2; ++m)
                    if (m == 0 || both) xf[k][m] = Sh::XT::frag(mine, 16 * m + r16, 32 * k + 8 * g, p.L1 - s * SC - 32 * k - 8 * g);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if constexpr (!PACKED && RT > RC) {
                    if (r > 0 && r % RC == 0) {
                        wave_order();
                        wt.store(mine + Sh::XT::BYTES, lane);
                        wave_order();
                        load_w(r / RC + 1 < RT / RC ? r / RC + 1 : 0, r / RC + 1 < RT / RC ? s : next);
                    }
                }
#pragma unroll
                for (int k = 0; k < SC / 32; ++k) {
                    Frag<NW> wf;
                    if constexpr (PACKED && RT <= 4) {
                        wf = wp[k][r];
                    } else if constexpr (PACKED) {
                        const v8bf* const at = reinterpret_cast<const v8bf*>(w1) + ((size_t)(s * (SC / 32) + k) * RT + r) * 64 + lane;
#pragma unroll
                        for (int q = 0; q < NW; ++q) wf.p[q] = at[q * (p.w1.plane / 8)];
                    } else {
                        wf = Sh::W1T::frag(mine + Sh::XT::BYTES, 16 * (r % RC) + r16, 32 * k + 8 * g, p.L1 - s * SC - 32 * k - 8 * g);
                    }
#pragma unroll
                    for (int m = 0; m < 2; ++m)
                        if (m == 0 || both) mma16<NW, NX>(acc[r][m], wf, xf[k][m]);
                }
            }
            load_p(next);
        }
        // the wavefronts' sums of a value, in order
        float* const sums = reinterpret_cast<float*>(lds);                // [NWV][32][RP], then t: [32][RP]
        float* const ts = sums + NWV * 32 * RP;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int m = 0; m < 2; ++m) *reinterpret_cast<v4f*>(sums + (wave * 32 + 16 * m + r16) * RP + 16 * r + 4 * g) = acc[r][m];
        __syncthreads();
        const float scale1 = p.scale1 ? p.scale1[adapter] : 1.0f, scale2 = p.scale2 ? p.scale2[adapter] : 1.0f;
        for (int id = threadIdx.x; id < 32 * 16 * RT; id += 64 * NWV) {
            const int m = id / (16 * RT), r = id - m * 16 * RT;
            float v = 0.0f;
            if (r < R && m < count) {
#pragma unroll
                for (int w = 0; w < NWV; ++w) v += sums[(w * 32 + m) * RP + r];
                v *= scale1;
                if (p.t && part == 0) p.t[(size_t)(rows.lo + m) * R + r] = v;
                v *= scale2;
            }
            ts[m * RP + r] = v;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < RT; ++k) {
            float v[8];
            *reinterpret_cast<v4f*>(v) = *reinterpret_cast<const v4f*>(ts + l32 * RP + 16 * k + 8 * h);
            *reinterpret_cast<v4f*>(v + 4) = *reinterpret_cast<const v4f*>(ts + l32 * RP + 16 * k + 8 * h + 4);
            tf[k] = frag_of<3>(v);
        }
        __syncthreads();                                                  // (the weights' tiles reuse t's place)
    } else if (p.t && part == 0) {
        for (int id = threadIdx.x; id < count * R; id += 64 * NWV) p.t[(size_t)rows.lo * R + id] = 0.0f;
    }

    // columns of y: the base's values of the wavefront's next two tiles and the weights of the next are on their way
    const TW* const w2 = static_cast<const TW*>(p.w2.p) + adapter * p.w2.each;
    WaveTile<TW, 32, 16 * RC, WVEC> wt;
    auto load_w = [&](int q, int c0) { wt.load(w2 + (size_t)c0 * p.w2.ld, (unsigned)p.w2.ld, p.L2 - c0, 16 * RC * q, R, lane); };
    constexpr int KC = !PACKED ? 1 : RT * NW <= 12 ? RT : 12 / NW;        // packed weights held at once
    Frag<NW> wf[KC];
    auto load_f = [&](int k0, int c0) {
        if constexpr (PACKED) {
            const v8bf* const at = reinterpret_cast<const v8bf*>(w2) + ((size_t)(c0 / 32) * RT + k0) * 64 + lane;
#pragma unroll
            for (int k = 0; k < KC; ++k)
#pragma unroll
                for (int q = 0; q < NW; ++q) wf[k].p[q] = at[k * 64 + q * (p.w2.plane / 8)];
        }
    };
    if (some && c0 < end) {
        if constexpr (PACKED)
            load_f(0, c0);
        else
            load_w(0, c0);
    }
    auto tile = [&](Base& mine_base) {
        const int next = c0 + 32 * NWV < end ? c0 + 32 * NWV : c0;
        v16f acc;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = (float)mine_base.v[e];
        load_base(mine_base, min(c0 + 64 * NWV, last));
        if (some) {
#pragma unroll
            for (int k = 0; k < RT; ++k) {
                if constexpr (PACKED) {
                    mma32<3, NW>(acc, tf[k], wf[k % KC]);
                    // (the next columns' ahead of the stores: a wait for a load is one for all that was issued before it)
                    if (k % KC == KC - 1) load_f(k + 1 < RT ? k + 1 : 0, k + 1 < RT ? c0 : next);
                } else {
                    if (k % RC == 0) {
                        wave_order();
                        wt.store(mine, lane);
                        wave_order();
                        if (k / RC + 1 < RT / RC)
                            load_w(k / RC + 1, c0);
                        else
                            load_w(0, next);
                    }
                    mma32<3, NW>(acc, tf[k], Sh::W2T::frag(mine, l32, 16 * (k % RC) + 8 * h, R - 16 * k - 8 * h));
                }
            }
        }
        const unsigned col = c0 + l32;
        if (col < (unsigned)p.L2) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (8 * q < count) {
#pragma unroll
                    for (int e = 4 * q; e < 4 * q + 4; ++e)
                        if (8 * q + 4 * h + e % 4 < count) y[row_at(e, (int)p.ldy) + col] = (TX)acc[e];
                }
        }
        c0 += 32 * NWV;
    };
    while (c0 < end) {
        tile(have[0]);
        if (c0 < end) tile(have[1]);
    }
}

constexpr int kListed = 512;        // requests that a workgroup looks over at a time

// LDS of the gradients: a tile of x or dy and one of t or dt; two of each, for one barrier per tile instead of two, where three
// workgroups still fit.
template <typename TX, int RT>
struct OuterShape {
    static constexpr int X = kPlanes<TX> * 32 * kRowStride<8>, T = 3 * 32 * kRowStride<RT>, BUFFERS = (X + T) * 2 <= 24 << 10 ? 2 : 1;
    static constexpr int LDS = BUFFERS * (X + T) * 2 + (3 * kListed + 12) * 4;
};

// The gradients of the adapters.  A workgroup has 128 columns of x (B false: dA) or dy (true: dB) and of an adapter's tiles of 32 rows
// its share of p.splits; both kinds are in one launch.  Bound by the latency of a step, not by bytes: hence two tiles under way, and
// the adapter's requests listed once, so that a step finds its rows without a search (38 us with one, 29 without: 5003 ragged rows
// of 1280 and 5120 at rank 64, bf16, whose longest adapter sets the time).  16384 rows of 320 and 960 at rank 16, fp32: 27 us, 3.1 TB/s.
template <typename TX, int RT, bool VEC, bool B>
__device__ __forceinline__ void outer(const OuterArgs& p, unsigned char* lds, int chunk)
{
    constexpr int NX = kPlanes<TX>, CS = kRowStride<8>, RS = kRowStride<RT>;
    typedef OuterShape<TX, RT> Sh;
    __bf16* const tiles = reinterpret_cast<__bf16*>(lds);                // [BUFFERS] x [NX][32][CS], t [3][32][RS]
    int* const upto = reinterpret_cast<int*>(tiles + Sh::BUFFERS * (Sh::X + Sh::T));
    int* const first = upto + kListed + 1;           // this adapter's requests: upto [kListed + 1] tiles ahead of it, rows from first to behind
    int* const behind = first + kListed;
    int* const wsum = behind + kListed;              // [8]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, g = lane >> 4;
    const int L = p.L[B], R = p.R, c0 = chunk * 128, adapter = blockIdx.y, split = blockIdx.z;
    const TX* const x = static_cast<const TX*>(p.rows[B]) + c0;
    const int64_t ld = p.ld[B];
    const float* const t = p.t[B];
    v4f acc[2][RT];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[c][r] = v4f{0, 0, 0, 0};
    struct Tile {
        Stage<TX, 8, VEC, 32, 256> sx;
        Stage<float, RT, VEC, 32, 256> st;
        int lo, hi;
    } ahead[2];                                      // the two tiles on their way
    for (int q0 = 1; q0 <= p.requests; q0 += kListed) {
        __syncthreads();
        int before = 0, listed = 0;                  // tiles and requests of this adapter so far
        for (int part = 0; part < kListed; part += 256) {
            const int v = q0 + part + tid;
            Rows r = {0, 0, -1};
            if (v <= p.requests) r = rows_of(p, v);
            const int has = r.adapter == adapter ? (r.hi - r.lo + 31) / 32 : 0, sum = scan64(has), count = scan64(has > 0);
            if (lane == 63) {
                wsum[wave] = sum;
                wsum[4 + wave] = count;
            }
            __syncthreads();
            int at = listed + count - (has > 0), ahead_of = before + sum - has;
            for (int w = 0; w < 4; ++w) {
                if (w < wave) {
                    ahead_of += wsum[w];
                    at += wsum[4 + w];
                }
                before += wsum[w];
                listed += wsum[4 + w];
            }
            if (has > 0) {
                upto[at] = ahead_of;
                first[at] = r.lo;
                behind[at] = r.hi;
            }
            __syncthreads();
        }
        if (tid == 0) upto[listed] = before;
        __syncthreads();
        const int tbeg = (int)((int64_t)before * split / p.splits), tend = (int)((int64_t)before * (split + 1) / p.splits);
        int a = 0;                                   // upto[a] <= tbeg < upto[a + 1]; from there on one by one
        for (int b = listed; b - a > 1;) {
            const int m = (a + b) >> 1;
            if (upto[m] <= tbeg)
                a = m;
            else
                b = m;
        }
        int from = 0, next = 0, row0 = 0, end = 0;
        if (tbeg < tend) from = upto[a], next = upto[a + 1], row0 = first[a], end = behind[a];
        auto load = [&](Tile& its, int tile) {
            if (tile >= next) {
                ++a;
                from = next, next = upto[a + 1], row0 = first[a], end = behind[a];
            }
            its.lo = row0 + (tile - from) * 32;
            its.hi = min(end, its.lo + 32);
            its.sx.load(x, ld, its.lo, its.hi - 1, L - c0, tid);
            its.st.load(t, R, its.lo, its.hi - 1, R, tid);
        };
        auto step = [&](Tile& its, int tile, int buffer) {
            __bf16* const xt = tiles + (Sh::BUFFERS == 2 ? buffer : 0) * (Sh::X + Sh::T);
            __bf16* const tt = xt + Sh::X;
            if (Sh::BUFFERS == 1) __syncthreads();
            its.sx.store(xt, its.lo, its.hi, L - c0, tid);
            its.st.store(tt, its.lo, its.hi, R, tid);
            __syncthreads();
            if (tile + 2 < tend) load(its, tile + 2);
            Frag<NX> xf[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) xf[c] = col_frag16<NX>(xt, CS, 32 * CS, 0, 32 * wave + 16 * c, lane);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const Frag<3> tf = col_frag16<3>(tt, RS, 32 * RS, 0, 16 * r, lane);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if constexpr (B)
                        mma16<NX, 3>(acc[c][r], xf[c], tf);              // lane: rank r16, columns 4 g + i
                    else
                        mma16<3, NX>(acc[c][r], tf, xf[c]);              // lane: column r16, ranks 4 g + i
                }
            }
        };
        if (tbeg < tend) load(ahead[0], tbeg);
        if (tbeg + 1 < tend) load(ahead[1], tbeg + 1);
        for (int tile = tbeg; tile < tend; tile += 2) {
            step(ahead[0], tile, 0);
            if (tile + 1 < tend) step(ahead[1], tile + 1, 1);
        }
    }
    const float scale = B ? p.scaling[adapter] : 1.0f;
    float* const out = p.out[B] + (size_t)split * p.adapters * L * R + (size_t)adapter * L * R;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int col = c0 + 32 * wave + 16 * c + (B ? 4 * g + e : r16), rank = 16 * r + (B ? r16 : 4 * g + e);
                if (col >= L || rank >= R) continue;
                out[B ? (size_t)col * R + rank : (size_t)rank * L + col] = scale * acc[c][r][e];
            }
}

template <typename TX, int RT, bool VEC>
__global__ __launch_bounds__(256) void adapter_outer_kernel(OuterArgs p)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char outer_lds[];
    const int chunks_a = (p.L[0] + 127) / 128;
    if ((int)blockIdx.x < chunks_a)
        outer<TX, RT, VEC, false>(p, outer_lds, blockIdx.x);
    else
        outer<TX, RT, VEC, true>(p, outer_lds, blockIdx.x - chunks_a);
}

template <typename TX, int W, int RT, int NWV, bool VEC, bool WVEC>
int launch_map(const AdapterArgs& a, hipStream_t s)
{
    const int lds = MapShape<TX, W, RT>::bytes(NWV);
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&adapter_map_kernel<TX, W, RT, NWV, VEC, WVEC>), lds, done)) return FPQ_ERR_LAUNCH;
    const int64_t tiles = (int64_t)a.M / 32 + a.requests + 2;
    adapter_map_kernel<TX, W, RT, NWV, VEC, WVEC><<<dim3((unsigned)tiles, a.y ? a.parts : 1), dim3(64 * NWV), lds, s>>>(a);
    return FPQ_OK;
}

template <typename TX, int W, int RT, int NWV>
int map_of_tile(const AdapterArgs& a, hipStream_t s)
{
    if (a.w1.vec && a.w2.vec) return a.vec_x ? launch_map<TX, W, RT, NWV, true, true>(a, s) : launch_map<TX, W, RT, NWV, false, true>(a, s);
    if constexpr (W >= 2 || RT > kPlainRank / 16)
        return FPQ_ERR_UNSUPPORTED;                  // (the weights are packed then)
    else
        return a.vec_x ? launch_map<TX, W, RT, NWV, true, false>(a, s) : launch_map<TX, W, RT, NWV, false, false>(a, s);
}

template <typename TX, int W, int RT>
int map_of_rank(const AdapterArgs& a, int waves, hipStream_t s)
{
    constexpr int many = RT == 1 ? 16 : 8;                                // (registers)
    return waves == 16 ? map_of_tile<TX, W, RT, many>(a, s) : map_of_tile<TX, W, RT, 4>(a, s);
}

template <typename TX, int W>
int launch_map(const AdapterArgs& a, int waves, hipStream_t s)
{
    const int st = a.R <= 16 ? map_of_rank<TX, W, 1>(a, waves, s) : a.R <= 32 ? map_of_rank<TX, W, 2>(a, waves, s)
                 : a.R <= 64 ? map_of_rank<TX, W, 4>(a, waves, s) : map_of_rank<TX, W, 8>(a, waves, s);
    return st != FPQ_OK ? st : hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

template <typename TX, int RT, bool VEC>
int launch_outer(const OuterArgs& a, hipStream_t s)
{
    constexpr int lds = OuterShape<TX, RT>::LDS;
    static std::atomic<uint64_t> done{0};
    if (!allow_dynamic_lds(reinterpret_cast<const void*>(&adapter_outer_kernel<TX, RT, VEC>), lds, done)) return FPQ_ERR_LAUNCH;
    const int chunks = (a.L[0] + 127) / 128 + (a.L[1] + 127) / 128;
    adapter_outer_kernel<TX, RT, VEC><<<dim3(chunks, a.adapters, a.splits), dim3(256), lds, s>>>(a);
    return FPQ_OK;
}

template <typename TX, bool VEC>
int launch_outer(const OuterArgs& a, hipStream_t s)
{
    const int st = a.R <= 16 ? launch_outer<TX, 1, VEC>(a, s) : a.R <= 32 ? launch_outer<TX, 2, VEC>(a, s) : a.R <= 64 ? launch_outer<TX, 4, VEC>(a, s)
                                                                                                            : launch_outer<TX, 8, VEC>(a, s);
    return st != FPQ_OK ? st : hipGetLastError() == hipSuccess ? FPQ_OK : FPQ_ERR_LAUNCH;
}

}  // namespace fpq
