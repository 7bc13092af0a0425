// Blocks of codes, packing of operands, column sums, the gated projections' elementwise gradient, and the norm: what api_blocks.hip launches.
#pragma once
#include "matmul.h"

namespace fpq {

constexpr int64_t kBlock = 32;
static inline int64_t block_padded(int64_t n) { return (n + kBlock - 1) / kBlock * kBlock; }
static inline int64_t round8(int64_t n) { return (n + 7) / 8 * 8; }

// Matrices for the products, packed in one launch: planes of bf16 rows of whole 16-byte pieces, zeros behind the columns; of fp32 or bf16
// matrices, or of blocks (one plane; `scales`).
struct PackItem {
    const void* src;
    const uint8_t* scales;
    int64_t rows, cols, ld;
    __bf16* dst;
    int64_t ld_dst, plane;
    int64_t first;              // workgroup of the launch
    RowOf pieces;               // of eight elements
    int kind;                   // FPQ_TYPE_FP32, FPQ_TYPE_BF16, or 8 or 4: blocks
};
struct PackList {
    PackItem m[3];
    int count;
};
int launch_packs(PackList& p, hipStream_t s);
// `eight`: E4M3 blocks, else E2M1.
int launch_decode(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, bool eight, void* dst, int f32, int64_t ld_dst, hipStream_t s);
int launch_block_quantize(const void* x, int type, int64_t M, int64_t K, int64_t ld, bool eight, const uint8_t* mask, uint8_t* codes, uint8_t* scales,
                          hipStream_t s);

// Sums over the rows of a matrix, in parts of rows that a second launch adds up in order.
struct RowParts {
    int64_t rows;               // of a part
    int parts;
};
RowParts row_parts(int64_t M, int64_t cols);
size_t row_parts_bytes(int64_t M, int64_t cols);
int launch_column_sums(const void* x, int type, int64_t M, int64_t N, int64_t ld, float* out, float* part, hipStream_t s);
int launch_part_sums(const float* part, int parts, int64_t cols, float* out, hipStream_t s);

// Planes of (da, dg) as operands.  Beside bf16 operands two, 16 significant bits: one would round them by as much as the gradients are rounded
// themselves, errors of 0.0024 of a gradient's norm for 0.0017 (8192 x 1280 -> 5120 with the forward call: 717 us, with two 1166).
static inline int gate_planes(int type) { return type == FPQ_TYPE_FP32 ? 3 : 2; }
// (da, dg) of the gated projections as the products take them, and the bias's gradient.
struct GateBackward {
    int type, act;
    int64_t M, N;
    const void* pre;            // [M, 2 N], or codes
    const uint8_t* pre_scales;
    const void* gh;
    int64_t ld_gh;
    __bf16* d;                  // [plane][M][ld_d]; null: only the sums
    int64_t ld_d, plane;
    float *grad_bias, *part;    // or null
};
int launch_gate_backward(const GateBackward& p, hipStream_t s);

struct NormArgs {
    const void *x, *residual;
    const float* w;
    void *sum, *y;
    float* rstd;
    uint8_t *codes, *code_scales;
    QParams f;
    int hardware;               // f is the hardware's E4M3
    float scale;
    const float* scale_dev;
    int64_t M, K, ld_x, ld_residual, ld_sum, ld_y;
    int64_t first;              // row of a launch
    float eps;
    int past;                   // results are stored past the L2
};
int launch_norm(const NormArgs& p, int type, hipStream_t s);
struct NormBackward {
    const void* sum;
    const float *w, *rstd;
    const void *gy, *gs;
    void* gx;
    float *gw, *part;
    int64_t M, K, ld_sum, ld_gy, ld_gs, ld_gx;
    int past;
};
size_t norm_part_bytes(int64_t M, int64_t K);
int launch_norm_backward(const NormBackward& p, int type, hipStream_t s);

}  // namespace fpq
