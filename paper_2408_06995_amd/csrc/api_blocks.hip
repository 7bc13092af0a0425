// C ABI of the operators around a transformer block's projections (see include/fpq.h): blocks of codes, layers on them, gradients of linear
// layers, gated projections, the norm.  Argument validation on the host, then kernel launches on the caller's stream.
#include <math.h>

#include "blocks.h"
#include "rows.h"

using namespace fpq;

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 28, kMostColumns = (int64_t)1 << 20, kMostElements = (int64_t)1 << 34;

size_t align_up(size_t v) { return (v + 255) / 256 * 256; }
size_t size_of(int type) { return type == FPQ_TYPE_FP32 ? 4 : 2; }
int planes_of(int type) { return type == FPQ_TYPE_FP32 ? 3 : 1; }
bool type_ok(int type) { return type == FPQ_TYPE_FP32 || type == FPQ_TYPE_BF16; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
bool stride_ok(int64_t ld, int64_t cols, int64_t rows) { return rows <= 1 || (ld >= cols && ld <= kMostColumns); }
// (a single row's stride says nothing)
int64_t stride(int64_t ld, int64_t cols, int64_t rows) { return rows <= 1 ? (cols + 7) / 8 * 8 : ld; }

int check_sizes(int64_t M, int64_t N, int64_t K)
{
    if (M < 0 || M > kMostRows || N < 1 || N > kMostColumns || K < 1 || K > kMostColumns) return FPQ_ERR_SHAPE;
    if (M * N >= kMostElements || M * K >= kMostElements || N * K >= kMostElements) return FPQ_ERR_SHAPE;
    return FPQ_OK;
}

// Which blocks a format says: 8, 4, or a status
int block_bits(fpq_format_t f)
{
    if (fpq_format_check(f) != FPQ_OK) return FPQ_ERR_FORMAT;
    if (f.ebits == 4 && f.mbits == 3 && f.bias == 7 && f.maxval == 448.0f) return 8;
    if (f.ebits == 2 && f.mbits == 1 && f.bias == 1 && (f.maxval == 0.0f || f.maxval == 6.0f)) return 4;
    return FPQ_ERR_UNSUPPORTED;
}

// The workspace, piece by piece.
struct Room {
    char* at;
    template <typename T>
    T* take(size_t bytes)
    {
        T* const r = reinterpret_cast<T*>(at);
        at += align_up(bytes);
        return r;
    }
};

// Room for a matrix that the products cannot read as it is.
size_t planes_bytes(int64_t rows, int64_t cols, int planes) { return align_up((size_t)rows * round8(cols) * 2 * planes); }
size_t blocks_bytes(int64_t rows, int64_t cols) { return align_up((size_t)rows * block_padded(cols) * 2); }
bool reads(const void* p, int type, int64_t rows, int64_t cols, int64_t ld)
{
    return type == FPQ_TYPE_BF16 && aligned(p, 16) && cols % 8 == 0 && (rows <= 1 || ld % 8 == 0);
}

// A matrix as the products read it: where it is, or packed into the workspace by the launch that `packs` is collected for.
Operand operand(const void* p, int type, int64_t rows, int64_t cols, int64_t ld, Room& room, PackList& packs)
{
    ld = stride(ld, cols, rows);
    if (reads(p, type, rows, cols, ld)) return Operand{static_cast<const __bf16*>(p), ld, 0};
    const int64_t to = round8(cols);
    __bf16* const dst = room.take<__bf16>((size_t)rows * to * 2 * planes_of(type));
    packs.m[packs.count++] = PackItem{p, nullptr, rows, cols, ld, dst, to, rows * to, 0, {}, type};
    return Operand{dst, to, rows * to};
}
Operand operand_of_blocks(const void* codes, const uint8_t* scales, int64_t rows, int64_t cols, int bits, Room& room, PackList& packs)
{
    const int64_t to = block_padded(cols);
    __bf16* const dst = room.take<__bf16>((size_t)rows * to * 2);
    packs.m[packs.count++] = PackItem{codes, scales, rows, to, to, dst, to, 0, 0, {}, bits};
    return Operand{dst, to, 0};
}

bool workspace_bad(const void* workspace, size_t bytes, size_t need, int* st)
{
    *st = need && (!workspace || bytes < need) ? FPQ_ERR_WORKSPACE : need && !aligned(workspace, 16) ? FPQ_ERR_ALIGN : FPQ_OK;
    return *st != FPQ_OK;
}

size_t larger(size_t a, size_t b) { return a > b ? a : b; }

// The plans of grad_x [M, K] = d [M, N] w and grad_w [N, K] = d^T x: for x in its type and in blocks, of which a call takes one and its workspace's size the
// larger.  Products that follow each other share the room of partial results.
struct GradientPlans {
    GradientPlan values, blocks;
    size_t parts;
};
GradientPlans plans_of(int64_t M, int64_t N, int64_t K, int planes_d, int planes)
{
    GradientPlans p;
    p.values = plan_gradients(M, N, K, {planes_d, planes, planes});
    p.blocks = planes == 1 ? p.values : plan_gradients(M, N, K, {planes_d, planes, 1});
    p.parts = align_up(larger(gradient_part_bytes(p.values, M, N, K), gradient_part_bytes(p.blocks, M, N, K)));
    return p;
}
size_t linear_backward_bytes(int64_t M, int64_t N, int64_t K, int type, const GradientPlans& plans)
{
    const int p = planes_of(type);
    return planes_bytes(M, N, p) + planes_bytes(N, K, p) + larger(planes_bytes(M, K, p), blocks_bytes(M, K)) + larger(plans.parts, align_up(row_parts_bytes(M, N)));
}
size_t gated_backward_bytes(int64_t M, int64_t N, int64_t K, int type, const GradientPlans& plans)
{
    const int p = planes_of(type), pd = gate_planes(type);
    return planes_bytes(M, 2 * N, pd) + planes_bytes(2 * N, K, p) + larger(planes_bytes(M, K, p), blocks_bytes(M, K)) +
           larger(plans.parts, align_up(2 * row_parts_bytes(M, N)));
}

// The products of both gradients.  d: [M, N] in planes_d planes as the products read it, or to be packed with the others; x or its blocks; grad_x, grad_w may be null.
// grad_bias: the sums of d beside grad_w, or null.
int gradients(const Operand& d, int planes_d, int type, int64_t M, int64_t N, int64_t K, const void* x, const uint8_t* x_scales, int64_t ld_x, const void* w, int64_t ld_w,
              void* grad_x, int64_t ld_grad_x, void* grad_w, int64_t ld_grad_w, float* grad_bias, const GradientPlan& plan, Room& room, PackList& packs, hipStream_t s)
{
    const int np = planes_of(type);
    Operand ow{}, ox{};
    if (grad_x && M) ow = operand(w, type, N, K, ld_w, room, packs);
    if (grad_w && M) ox = x_scales ? operand_of_blocks(x, x_scales, M, K, 8, room, packs) : operand(x, type, M, K, ld_x, room, packs);
    int st = packs.count ? launch_packs(packs, s) : FPQ_OK;
    if (st != FPQ_OK) return st;
    Product px{}, pw{};
    px.a = pw.a = d;
    px.planes_a = pw.planes_a = planes_d;
    px.out_f32 = pw.out_f32 = type == FPQ_TYPE_FP32;
    px.col_b = pw.col_b = pw.col_a = true;
    px.b = ow;
    px.M = M;
    px.N = K;
    px.K = N;
    px.planes_b = np;
    px.out = grad_x;
    px.ld_out = stride(ld_grad_x, K, M);
    pw.b = ox;
    pw.M = N;
    pw.N = K;
    pw.K = M;
    pw.planes_b = x_scales ? 1 : np;
    pw.out = grad_w;
    pw.ld_out = stride(ld_grad_w, K, N);
    pw.sums = grad_bias;
    if (grad_x && grad_w && M) return launch_products(px, pw, plan, room.at, s);
    if (grad_x && M) return launch_product(px, plan.x, room.at, s);
    return grad_w ? launch_product(pw, plan.w, room.at, s) : FPQ_OK;
}

// What both backward calls ask of x, w and the gradients
int check_gradients(int type, int64_t M, int64_t N, int64_t K, const void* x, const uint8_t* x_scales, int64_t ld_x, const void* w, int64_t ld_w,
                    const void* grad_x, int64_t ld_grad_x, const void* grad_w, int64_t ld_grad_w, const float* grad_bias)
{
    if (M && ((grad_w && !x) || (grad_x && !w))) return FPQ_ERR_NULL;
    if (grad_x && (!stride_ok(ld_grad_x, K, M) || !stride_ok(ld_w, K, N))) return FPQ_ERR_SHAPE;
    if (grad_w && (!stride_ok(ld_grad_w, K, N) || (!x_scales && !stride_ok(ld_x, K, M)))) return FPQ_ERR_SHAPE;
    const size_t size = size_of(type);
    if (!aligned(x, x_scales ? 16 : size) || !aligned(w, size) || !aligned(grad_x, size) || !aligned(grad_w, size) || !aligned(grad_bias, 4)) return FPQ_ERR_ALIGN;
    return FPQ_OK;
}

RowsArgs rows_args(const void* x, int type, int64_t M, int64_t N, int64_t K, int64_t ld_x, const float* bias)
{
    RowsArgs r{};
    r.x = x;
    r.ld_x = stride(ld_x, K, M);
    r.M = (int)M;
    r.N = (int)N;
    r.K = (int)K;
    r.bias = bias;
    r.f32 = type == FPQ_TYPE_FP32;
    return r;
}

// Whether the form of few rows takes gated projections: weights read where they are.  In bf16 up to 16 rows, more only of weights that the L2 holds: in
// 64 rows their share of the matrix unit and x again in every workgroup cost more than the tiles' rows without a result (48 rows of 4096 -> 10240:
// 55.8 us, in tiles 36.4; of 1280 -> 5120: 14.2 and 16.2).  In fp32 tiles have to pack the weights first (64 rows of 4096 -> 10240: 143 us, in tiles 281).
bool few_rows(int64_t M, int64_t N, int64_t K, int type)
{
    return M <= kFewRows && (type == FPQ_TYPE_FP32 || M <= 16 || 4 * N * K <= (int64_t)32 << 20);
}

int check_norm(const fpq_norm_args_t* p)
{
    if (!p) return FPQ_ERR_NULL;
    if (!type_ok(p->type)) return FPQ_ERR_UNSUPPORTED;
    return check_sizes(p->M, 1, p->K);
}

}  // namespace

extern "C" {

int64_t fpq_block_padded(int64_t n) { return n < 0 ? 0 : block_padded(n); }

int fpq_block_quantize(const void* x, int x_type, int64_t M, int64_t K, int64_t ld_x, fpq_format_t f, const uint8_t* mask, uint8_t* codes, uint8_t* scales,
                       void* stream)
{
    const int bits = block_bits(f);
    if (bits < 0) return bits;
    if (!type_ok(x_type) || (mask && bits != 4)) return FPQ_ERR_UNSUPPORTED;
    int st = check_sizes(M, 1, K);
    if (st != FPQ_OK) return st;
    if (M == 0) return FPQ_OK;
    if (!x || !codes || !scales) return FPQ_ERR_NULL;
    if (!stride_ok(ld_x, K, M)) return FPQ_ERR_SHAPE;
    if (!aligned(x, size_of(x_type)) || !aligned(codes, 16)) return FPQ_ERR_ALIGN;
    return launch_block_quantize(x, x_type, M, K, stride(ld_x, K, M), bits == 8, mask, codes, scales, static_cast<hipStream_t>(stream));
}

int fpq_block_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K, fpq_format_t f, void* out, int out_type, int64_t ld_out, void* stream)
{
    const int bits = block_bits(f);
    if (bits < 0) return bits;
    if (!type_ok(out_type)) return FPQ_ERR_UNSUPPORTED;
    int st = check_sizes(M, 1, K);
    if (st != FPQ_OK) return st;
    if (M == 0) return FPQ_OK;
    if (!codes || !scales || !out) return FPQ_ERR_NULL;
    if (!stride_ok(ld_out, K, M)) return FPQ_ERR_SHAPE;
    if (!aligned(out, size_of(out_type)) || !aligned(codes, 16)) return FPQ_ERR_ALIGN;
    return launch_decode(codes, scales, M, K, bits == 8, out, out_type == FPQ_TYPE_FP32, stride(ld_out, K, M), static_cast<hipStream_t>(stream));
}

static size_t block_linear_bytes(int64_t M, int64_t N, int64_t K, int type, const ProductPlan& plan)
{
    return planes_bytes(M, K, planes_of(type)) + blocks_bytes(N, K) + align_up(product_part_bytes(plan, M, N, false, false));
}

size_t fpq_block_linear_workspace_size(int64_t M, int64_t N, int64_t K, int type)
{
    if (!type_ok(type) || check_sizes(M, N, K) != FPQ_OK || M <= kFewRows) return 0;
    return block_linear_bytes(M, N, K, type, plan_product(M, N, K, planes_of(type), 1, false, false));
}

int fpq_block_linear(const fpq_linear_args_t* p, const void* x, const uint8_t* codes, const uint8_t* scales, const float* bias, void* y, void* workspace,
                     size_t workspace_bytes, void* stream)
{
    if (!p) return FPQ_ERR_NULL;
    if (!type_ok(p->type) || p->reserved) return FPQ_ERR_UNSUPPORTED;
    int st = check_sizes(p->M, p->N, p->K);
    if (st != FPQ_OK) return st;
    if (p->M == 0) return FPQ_OK;
    if (!x || !codes || !scales || !y) return FPQ_ERR_NULL;
    if (!stride_ok(p->ld_x, p->K, p->M) || !stride_ok(p->ld_y, p->N, p->M)) return FPQ_ERR_SHAPE;
    const size_t size = size_of(p->type);
    if (!aligned(x, size) || !aligned(y, size) || !aligned(codes, 16) || !aligned(bias, 4)) return FPQ_ERR_ALIGN;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (p->M <= kFewRows) {
        RowsArgs r = rows_args(x, p->type, p->M, p->N, p->K, p->ld_x, bias);
        const int64_t kp = block_padded(p->K);
        r.w = codes;
        r.ld_w = kp / 2;
        r.scales = scales;
        r.ld_s = kp / kBlock;
        r.out = y;
        r.ld_out = stride(p->ld_y, p->N, p->M);
        return p->M <= (r.f32 ? 4 : 2) && token_blocks_lds(p->M, p->K, r.f32) <= 65536 ? launch_token_blocks(r, s) : launch_rows_blocks(r, s);
    }
    const ProductPlan plan = plan_product(p->M, p->N, p->K, planes_of(p->type), 1, false, false);
    if (workspace_bad(workspace, workspace_bytes, block_linear_bytes(p->M, p->N, p->K, p->type, plan), &st)) return st;
    Room room{static_cast<char*>(workspace)};
    PackList packs{};
    Product q{};
    q.a = operand(x, p->type, p->M, p->K, p->ld_x, room, packs);
    q.b = operand_of_blocks(codes, scales, p->N, p->K, 4, room, packs);
    st = launch_packs(packs, s);
    if (st != FPQ_OK) return st;
    q.M = p->M;
    q.N = p->N;
    q.K = p->K;
    q.planes_a = planes_of(p->type);
    q.planes_b = 1;
    q.out = y;
    q.ld_out = stride(p->ld_y, p->N, p->M);
    q.out_f32 = p->type == FPQ_TYPE_FP32;
    q.bias = bias;
    return launch_product(q, plan, room.at, s);
}

size_t fpq_linear_backward_workspace_size(int64_t M, int64_t N, int64_t K, int type)
{
    if (!type_ok(type) || check_sizes(M, N, K) != FPQ_OK) return 0;
    return linear_backward_bytes(M, N, K, type, plans_of(M, N, K, planes_of(type), planes_of(type)));
}

int fpq_linear_backward(const fpq_linear_args_t* p, const void* x, const uint8_t* x_scales, const void* w, const void* grad_y, void* grad_x, void* grad_w,
                        float* grad_bias, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!p) return FPQ_ERR_NULL;
    if (!type_ok(p->type) || p->reserved) return FPQ_ERR_UNSUPPORTED;
    const int64_t M = p->M, N = p->N, K = p->K;
    int st = check_sizes(M, N, K);
    if (st != FPQ_OK) return st;
    if (M && !grad_y) return FPQ_ERR_NULL;
    if (!stride_ok(p->ld_grad_y, N, M)) return FPQ_ERR_SHAPE;
    if (!aligned(grad_y, size_of(p->type))) return FPQ_ERR_ALIGN;
    st = check_gradients(p->type, M, N, K, x, x_scales, p->ld_x, w, p->ld_w, grad_x, p->ld_grad_x, grad_w, p->ld_grad_w, grad_bias);
    if (st != FPQ_OK) return st;
    const int np = planes_of(p->type);
    const GradientPlans plans = plans_of(M, N, K, np, np);
    if (workspace_bad(workspace, workspace_bytes, linear_backward_bytes(M, N, K, p->type, plans), &st)) return st;
    const GradientPlan& plan = x_scales ? plans.blocks : plans.values;
    hipStream_t s = static_cast<hipStream_t>(stream);
    Room room{static_cast<char*>(workspace)};
    // The bias's gradient comes with the weights' where their product gives both, else from a pass of its own.
    const bool both = grad_bias && grad_w && ((grad_x && plan.tile >= 0) || plan_sums(plan, x_scales ? 1 : np));
    if (grad_bias && !both) st = launch_column_sums(grad_y, p->type, M, N, stride(p->ld_grad_y, N, M), grad_bias, reinterpret_cast<float*>(room.at), s);
    if (st != FPQ_OK || (!grad_x && !grad_w)) return st;
    PackList packs{};
    Operand d{};
    if (M) d = operand(grad_y, p->type, M, N, p->ld_grad_y, room, packs);
    return gradients(d, np, p->type, M, N, K, x, x_scales, p->ld_x, w, p->ld_w, grad_x, p->ld_grad_x, grad_w, p->ld_grad_w, both ? grad_bias : nullptr, plan, room, packs, s);
}

static int check_gated(const fpq_gated_args_t* p)
{
    if (!p) return FPQ_ERR_NULL;
    if (!type_ok(p->type) || (p->act != FPQ_GATE_SILU && p->act != FPQ_GATE_GELU)) return FPQ_ERR_UNSUPPORTED;
    return check_sizes(p->M, 2 * (p->N < 0 ? 0 : p->N > kMostColumns ? kMostColumns : p->N), p->K);
}

static size_t gated_bytes(int64_t M, int64_t N, int64_t K, int type, const ProductPlan& plan)
{
    const int p = planes_of(type);
    return planes_bytes(M, K, p) + planes_bytes(2 * N, K, p) + align_up(product_part_bytes(plan, M, N, false, true));
}

size_t fpq_gated_workspace_size(int64_t M, int64_t N, int64_t K, int type)
{
    const fpq_gated_args_t a{type, 0, M, N, K, 0, 0, 0, 0, 0, 0};
    if (check_gated(&a) != FPQ_OK || M <= 16) return 0;
    // (nothing is kept there by the form of few rows; from 17 rows on, which form runs changes how large a workspace has to be, not whether there is one)
    if (few_rows(M, N, K, type)) return align_up(1);
    return gated_bytes(M, N, K, type, plan_product(M, N, K, planes_of(type), planes_of(type), false, true));
}

int fpq_gated(const fpq_gated_args_t* p, const void* x, const void* w, const float* bias, void* h, void* pre, uint8_t* pre_scales, void* workspace,
              size_t workspace_bytes, void* stream)
{
    int st = check_gated(p);
    if (st != FPQ_OK) return st;
    const int64_t M = p->M, N = p->N, K = p->K;
    if (M == 0) return FPQ_OK;
    if (!x || !w || !h || (pre_scales && !pre)) return FPQ_ERR_NULL;
    if (!stride_ok(p->ld_x, K, M) || !stride_ok(p->ld_w, K, 2 * N) || !stride_ok(p->ld_h, N, M)) return FPQ_ERR_SHAPE;
    const size_t size = size_of(p->type);
    if (!aligned(x, size) || !aligned(w, size) || !aligned(h, size) || !aligned(pre, pre_scales ? 16 : size) || !aligned(bias, 4)) return FPQ_ERR_ALIGN;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (few_rows(M, N, K, p->type)) {
        if (workspace_bad(workspace, workspace_bytes, fpq_gated_workspace_size(M, N, K, p->type), &st)) return st;
        RowsArgs r = rows_args(x, p->type, M, N, K, p->ld_x, bias);
        r.w = w;
        r.ld_w = p->ld_w;
        r.gate = Gate{p->act, h, stride(p->ld_h, N, M), pre, 2 * N, pre_scales};
        return launch_rows_gated(r, s);
    }
    const ProductPlan plan = plan_product(M, N, K, planes_of(p->type), planes_of(p->type), false, true);
    if (workspace_bad(workspace, workspace_bytes, gated_bytes(M, N, K, p->type, plan), &st)) return st;
    Room room{static_cast<char*>(workspace)};
    PackList packs{};
    Product q{};
    q.a = operand(x, p->type, M, K, p->ld_x, room, packs);
    q.b = operand(w, p->type, 2 * N, K, p->ld_w, room, packs);
    st = packs.count ? launch_packs(packs, s) : FPQ_OK;
    if (st != FPQ_OK) return st;
    q.M = M;
    q.N = N;
    q.K = K;
    q.planes_a = q.planes_b = planes_of(p->type);
    q.out_f32 = p->type == FPQ_TYPE_FP32;
    q.bias = bias;
    q.gated = true;
    q.gate = Gate{p->act, h, stride(p->ld_h, N, M), pre, 2 * N, pre_scales};
    return launch_product(q, plan, room.at, s);
}

size_t fpq_gated_backward_workspace_size(int64_t M, int64_t N, int64_t K, int type)
{
    const fpq_gated_args_t a{type, 0, M, N, K, 0, 0, 0, 0, 0, 0};
    if (check_gated(&a) != FPQ_OK) return 0;
    return gated_backward_bytes(M, N, K, type, plans_of(M, 2 * N, K, gate_planes(type), planes_of(type)));
}

int fpq_gated_backward(const fpq_gated_args_t* p, const void* x, const uint8_t* x_scales, const void* w, const void* pre, const uint8_t* pre_scales,
                       const void* grad_h, void* grad_x, void* grad_w, float* grad_bias, void* workspace, size_t workspace_bytes, void* stream)
{
    int st = check_gated(p);
    if (st != FPQ_OK) return st;
    const int64_t M = p->M, N = p->N, K = p->K;
    if (M && (!pre || !grad_h)) return FPQ_ERR_NULL;
    if (!stride_ok(p->ld_grad_h, N, M)) return FPQ_ERR_SHAPE;
    const size_t size = size_of(p->type);
    if (!aligned(grad_h, size) || !aligned(pre, pre_scales ? 16 : size)) return FPQ_ERR_ALIGN;
    st = check_gradients(p->type, M, 2 * N, K, x, x_scales, p->ld_x, w, p->ld_w, grad_x, p->ld_grad_x, grad_w, p->ld_grad_w, grad_bias);
    if (st != FPQ_OK) return st;
    const GradientPlans plans = plans_of(M, 2 * N, K, gate_planes(p->type), planes_of(p->type));
    if (workspace_bad(workspace, workspace_bytes, gated_backward_bytes(M, N, K, p->type, plans), &st)) return st;
    if (!grad_x && !grad_w && !grad_bias) return FPQ_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    Room room{static_cast<char*>(workspace)};
    GateBackward g{};
    g.type = p->type;
    g.act = p->act;
    g.M = M;
    g.N = N;
    g.pre = pre;
    g.pre_scales = pre_scales;
    g.gh = grad_h;
    g.ld_gh = stride(p->ld_grad_h, N, M);
    g.ld_d = round8(2 * N);
    g.plane = M * g.ld_d;
    __bf16* const d = room.take<__bf16>(planes_bytes(M, 2 * N, gate_planes(p->type)));
    if (grad_x || grad_w) g.d = d;
    g.grad_bias = grad_bias;
    g.part = reinterpret_cast<float*>(room.at);
    st = launch_gate_backward(g, s);
    if (st != FPQ_OK || !g.d) return st;
    PackList packs{};
    return gradients(Operand{d, g.ld_d, g.plane}, gate_planes(p->type), p->type, M, 2 * N, K, x, x_scales, p->ld_x, w, p->ld_w, grad_x, p->ld_grad_x, grad_w, p->ld_grad_w, nullptr,
                     x_scales ? plans.blocks : plans.values, room, packs, s);
}

int fpq_rms_norm(const fpq_norm_args_t* p, const void* x, const void* residual, const float* w, void* sum, void* y, float* rstd, uint8_t* codes, fpq_format_t f,
                 float scale, const float* scale_dev, uint8_t* code_scales, void* stream)
{
    int st = check_norm(p);
    if (st != FPQ_OK) return st;
    if (!(p->eps >= 0.0f) || isinf(p->eps)) return FPQ_ERR_SCALE;
    if (codes && !code_scales) {
        if (fpq_format_check(f) != FPQ_OK) return FPQ_ERR_FORMAT;
        if (!scale_dev && (!(scale > 0.0f) || isinf(scale))) return FPQ_ERR_SCALE;
    }
    if (p->M == 0) return FPQ_OK;
    if (!x || (residual && !sum) || (code_scales && !codes)) return FPQ_ERR_NULL;
    const int64_t M = p->M, K = p->K;
    if (!stride_ok(p->ld_x, K, M) || (residual && !stride_ok(p->ld_residual, K, M)) || (sum && !stride_ok(p->ld_sum, K, M)) || (y && !stride_ok(p->ld_y, K, M)))
        return FPQ_ERR_SHAPE;
    const size_t size = size_of(p->type);
    if (!aligned(x, size) || !aligned(residual, size) || !aligned(sum, size) || !aligned(y, size) || !aligned(w, 4) || !aligned(rstd, 4) || !aligned(codes, 16) ||
        !aligned(scale_dev, 4))
        return FPQ_ERR_ALIGN;
    NormArgs a{};
    a.x = x;
    a.residual = residual;
    a.w = w;
    a.sum = sum;
    a.y = y;
    a.rstd = rstd;
    a.codes = codes;
    a.code_scales = code_scales;
    if (codes && !code_scales) {
        a.f = QParams{f.mbits, f.bias, f.ebits + f.mbits, f.maxval != 0.0f ? f.maxval : fpq_format_max(f.ebits, f.mbits, f.bias)};
        a.hardware = f.ebits == 4 && f.mbits == 3 && f.bias == 7 && f.maxval == 448.0f;
    }
    a.scale = scale;
    a.scale_dev = scale_dev;
    a.M = M;
    a.K = K;
    a.ld_x = stride(p->ld_x, K, M);
    a.ld_residual = stride(p->ld_residual, K, M);
    a.ld_sum = stride(p->ld_sum, K, M);
    a.ld_y = stride(p->ld_y, K, M);
    a.eps = p->eps;
    return launch_norm(a, p->type, static_cast<hipStream_t>(stream));
}

size_t fpq_rms_norm_backward_workspace_size(int64_t M, int64_t K)
{
    return check_sizes(M, 1, K) == FPQ_OK ? align_up(norm_part_bytes(M, K)) : 0;
}

int fpq_rms_norm_backward(const fpq_norm_args_t* p, const void* sum, const float* w, const float* rstd, const void* grad_y, const void* grad_sum, void* grad_x,
                          float* grad_w, void* workspace, size_t workspace_bytes, void* stream)
{
    int st = check_norm(p);
    if (st != FPQ_OK) return st;
    const int64_t M = p->M, K = p->K;
    if (M && (!sum || !rstd || !grad_y)) return FPQ_ERR_NULL;
    if (!stride_ok(p->ld_sum, K, M) || !stride_ok(p->ld_grad_y, K, M) || (grad_sum && !stride_ok(p->ld_grad_sum, K, M)) ||
        (grad_x && !stride_ok(p->ld_grad_x, K, M)))
        return FPQ_ERR_SHAPE;
    const size_t size = size_of(p->type);
    if (!aligned(sum, size) || !aligned(grad_y, size) || !aligned(grad_sum, size) || !aligned(grad_x, size) || !aligned(w, 4) || !aligned(rstd, 4) || !aligned(grad_w, 4))
        return FPQ_ERR_ALIGN;
    if (grad_w && workspace_bad(workspace, workspace_bytes, fpq_rms_norm_backward_workspace_size(M, K), &st)) return st;
    if (!grad_x && !grad_w) return FPQ_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    NormBackward a{};
    a.sum = sum;
    a.w = w;
    a.rstd = rstd;
    a.gy = grad_y;
    a.gs = grad_sum;
    a.gx = grad_x;
    a.gw = grad_w;
    a.part = static_cast<float*>(workspace);
    a.M = M;
    a.K = K;
    a.ld_sum = stride(p->ld_sum, K, M);
    a.ld_gy = stride(p->ld_grad_y, K, M);
    a.ld_gs = stride(p->ld_grad_sum, K, M);
    a.ld_gx = stride(p->ld_grad_x, K, M);
    return launch_norm_backward(a, p->type, s);
}

}  // extern "C"
