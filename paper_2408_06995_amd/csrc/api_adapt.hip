// C ABI of the operators for adapting a quantized model (see include/fpq.h): argument validation on the host, then kernel
// launches on the caller's stream.
#include <math.h>

#include "adamw.h"
#include "adapter.h"
#include "attention.h"

using namespace fpq;

namespace {

constexpr int64_t kMost = (int64_t)1 << 30, kMostColumns = (int64_t)1 << 24;

size_t align_up(size_t v) { return (v + 255) / 256 * 256; }
size_t size_of(int type) { return type == FPQ_TYPE_FP32 ? 4 : 2; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int check_attention(const fpq_attention_args_t* p)
{
    if (!p) return FPQ_ERR_NULL;
    if (p->type != FPQ_TYPE_FP32 && p->type != FPQ_TYPE_BF16) return FPQ_ERR_UNSUPPORTED;
    if (p->causal != 0 && p->causal != 1) return FPQ_ERR_UNSUPPORTED;
    for (int64_t v : {p->batch, p->q_heads, p->kv_heads, p->q_len, p->kv_len, p->head_dim})
        if (v < 0 || v > kMost) return FPQ_ERR_SHAPE;
    if (p->q_heads == 0 || p->kv_heads == 0 || p->head_dim == 0 || p->q_heads % p->kv_heads) return FPQ_ERR_SHAPE;
    if (p->head_dim > 160) return FPQ_ERR_UNSUPPORTED;
    if (p->q_heads / p->kv_heads * p->q_len > kMost) return FPQ_ERR_SHAPE;
    // Nearer to the ends of fp32 the kernels' units overflow: the lag of the running maximum, 8 / (scale log2 e), and a row's -lse / scale
    // are finite for every scale from here on, and a log-sum over the scale is a normal number up to there.
    if (!(p->scale >= 0x1p-100f && p->scale <= 0x1p100f)) return FPQ_ERR_SCALE;
    // the grids, and the sizes of the partial results
    const double rows = (double)p->batch * p->q_heads * (p->q_len + 128), keys = (double)p->batch * p->kv_heads * (p->kv_len + 128);
    if (rows > 0x1p31 || keys > 0x1p36) return FPQ_ERR_SHAPE;
    return FPQ_OK;
}

AttentionPlan plan_of(const fpq_attention_args_t* p, bool causal)
{
    return plan_attention(p->batch, p->kv_heads, p->q_heads / p->kv_heads, p->q_len, p->kv_len, p->head_dim, p->type, causal);
}

size_t rows_of(const fpq_attention_args_t* p) { return (size_t)p->batch * p->q_heads * p->q_len; }
size_t keys_of(const fpq_attention_args_t* p) { return (size_t)p->batch * p->kv_heads * p->kv_len; }
bool no_rows(const fpq_attention_args_t* p) { return rows_of(p) == 0; }

// (a single token's stride says nothing)
Strides strides(const int64_t* s, int64_t len, int64_t dim) { return Strides{s[0], len <= 1 ? dim : s[1], s[2]}; }

// Every row of [batch, len, heads, dim] starts at a multiple of `to` bytes.
bool rows_aligned(const void* p, const int64_t* s, int64_t batch, int64_t len, int64_t heads, size_t size, size_t to)
{
    auto ok = [&](int64_t stride, int64_t n) { return n <= 1 || (stride * (int64_t)size) % (int64_t)to == 0; };
    return aligned(p, to) && ok(s[0], batch) && ok(s[1], len) && ok(s[2], heads);
}

// Rows that the kernels can take 16 bytes at a time: aligned, whole pieces, one behind the other, and a tile of them within 32-bit
// offsets.
bool rows_vec(const void* p, const int64_t* s, int64_t batch, int64_t len, int64_t heads, int64_t dim, size_t size)
{
    return rows_aligned(p, s, batch, len, heads, size, 16) && dim * size % 16 == 0 && (len <= 1 || (s[1] >= dim && s[1] < (int64_t)1 << 22));
}

// A workgroup of up to 256 threads per block and part: a launch has fewer than 2^32 threads.
bool grid_ok(const fpq_attention_args_t* p, int64_t blocks, int64_t parts)
{
    return (double)p->batch * (double)p->kv_heads * (double)blocks * (double)parts < 0x1p24;
}

AttentionArgs args_of(const fpq_attention_args_t* p)
{
    AttentionArgs a{};
    a.lens = p->kv_lens;
    a.qs = strides(p->q_strides, p->q_len, p->head_dim);
    a.ks = strides(p->k_strides, p->kv_len, p->head_dim);
    a.vs = strides(p->v_strides, p->kv_len, p->head_dim);
    a.os = strides(p->o_strides, p->q_len, p->head_dim);
    a.batch = (int)p->batch;
    a.kv_heads = (int)p->kv_heads;
    a.group = (int)(p->q_heads / p->kv_heads);
    a.q_len = (int)p->q_len;
    a.kv_len = (int)p->kv_len;
    a.dim = (int)p->head_dim;
    a.causal = p->causal;
    a.scale = p->scale;
    return a;
}

// Two values per row of 32 at a time of each head.
size_t stats_size(const fpq_attention_args_t* p) { return (size_t)p->batch * p->q_heads * ((p->q_len + 31) / 32) * 256; }

// Room for the planes of `rows` packed rows of a tensor.
size_t planes_size(const fpq_attention_args_t* p, size_t rows)
{
    return align_up(rows * ((p->head_dim + 7) / 8 * 8) * 2 * (p->type == FPQ_TYPE_FP32 ? 3 : 1));
}

PackArgs pack_args(const fpq_attention_args_t* p)
{
    PackArgs a{};
    a.batch = (int)p->batch;
    a.kv_len = (int)p->kv_len;
    a.dim = (int)p->head_dim;
    a.lens = p->kv_lens;
    return a;
}

// Whether the feed can read a tensor as it is.
bool feed_reads(const fpq_attention_args_t* p, const void* t, const int64_t* s, int64_t len, int64_t heads)
{
    return p->type == FPQ_TYPE_BF16 && rows_vec(t, s, p->batch, len, heads, p->head_dim, 2);
}

// Room for the planes of a tensor of keys or values, or of queries, that the feed cannot read as it is.
size_t packed_keys(const fpq_attention_args_t* p, const void* t, const int64_t* s)
{
    return feed_reads(p, t, s, p->kv_len, p->kv_heads) ? 0 : planes_size(p, keys_of(p));
}
size_t packed_rows(const fpq_attention_args_t* p, const void* t, const int64_t* s)
{
    return feed_reads(p, t, s, p->q_len, p->q_heads) ? 0 : planes_size(p, rows_of(p));
}

// Room for the results of parts: of rows with their log-sums, of the queries' gradient, of the two of keys and values.
size_t forward_parts(const fpq_attention_args_t* p, const AttentionPlan& plan)
{
    return plan.splits > 1 ? align_up(plan.splits * rows_of(p) * p->head_dim * 4) + align_up(plan.splits * rows_of(p) * 4) : 0;
}
size_t query_parts(const fpq_attention_args_t* p, const AttentionPlan& plan)
{
    return plan.q_splits > 1 ? align_up(plan.q_splits * rows_of(p) * p->head_dim * 4) : 0;
}
size_t key_parts(const fpq_attention_args_t* p, const AttentionPlan& plan)
{
    return plan.k_splits > 1 ? align_up(2 * plan.k_splits * keys_of(p) * p->head_dim * 4) : 0;
}

// How the feed reads a tensor: as it is, or packed at `at` by the call's packing launch.
Source source(PackArgs& pack, const fpq_attention_args_t* p, const void* t, const int64_t* s, int64_t len, int64_t heads, bool keys, char*& at)
{
    const Strides st = strides(s, len, p->head_dim);
    if (feed_reads(p, t, s, len, heads)) return Source{static_cast<const __bf16*>(t), st, 0};
    Pack& m = pack.m[pack.count++];
    m = Pack{t, st, reinterpret_cast<__bf16*>(at), (int)heads, (int)len, keys};
    at += planes_size(p, (size_t)p->batch * len * heads);
    return packed_source(m, p->batch, p->head_dim);
}

// FPQ_OK and the pieces of all tensors
int check_adamw(const fpq_adamw_tensor_t* t, int count, int64_t* pieces)
{
    if (count < 0) return FPQ_ERR_SHAPE;
    if (count && !t) return FPQ_ERR_NULL;
    int64_t sum = 0;
    for (int k = 0; k < count; ++k) {
        const fpq_adamw_tensor_t& x = t[k];
        if (x.n < 0 || x.n >= (int64_t)1 << 31) return FPQ_ERR_SHAPE;
        for (int type : {x.param_type, x.grad_type})
            if (type != FPQ_TYPE_FP32 && type != FPQ_TYPE_BF16) return FPQ_ERR_UNSUPPORTED;
        if ((x.state_bits != 32 && x.state_bits != 8) || x.reserved) return FPQ_ERR_UNSUPPORTED;
        if (x.n == 0) continue;
        if (!x.param || !x.grad || !x.m || !x.v || (x.state_bits == 8 && (!x.m_scale || !x.v_scale))) return FPQ_ERR_NULL;
        const size_t state = x.state_bits == 8 ? 1 : 4;
        if (!aligned(x.param, size_of(x.param_type)) || !aligned(x.grad, size_of(x.grad_type)) || !aligned(x.m, state) || !aligned(x.v, state) ||
            !aligned(x.copy, 2) || (state == 1 && (!aligned(x.m_scale, 4) || !aligned(x.v_scale, 4))))
            return FPQ_ERR_ALIGN;
        sum += (x.n + kAdamwPiece - 1) / kAdamwPiece;
    }
    if (sum >= (int64_t)1 << 31) return FPQ_ERR_SHAPE;
    *pieces = sum;
    return FPQ_OK;
}

int check_adapter_sizes(int64_t M, int64_t N, int64_t K, int64_t R, int64_t requests, int64_t adapters)
{
    // (of M, requests and adapters, so that no dimension of a grid is too large)
    if (M < 0 || M > (int64_t)1 << 28 || requests < 0 || requests > 1 << 21 || adapters < 1 || adapters > 32767) return FPQ_ERR_SHAPE;
    if (N < 1 || N > kMostColumns || K < 1 || K > kMostColumns || R < 1) return FPQ_ERR_SHAPE;
    if (R > kMaxRank) return FPQ_ERR_UNSUPPORTED;
    return FPQ_OK;
}

// Every row of [rows, n] starts at a multiple of `to` bytes.
bool matrix_aligned(const void* p, int64_t ld, int64_t rows, size_t size, size_t to)
{
    return aligned(p, to) && (rows <= 1 || ld * (int64_t)size % (int64_t)to == 0);
}

// A tile of rows is addressed with 32-bit offsets.
bool stride_ok(int64_t ld, int64_t cols) { return ld >= cols && ld <= kMostColumns; }

// Sizes and pointers that both calls have; a row of fewer elements than its stride's claim is an error.
int check_adapter(const fpq_adapter_args_t* p, const void* x, const void* a, const void* b)
{
    if (!p) return FPQ_ERR_NULL;
    if (p->x_type != FPQ_TYPE_FP32 && p->x_type != FPQ_TYPE_BF16) return FPQ_ERR_UNSUPPORTED;
    if (p->w_type != FPQ_TYPE_FP32 && p->w_type != FPQ_TYPE_BF16) return FPQ_ERR_UNSUPPORTED;
    if (p->x_type == FPQ_TYPE_BF16 && p->w_type != FPQ_TYPE_BF16) return FPQ_ERR_UNSUPPORTED;
    const int st = check_adapter_sizes(p->M, p->N, p->K, p->R, p->requests, p->adapters);
    if (st != FPQ_OK) return st;
    if (p->M && !stride_ok(p->ld_x, p->K)) return FPQ_ERR_SHAPE;
    if (!p->scaling || !p->row_start || (p->requests && !p->adapter) || !a || !b || (p->M && !x)) return FPQ_ERR_NULL;
    if (!aligned(p->scaling, 4) || !aligned(p->row_start, 4) || !aligned(p->adapter, 4) || !aligned(x, size_of(p->x_type)) ||
        !aligned(a, size_of(p->w_type)) || !aligned(b, size_of(p->w_type)))
        return FPQ_ERR_ALIGN;
    return FPQ_OK;
}

// Forward: whether a workspace for packed weights is asked for.  Ranks up to 16 read weights of any alignment where they are.
bool pack_forward(int64_t R, int64_t K) { return R > kPlainRank && (R % 8 != 0 || K % 8 != 0); }

// Packs the weights of a map into the workspace: W1 [R, L1], W2 [L2, R].
int pack_weights(const fpq_adapter_args_t* p, const void* a, const void* b, bool forward, void* workspace, AdapterArgs& r, hipStream_t s)
{
    const int64_t planes = p->w_type == FPQ_TYPE_FP32 ? 3 : 1, n1 = packed_elements(forward ? p->K : p->N, p->R), n2 = packed_elements(forward ? p->N : p->K, p->R);
    __bf16* const w1 = static_cast<__bf16*>(workspace);
    __bf16* const w2 = w1 + align_up((size_t)p->adapters * planes * n1 * 2) / 2;
    r.w1 = Weights{w1, planes * n1, n1, 0, 1};
    r.w2 = Weights{w2, planes * n2, n2, 0, 1};
    return launch_adapter_pack(AdapterPack{a, b, w1, w2, (int)p->N, (int)p->K, (int)p->R, (int)p->adapters, forward}, p->w_type, s);
}

AdapterArgs args_of(const fpq_adapter_args_t* p)
{
    AdapterArgs r{};
    r.row_start = p->row_start;
    r.adapter = p->adapter;
    r.M = (int)p->M;
    r.R = (int)p->R;
    r.requests = (int)p->requests;
    r.adapters = (int)p->adapters;
    return r;
}

// Bytes of a pool's packed weights along `len`, fp32 or bf16.
size_t packed_weights(int w_type, int64_t adapters, int64_t len, int64_t R)
{
    return align_up((size_t)adapters * packed_elements(len, R) * 2 * (w_type == FPQ_TYPE_FP32 ? 3 : 1));
}

bool finite_not_negative(double v) { return v >= 0.0 && !isinf(v); }

}  // namespace

extern "C" {

size_t fpq_adapter_workspace_size(int64_t M, int64_t N, int64_t K, int64_t R, int64_t requests, int64_t adapters)
{
    if (check_adapter_sizes(M, N, K, R, requests, adapters) != FPQ_OK) return 0;
    return pack_forward(R, K) ? packed_weights(FPQ_TYPE_FP32, adapters, N, R) + packed_weights(FPQ_TYPE_FP32, adapters, K, R) : 0;
}

int fpq_adapter_apply(const fpq_adapter_args_t* p, const void* x, const void* a, const void* b, const void* base, void* y, float* t,
                      void* workspace, size_t workspace_bytes, void* stream)
{
    const int st = check_adapter(p, x, a, b);
    if (st != FPQ_OK) return st;
    if (p->M == 0) return FPQ_OK;
    if (!y) return FPQ_ERR_NULL;
    if (!stride_ok(p->ld_y, p->N) || (base && !stride_ok(p->ld_base, p->N))) return FPQ_ERR_SHAPE;
    const size_t size = size_of(p->x_type), w = size_of(p->w_type);
    if (!aligned(y, size) || !aligned(base, size) || !aligned(t, 4)) return FPQ_ERR_ALIGN;
    const size_t need = fpq_adapter_workspace_size(p->M, p->N, p->K, p->R, p->requests, p->adapters);
    if (need && (!workspace || workspace_bytes < need)) return FPQ_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return FPQ_ERR_ALIGN;
    const AdapterPlan plan = plan_adapter(p->M, p->N, p->K, p->requests, p->adapters);
    hipStream_t s = static_cast<hipStream_t>(stream);
    AdapterArgs r = args_of(p);
    r.x = x;
    r.ldx = p->ld_x;
    r.base = base;
    r.ld_base = p->ld_base;
    r.y = y;
    r.ldy = p->ld_y;
    r.t = t;
    r.w1 = Weights{a, p->R * p->K, 0, (int)p->K, p->K * w % 16 == 0 && aligned(a, 16)};
    r.w2 = Weights{b, p->N * p->R, 0, (int)p->R, p->R * w % 16 == 0 && aligned(b, 16)};
    r.scale2 = p->scaling;
    r.L1 = (int)p->K;
    r.L2 = (int)p->N;
    r.vec_x = p->K * size % 16 == 0 && matrix_aligned(x, p->ld_x, p->M, size, 16);
    r.parts = plan.parts_n;
    const bool packed = p->R > kPlainRank && !(r.w1.vec && r.w2.vec);
    if (packed) {
        if (!need) return FPQ_ERR_ALIGN;
        const int done = pack_weights(p, a, b, true, workspace, r, s);
        if (done != FPQ_OK) return done;
    }
    return launch_adapter_map(r, p->x_type, p->w_type, packed, plan.waves, s);
}

size_t fpq_adapter_backward_workspace_size(int64_t M, int64_t N, int64_t K, int64_t R, int64_t requests, int64_t adapters)
{
    if (check_adapter_sizes(M, N, K, R, requests, adapters) != FPQ_OK) return 0;
    const AdapterPlan plan = plan_adapter(M, N, K, requests, adapters);
    const size_t each = (size_t)adapters * R * 4;
    return align_up((size_t)M * R * 4) + packed_weights(FPQ_TYPE_FP32, adapters, N, R) + packed_weights(FPQ_TYPE_FP32, adapters, K, R) +
           (plan.splits > 1 ? align_up(plan.splits * each * K) + align_up(plan.splits * each * N) : 0);
}

int fpq_adapter_backward(const fpq_adapter_args_t* p, const void* x, const void* a, const void* b, const float* t, const void* grad_y,
                         const void* grad_x_base, void* grad_x, float* grad_a, float* grad_b, void* workspace, size_t workspace_bytes, void* stream)
{
    const int st = check_adapter(p, x, a, b);
    if (st != FPQ_OK) return st;
    if (!grad_a || !grad_b || (p->M && (!t || !grad_y))) return FPQ_ERR_NULL;
    if (p->M && !stride_ok(p->ld_grad_y, p->N)) return FPQ_ERR_SHAPE;
    if (p->M && grad_x && (!stride_ok(p->ld_grad_x, p->K) || (grad_x_base && !stride_ok(p->ld_grad_x_base, p->K)))) return FPQ_ERR_SHAPE;
    const size_t size = size_of(p->x_type);
    if (!aligned(t, 4) || !aligned(grad_y, size) || !aligned(grad_x_base, size) || !aligned(grad_x, size) || !aligned(grad_a, 4) || !aligned(grad_b, 4))
        return FPQ_ERR_ALIGN;
    const size_t need = fpq_adapter_backward_workspace_size(p->M, p->N, p->K, p->R, p->requests, p->adapters);
    if (!workspace || workspace_bytes < need) return FPQ_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return FPQ_ERR_ALIGN;
    const AdapterPlan plan = plan_adapter(p->M, p->N, p->K, p->requests, p->adapters);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int N = (int)p->N, K = (int)p->K, R = (int)p->R;
    char* at = static_cast<char*>(workspace);
    auto take = [&](size_t bytes) {
        char* const r = at;
        at += bytes;
        return r;
    };
    float* const dt = reinterpret_cast<float*>(take(align_up((size_t)p->M * R * 4)));
    int done = FPQ_OK;
    if (p->M) {
        AdapterArgs r = args_of(p);
        done = pack_weights(p, a, b, false, at, r, s);
        if (done != FPQ_OK) return done;
        at += packed_weights(FPQ_TYPE_FP32, p->adapters, N, R) + packed_weights(FPQ_TYPE_FP32, p->adapters, K, R);
        r.parts = plan.parts_k;
        r.x = grad_y;
        r.ldx = p->ld_grad_y;
        r.base = grad_x ? grad_x_base : nullptr;
        r.ld_base = p->ld_grad_x_base;
        r.y = grad_x;
        r.ldy = p->ld_grad_x;
        r.t = dt;
        r.scale1 = p->scaling;
        r.L1 = N;
        r.L2 = K;
        r.vec_x = p->N * size % 16 == 0 && matrix_aligned(grad_y, p->ld_grad_y, p->M, size, 16);
        done = launch_adapter_map(r, p->x_type, p->w_type, true, plan.waves, s);
        if (done != FPQ_OK) return done;
    }
    const size_t na = (size_t)p->adapters * R * K, nb = (size_t)p->adapters * R * N;
    OuterArgs o{};
    o.rows[0] = x;
    o.rows[1] = grad_y;
    o.ld[0] = p->ld_x;
    o.ld[1] = p->ld_grad_y;
    o.t[0] = dt;
    o.t[1] = t;
    o.L[0] = K;
    o.L[1] = N;
    o.scaling = p->scaling;
    o.row_start = p->row_start;
    o.adapter = p->adapter;
    o.M = (int)p->M;
    o.R = R;
    o.requests = (int)p->requests;
    o.adapters = (int)p->adapters;
    o.splits = plan.splits;
    o.out[0] = plan.splits > 1 ? reinterpret_cast<float*>(take(align_up(plan.splits * na * 4))) : grad_a;
    o.out[1] = plan.splits > 1 ? reinterpret_cast<float*>(take(align_up(plan.splits * nb * 4))) : grad_b;
    o.vec_rows[0] = p->K * size % 16 == 0 && matrix_aligned(x, p->ld_x, p->M, size, 16);
    o.vec_rows[1] = p->N * size % 16 == 0 && matrix_aligned(grad_y, p->ld_grad_y, p->M, size, 16);
    o.vec_t = R % 4 == 0 && aligned(t, 16);
    done = launch_adapter_outer(o, p->x_type, s);
    if (done != FPQ_OK || plan.splits == 1) return done;
    return launch_adapter_sums(o.out[0], o.out[1], plan.splits, na, nb, grad_a, grad_b, s);
}

size_t fpq_adamw_plan_size(const fpq_adamw_tensor_t* tensors, int count)
{
    int64_t pieces;
    if (check_adamw(tensors, count, &pieces) != FPQ_OK) return 0;
    return adamw_entries_at(pieces) + (size_t)count * sizeof(AdamwEntry);
}

int fpq_adamw_plan(const fpq_adamw_tensor_t* tensors, int count, void* plan, size_t plan_bytes, int64_t* pieces_out, void* stream)
{
    int64_t pieces;
    const int st = check_adamw(tensors, count, &pieces);
    if (st != FPQ_OK) return st;
    if (!pieces_out) return FPQ_ERR_NULL;
    if (pieces && !plan) return FPQ_ERR_NULL;
    if (plan_bytes < fpq_adamw_plan_size(tensors, count)) return FPQ_ERR_WORKSPACE;
    if (!aligned(plan, 16)) return FPQ_ERR_ALIGN;
    *pieces_out = pieces;
    if (!pieces) return FPQ_OK;
    return launch_adamw_plan(tensors, count, pieces, plan, static_cast<hipStream_t>(stream));
}

int fpq_adamw_step(const void* plan, int64_t pieces, double lr, double beta1, double beta2, double eps, double weight_decay, int64_t step,
                   const float* grad_scale, void* stream)
{
    if (pieces < 0 || pieces >= (int64_t)1 << 31 || step < 1) return FPQ_ERR_SHAPE;
    if (!finite_not_negative(lr) || !finite_not_negative(weight_decay) || !(eps > 0.0) || isinf(eps) || !(beta1 >= 0.0 && beta1 < 1.0) ||
        !(beta2 >= 0.0 && beta2 < 1.0))
        return FPQ_ERR_SCALE;
    if (!pieces) return FPQ_OK;
    if (!plan) return FPQ_ERR_NULL;
    if (!aligned(plan, 16) || !aligned(grad_scale, 4)) return FPQ_ERR_ALIGN;
    return launch_adamw(plan, pieces, lr, beta1, beta2, eps, weight_decay, step, grad_scale, static_cast<hipStream_t>(stream));
}

// (what is stated is enough with and without `causal`, and for tensors of any layout; a call asks for what it uses)
size_t fpq_attention_workspace_size(const fpq_attention_args_t* p)
{
    if (check_attention(p) != FPQ_OK || no_rows(p)) return 0;
    size_t most = 0;
    for (bool causal : {false, true}) {
        const AttentionPlan plan = plan_of(p, causal);
        const size_t size = forward_parts(p, plan) + (plan.by_keys ? 0 : 2 * planes_size(p, keys_of(p)));
        most = size > most ? size : most;
    }
    return most;
}

int fpq_attention(const fpq_attention_args_t* p, const void* q, const void* k, const void* v, void* o, float* lse, void* workspace,
                  size_t workspace_bytes, void* stream)
{
    const int st = check_attention(p);
    if (st != FPQ_OK) return st;
    if (no_rows(p)) return FPQ_OK;
    if (!q || !o || (p->kv_len && (!k || !v))) return FPQ_ERR_NULL;
    const size_t size = size_of(p->type);
    if (!aligned(q, size) || !aligned(k, size) || !aligned(v, size) || !aligned(o, size) || !aligned(lse, 4) || !aligned(p->kv_lens, 4))
        return FPQ_ERR_ALIGN;
    const AttentionPlan plan = plan_of(p, p->causal);
    if (!grid_ok(p, plan.blocks, plan.splits)) return FPQ_ERR_SHAPE;
    const size_t need = forward_parts(p, plan) + (plan.by_keys ? 0 : packed_keys(p, k, p->k_strides) + packed_keys(p, v, p->v_strides));
    if (need && (!workspace || workspace_bytes < need)) return FPQ_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return FPQ_ERR_ALIGN;
    AttentionArgs a = args_of(p);
    a.q = q;
    a.k = k;
    a.v = v;
    a.out = o;
    a.lse = lse;
    a.blocks = plan.blocks;
    a.q_pad = plan.q_pad;
    a.splits = plan.splits;
    a.vec_out = p->head_dim % 4 == 0 && rows_aligned(o, p->o_strides, p->batch, p->q_len, p->q_heads, size, 4 * size);
    a.vec = rows_vec(q, p->q_strides, p->batch, p->q_len, p->q_heads, p->head_dim, size) &&
            rows_vec(k, p->k_strides, p->batch, p->kv_len, p->kv_heads, p->head_dim, size) &&
            rows_vec(v, p->v_strides, p->batch, p->kv_len, p->kv_heads, p->head_dim, size);
    char* at = static_cast<char*>(workspace);
    if (plan.splits > 1) {
        a.part = reinterpret_cast<float*>(at);
        a.part_lse = reinterpret_cast<float*>(at + align_up(plan.splits * rows_of(p) * p->head_dim * 4));
        at += forward_parts(p, plan);
    }
    if (!plan.by_keys) {
        PackArgs pack = pack_args(p);
        a.fk = source(pack, p, k, p->k_strides, p->kv_len, p->kv_heads, true, at);
        a.fv = source(pack, p, v, p->v_strides, p->kv_len, p->kv_heads, true, at);
        const int packed = launch_pack(pack, p->type, static_cast<hipStream_t>(stream));
        if (packed != FPQ_OK) return packed;
    }
    return launch_attention(a, p->type, plan, static_cast<hipStream_t>(stream));
}

size_t fpq_attention_backward_workspace_size(const fpq_attention_args_t* p)
{
    if (check_attention(p) != FPQ_OK) return 0;
    size_t most = 0;
    for (bool causal : {false, true}) {
        const AttentionPlan plan = plan_of(p, causal);
        const size_t size = query_parts(p, plan) + key_parts(p, plan);
        most = size > most ? size : most;
    }
    return stats_size(p) + most + 2 * planes_size(p, keys_of(p)) + 2 * planes_size(p, rows_of(p));
}

int fpq_attention_backward(const fpq_attention_args_t* p, const void* q, const void* k, const void* v, const void* o, const float* lse,
                           const void* grad_o, void* grad_q, void* grad_k, void* grad_v, void* workspace, size_t workspace_bytes, void* stream)
{
    const int st = check_attention(p);
    if (st != FPQ_OK) return st;
    if (p->batch == 0 || (p->q_len == 0 && p->kv_len == 0)) return FPQ_OK;
    if (p->q_len && (!q || !o || !lse || !grad_o || !grad_q)) return FPQ_ERR_NULL;
    if (p->kv_len && (!k || !v || !grad_k || !grad_v)) return FPQ_ERR_NULL;
    const size_t size = size_of(p->type);
    for (const void* x : {q, k, v, o, grad_o, static_cast<const void*>(grad_q), static_cast<const void*>(grad_k), static_cast<const void*>(grad_v)})
        if (!aligned(x, size)) return FPQ_ERR_ALIGN;
    if (!aligned(lse, 4) || !aligned(p->kv_lens, 4)) return FPQ_ERR_ALIGN;
    const AttentionPlan plan = plan_of(p, p->causal);
    if (!grid_ok(p, plan.q_blocks, plan.q_splits) || !grid_ok(p, plan.k_blocks, plan.k_splits)) return FPQ_ERR_SHAPE;
    const size_t need = stats_size(p) + query_parts(p, plan) + key_parts(p, plan) + packed_keys(p, k, p->k_strides) + packed_keys(p, v, p->v_strides) +
                        packed_rows(p, q, p->q_strides) + packed_rows(p, grad_o, p->grad_o_strides);
    if (need && (!workspace || workspace_bytes < need)) return FPQ_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return FPQ_ERR_ALIGN;
    AttentionArgs a = args_of(p);
    a.q = q;
    a.k = k;
    a.v = v;
    a.o = o;
    a.go = grad_o;
    a.gq = grad_q;
    a.gk = grad_k;
    a.gv = grad_v;
    a.lse = const_cast<float*>(lse);
    a.gos = strides(p->grad_o_strides, p->q_len, p->head_dim);
    a.gqs = strides(p->grad_q_strides, p->q_len, p->head_dim);
    a.gks = strides(p->grad_k_strides, p->kv_len, p->head_dim);
    a.gvs = strides(p->grad_v_strides, p->kv_len, p->head_dim);
    a.vec_out = p->head_dim % 4 == 0 && rows_aligned(grad_q, p->grad_q_strides, p->batch, p->q_len, p->q_heads, size, 4 * size);
    a.vec = rows_vec(q, p->q_strides, p->batch, p->q_len, p->q_heads, p->head_dim, size) &&
            rows_vec(k, p->k_strides, p->batch, p->kv_len, p->kv_heads, p->head_dim, size) &&
            rows_vec(v, p->v_strides, p->batch, p->kv_len, p->kv_heads, p->head_dim, size) &&
            rows_vec(o, p->o_strides, p->batch, p->q_len, p->q_heads, p->head_dim, size) &&
            rows_vec(grad_o, p->grad_o_strides, p->batch, p->q_len, p->q_heads, p->head_dim, size);
    char* at = static_cast<char*>(workspace);
    a.stats = reinterpret_cast<float*>(at);
    at += stats_size(p);
    float* const part_q = reinterpret_cast<float*>(at);
    at += query_parts(p, plan);
    float* const part_kv = reinterpret_cast<float*>(at);
    at += key_parts(p, plan);
    PackArgs pack = pack_args(p);
    a.fk = source(pack, p, k, p->k_strides, p->kv_len, p->kv_heads, true, at);
    a.fv = source(pack, p, v, p->v_strides, p->kv_len, p->kv_heads, true, at);
    a.fq = source(pack, p, q, p->q_strides, p->q_len, p->q_heads, false, at);
    a.fgo = source(pack, p, grad_o, p->grad_o_strides, p->q_len, p->q_heads, false, at);
    const int packed = launch_pack(pack, p->type, static_cast<hipStream_t>(stream));
    if (packed != FPQ_OK) return packed;
    return launch_attention_backward(a, p->type, plan, part_q, part_kv, static_cast<hipStream_t>(stream));
}

}  // extern "C"
