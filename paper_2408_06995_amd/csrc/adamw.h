// The optimizer's plan in device memory: per piece of kAdamwPiece elements the tensor and the piece's place in it, then the tensors.
#pragma once
#include "fpq_host.h"

namespace fpq {

constexpr int kAdamwPiece = 2048;

struct AdamwEntry {
    void* param;
    const void* grad;
    void *m, *v;
    float *m_scale, *v_scale;
    void* copy;
    int64_t n;
    int32_t param_type, grad_type;
    int32_t eight;              // 8-bit states
    int32_t vec;                // every array is aligned for four elements at a time
};
static_assert(sizeof(AdamwEntry) == 80, "entry");

__host__ __device__ inline size_t adamw_entries_at(int64_t pieces) { return ((size_t)pieces * 8 + 15) / 16 * 16; }

int launch_adamw_plan(const fpq_adamw_tensor_t* tensors, int count, int64_t pieces, void* plan, hipStream_t s);
int launch_adamw(const void* plan, int64_t pieces, double lr, double beta1, double beta2, double eps, double weight_decay, int64_t step,
                 const float* grad_scale, hipStream_t s);

}  // namespace fpq
