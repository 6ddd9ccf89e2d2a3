// Host-side interfaces between the C ABI (capi_block.cu) and the language-model block kernels.
#pragma once

#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

#include "internal.h"
#include "qnn.h"

namespace qnn {

// ---- norms around a block -- norm.cu
cudaError_t launch_block_norm(const qnn_norm_desc &d, const void *x, const void *residual, const void *gate,
                              const void *post_w, const void *post_b, const void *pre_w, const void *pre_b, void *r,
                              void *h, cudaStream_t st);

// ---- routing and the experts' plan -- route.cu
cudaError_t launch_route_topk(const qnn_route_desc &d, const void *logits, const float *bias, float *weights,
                              int32_t *ids, cudaStream_t st);
size_t expert_plan_workspace(int64_t slots, int experts);
cudaError_t launch_expert_plan(const int32_t *ids, int64_t slots, int experts, int32_t *offsets, int32_t *order,
                               int32_t *position, void *workspace, cudaStream_t st);

}  // namespace qnn
