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

// ---- matrix products: weight image and the sum over a token's experts -- matmul_prep.cu
struct MatmulArgs;
cudaError_t launch_matmul_prep(const qnn_matmul_desc &d, const void *w, const float *scale, const float *bias,
                               void *image, cudaStream_t st);
cudaError_t launch_combine(int dtype, const float *z, int64_t ldz, const float *weights, const int32_t *position,
                           int64_t tokens, int top, int m, const void *residual, int64_t ldres, void *y, int64_t ldy,
                           cudaStream_t st);
// rows of 16-bit values to rows ldd apart (a multiple of 8), in order or as a plan has them: for the tiled loads, which
// take 16-byte aligned rows that lie one after another
cudaError_t launch_take_rows(const void *src, int64_t lds, const int32_t *order, int top, void *dst, int64_t ldd, int64_t rows,
                             int cols, cudaStream_t st);
// ---- tcgen05 -- matmul_tc.cu (rows of x 16-byte aligned)
cudaError_t launch_matmul_tc(const MatmulArgs &a, int dtype, int bits, cudaStream_t st);
// ---- few rows: streamed weights -- matmul_stream.cu
cudaError_t launch_matmul_stream(const MatmulArgs &a, int dtype, int bits, cudaStream_t st);

}  // namespace qnn
