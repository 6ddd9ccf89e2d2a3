// Host-side interfaces between the C ABI (capi_block.cu) and the language-model block kernels.
#pragma once

#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

#include "internal.h"
#include "qnn.h"

namespace qnn {

// ---- norms around a block -- norm.cu
// Blocks of the resident norm kernel and their rings.  As many blocks as the threads of an SM allow (64 registers each) while
// every block has two stages or more; all of them have to fit the SM at once, with their static memory and the 1 KB that the
// system takes of each, or those that do not start only when the others have done their rows.  (161318 rows of 832, 16
// blocks an SM: 294 us with rings of four stages, of which 15 fit, 215 with three; 101066 rows of 1328, ten blocks: 295 and
// 205 us.)
constexpr int kNormItems = 2;                  // vectors of eight values a thread
constexpr uint32_t kNormRoom = 208 * 1024;     // of ring on an SM at most: the rest of the 256 KB stays L1
constexpr uint32_t kNormSm = 228 * 1024;       // shared memory of an SM
constexpr uint32_t kNormStatic = 1152;         // of a block
struct NormRing {
    int threads, per_sm, stages;
    uint32_t x_bytes, res_bytes, smem;  // of a row of x and of the residual (0 without one); of a block's ring
};
inline NormRing norm_ring(int d, uint32_t x_bytes, uint32_t res_bytes)
{
    NormRing r = {((d + 8 * kNormItems - 1) / (8 * kNormItems) + 31) / 32 * 32, 0, 0, x_bytes, res_bytes, 0};
    if (r.threads < 64) r.threads = 64;
    const uint32_t stage = x_bytes + res_bytes;
    auto room = [](int blocks) {  // of each of so many blocks; memory is given out in units of 128 bytes
        const uint32_t ring = kNormRoom / blocks, whole = kNormSm / blocks / 128 * 128 - kNormStatic - 1024;
        return ring < whole ? ring : whole;
    };
    r.per_sm = 1024 / r.threads;
    while (r.per_sm > 1 && room(r.per_sm) < 2 * stage) --r.per_sm;
    const uint32_t fit = room(r.per_sm) / stage;
    r.stages = fit > 4 ? 4 : static_cast<int>(fit);
    r.smem = r.stages * stage;
    return r;
}
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
