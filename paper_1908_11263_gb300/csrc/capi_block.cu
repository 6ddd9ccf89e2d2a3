// C ABI of the language-model block operators (declared in include/qnn.h): argument validation and dispatch.  Every
// check happens before anything is enqueued; a call that returns an error has launched nothing.
#include <cmath>

#include "block_internal.h"
#include "matmul.cuh"

namespace qnn {
namespace {

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
qnn_status from_cuda(cudaError_t e) { return e == cudaSuccess ? QNN_OK : QNN_ECUDA; }
bool dtype_ok(int32_t t) { return t == QNN_F16 || t == QNN_BF16 || t == QNN_F32; }
uintptr_t dtype_size(int32_t t) { return t == QNN_F32 ? 4 : 2; }
bool flag_ok(int32_t v) { return v == 0 || v == 1; }

// What the kernels' 32-bit counters of tiles and of units of work hold, whatever tile the launch takes: 2^40 weights in
// 32 x 64 blocks, 2^38 outputs and 2^20 rows of x give less than 2^30 tiles and 2^31 units.
constexpr int64_t kMaxBlocks = 1ll << 29, kMaxOutputs = 1ll << 38, kMaxRows = 1 << 20;

qnn_status check_matmul(const qnn_matmul_desc *d)
{
    if (!d || d->struct_size != sizeof(qnn_matmul_desc)) return QNN_EINVAL;
    if (d->experts <= 0 || d->m <= 0 || d->k <= 0 || !flag_ok(d->gated)) return QNN_EINVAL;
    if (d->act < QNN_ACT_NONE || d->act > QNN_ACT_GELU_TANH || !dtype_ok(d->dtype)) return QNN_EINVAL;
    if (d->dtype == QNN_F32 || (d->bits != 16 && d->bits != 8 && d->bits != 4 && d->bits != 2)) return QNN_EUNSUPPORTED;
    if (d->experts > 1024 || d->m > (1 << 24) || d->k > (1 << 24)) return QNN_EUNSUPPORTED;
    if (d->bits < 8 && d->k % (8 / d->bits)) return QNN_EUNSUPPORTED;
    const MatmulImage g = matmul_image(d->experts, d->m, d->k, d->bits, d->gated);
    return static_cast<int64_t>(d->experts) * g.mb * g.kb > kMaxBlocks ? QNN_EUNSUPPORTED : QNN_OK;
}

// An output of `rows` rows.
qnn_status check_rows(const qnn_matmul_desc &d, int64_t rows)
{
    return rows > kMaxRows || rows * d.m > kMaxOutputs ? QNN_EUNSUPPORTED : QNN_OK;
}

MatmulArgs base_args(const qnn_matmul_desc &d, const void *image, const void *x, int64_t ldx, void *y, int64_t ldy)
{
    const MatmulImage g = matmul_image(d.experts, d.m, d.k, d.bits, d.gated);
    MatmulArgs a = {};
    a.image = static_cast<const uint8_t *>(image);
    a.params = reinterpret_cast<const float2 *>(a.image + g.param_off);
    a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy;
    a.m = d.m; a.k = d.k; a.kb = g.kb; a.mb = g.mb; a.experts = d.experts; a.top = 1;
    a.act = d.act; a.gated = d.gated;
    a.x_vec = aligned(x, 16) && ldx % 8 == 0;
    return a;
}

qnn_status check_image(const qnn_matmul_desc &d, const void *image, size_t bytes)
{
    if (!image || bytes < matmul_image(d.experts, d.m, d.k, d.bits, d.gated).bytes) return QNN_EINVAL;
    return aligned(image, 256) ? QNN_OK : QNN_EALIGN;
}

// The tensor-core kernel takes over where a matrix meets more rows of x than this, on average for experts.  Measured on
// both sides (us, streaming / tensor cores): 32 rows of 4096 x 4096 INT-4 9.4 / 17.6, 16-bit 10.7 / 16.0; 64 experts of
// 2 * 1024 x 2048, INT-4 with 16 rows an expert 82 / 106, 16-bit with 4 rows 77 / 76, with 6 rows 101 / 85, with 8 rows
// 109 / 83 (the stream reads 16-bit weights again for every 8 or 16 rows; of packed ones it mostly expands the codes).
bool on_tensor_cores(int64_t rows, int experts, int bits)
{
    return rows > (experts ? static_cast<int64_t>(bits == 16 ? 6 : 16) * experts : 32);
}

int64_t align8(int64_t v) { return (v + 7) / 8 * 8; }
size_t align256(size_t v) { return (v + 255) / 256 * 256; }

// Bytes for the rows of x as the tensor-core kernel takes them, where x has not got them so: `rows` rows, in the order
// of the plan for a dispatch, 16-byte aligned.
size_t staging_bytes(const qnn_matmul_desc &d, int64_t rows, int experts, bool gather, const void *x, int64_t ldx)
{
    if (!on_tensor_cores(rows, experts, d.bits) || (!gather && aligned(x, 16) && ldx % 8 == 0)) return 0;
    return static_cast<size_t>(rows) * align8(d.k) * 2;
}

cudaError_t run_product(MatmulArgs a, const qnn_matmul_desc &d, void *staging, cudaStream_t st)
{
    if (!on_tensor_cores(a.rows, a.offsets ? a.experts : 0, d.bits)) return launch_matmul_stream(a, d.dtype, d.bits, st);
    if (a.gather || !a.x_vec) {
        const cudaError_t e = launch_take_rows(a.x, a.ldx, a.gather ? a.order : nullptr, a.top, staging, align8(d.k), a.rows, d.k, st);
        if (e != cudaSuccess) return e;
        a.x = staging;
        a.ldx = align8(d.k);
        a.x_rows = a.rows;
        a.gather = 0;
    }
    return launch_matmul_tc(a, d.dtype, d.bits, st);
}

// Rows of the 32-bit products that a combine sums over.
int64_t combine_ld(const qnn_matmul_desc &d) { return (static_cast<int64_t>(d.m) + 7) / 8 * 8; }

qnn_status check_slots(const qnn_matmul_desc *d, int64_t tokens, int32_t top)
{
    const qnn_status st = check_matmul(d);
    if (st != QNN_OK) return st;
    if (tokens < 0 || top <= 0) return QNN_EINVAL;
    if (top > 1024 || tokens > kMaxRows) return QNN_EUNSUPPORTED;
    return check_rows(*d, tokens * top);
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" {

qnn_status qnn_block_norm(const qnn_norm_desc *d, const void *x, const void *residual, const void *gate,
                          const void *post_w, const void *post_b, const void *pre_w, const void *pre_b, void *r,
                          void *h, void *stream)
{
    if (!d || d->struct_size != sizeof(qnn_norm_desc)) return QNN_EINVAL;
    if (!dtype_ok(d->dtype) || !dtype_ok(d->residual_dtype) || !dtype_ok(d->param_dtype)) return QNN_EINVAL;
    if (d->kind != QNN_NORM_RMS && d->kind != QNN_NORM_LAYER) return QNN_EINVAL;
    if (!flag_ok(d->post_norm) || d->t < 0 || d->d <= 0) return QNN_EINVAL;
    if (!(d->eps >= 0.f) || std::isinf(d->eps)) return QNN_EINVAL;
    if (d->t > 0 && (!x || (!r && !h))) return QNN_EINVAL;
    if (d->ldx < d->d || (residual && d->ldres < d->d) || (r && d->ldr < d->d) || (h && d->ldh < d->d))
        return QNN_EINVAL;
    if (gate && (d->gates <= 0 || d->t % d->gates)) return QNN_EINVAL;
    if (d->residual_dtype != d->dtype && d->residual_dtype != QNN_F32) return QNN_EUNSUPPORTED;
    if (d->param_dtype != d->dtype && d->param_dtype != QNN_F32) return QNN_EUNSUPPORTED;
    if (d->d > 32768 || d->t > 0x7fffffffll) return QNN_EUNSUPPORTED;
    const uintptr_t sx = dtype_size(d->dtype), sr = dtype_size(d->residual_dtype), sp = dtype_size(d->param_dtype);
    if (!aligned(x, sx) || !aligned(h, sx) || !aligned(residual, sr) || !aligned(r, sr)) return QNN_EALIGN;
    if (!aligned(gate, sp) || !aligned(post_w, sp) || !aligned(post_b, sp) || !aligned(pre_w, sp) || !aligned(pre_b, sp))
        return QNN_EALIGN;
    return from_cuda(launch_block_norm(*d, x, residual, gate, post_w, post_b, pre_w, pre_b, r, h,
                                       static_cast<cudaStream_t>(stream)));
}

qnn_status qnn_route_topk(const qnn_route_desc *d, const void *logits, const float *bias, float *weights,
                          int32_t *ids, void *stream)
{
    if (!d || d->struct_size != sizeof(qnn_route_desc)) return QNN_EINVAL;
    if (!dtype_ok(d->dtype) || !flag_ok(d->renormalise)) return QNN_EINVAL;
    if (d->experts <= 0 || d->k <= 0 || d->k > d->experts || d->t < 0 || d->ld < d->experts) return QNN_EINVAL;
    if (d->score != QNN_SCORE_SOFTMAX && d->score != QNN_SCORE_SIGMOID) return QNN_EINVAL;
    if (d->group_score != QNN_GROUP_MAX && d->group_score != QNN_GROUP_TOP2) return QNN_EINVAL;
    if (d->groups <= 0 || d->experts % d->groups || d->top_groups <= 0 || d->top_groups > d->groups) return QNN_EINVAL;
    if (!std::isfinite(d->scale)) return QNN_EINVAL;
    if (d->t > 0 && (!logits || !weights || !ids)) return QNN_EINVAL;
    if (d->experts > 1024 || d->k > 32 || d->groups > 32 || d->t > 0x7fffffffll) return QNN_EUNSUPPORTED;
    if (!aligned(logits, dtype_size(d->dtype)) || !aligned(bias, 4) || !aligned(weights, 4) || !aligned(ids, 4))
        return QNN_EALIGN;
    return from_cuda(launch_route_topk(*d, logits, bias, weights, ids, static_cast<cudaStream_t>(stream)));
}

qnn_status qnn_expert_plan_workspace_size(int64_t slots, int32_t experts, size_t *bytes)
{
    if (!bytes || slots < 0 || experts <= 0) return QNN_EINVAL;
    if (slots > 0x7fffffffll - 2048 || experts > 1024) return QNN_EUNSUPPORTED;
    *bytes = expert_plan_workspace(slots, experts);
    return QNN_OK;
}

qnn_status qnn_expert_plan(const int32_t *ids, int64_t slots, int32_t experts, int32_t *offsets, int32_t *order,
                           int32_t *position, void *workspace, size_t workspace_bytes, void *stream)
{
    size_t need = 0;
    const qnn_status st = qnn_expert_plan_workspace_size(slots, experts, &need);
    if (st != QNN_OK) return st;
    if (!offsets || (slots > 0 && (!ids || !order || !position))) return QNN_EINVAL;
    if (!aligned(ids, 4) || !aligned(offsets, 4) || !aligned(order, 4) || !aligned(position, 4)) return QNN_EALIGN;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return QNN_EWORKSPACE;
    return from_cuda(launch_expert_plan(ids, slots, experts, offsets, order, position, workspace,
                                        static_cast<cudaStream_t>(stream)));
}

qnn_status qnn_matmul_image_size(const qnn_matmul_desc *d, size_t *bytes)
{
    if (!bytes) return QNN_EINVAL;
    const qnn_status st = check_matmul(d);
    if (st != QNN_OK) return st;
    *bytes = matmul_image(d->experts, d->m, d->k, d->bits, d->gated).bytes;
    return QNN_OK;
}

qnn_status qnn_matmul_prepare(const qnn_matmul_desc *d, const void *w, const float *scale, const float *bias,
                              void *image, size_t image_bytes, void *stream)
{
    qnn_status st = check_matmul(d);
    if (st != QNN_OK) return st;
    if (!w) return QNN_EINVAL;
    st = check_image(*d, image, image_bytes);
    if (st != QNN_OK) return st;
    if (!aligned(w, d->bits == 16 ? 2 : 1) || !aligned(scale, 4) || !aligned(bias, 4)) return QNN_EALIGN;
    return from_cuda(launch_matmul_prep(*d, w, scale, bias, image, static_cast<cudaStream_t>(stream)));
}

qnn_status qnn_matmul_workspace_size(const qnn_matmul_desc *d, int64_t t, const void *x, int64_t ldx, size_t *bytes)
{
    if (!bytes) return QNN_EINVAL;
    const qnn_status st = check_matmul(d);
    if (st != QNN_OK) return st;
    if (t < 0 || ldx < d->k) return QNN_EINVAL;
    *bytes = staging_bytes(*d, t, 0, false, x, ldx);
    return check_rows(*d, t);
}

qnn_status qnn_matmul_run(const qnn_matmul_desc *d, const void *image, size_t image_bytes, int64_t t, const void *x,
                          int64_t ldx, const void *residual, int64_t ldres, void *y, int64_t ldy, int32_t out_f32,
                          void *workspace, size_t workspace_bytes, void *stream)
{
    size_t need = 0;
    qnn_status st = qnn_matmul_workspace_size(d, t, x, ldx, &need);
    if (st != QNN_OK) return st;
    if (d->experts != 1 || !flag_ok(out_f32) || (t > 0 && (!x || !y))) return QNN_EINVAL;
    if (ldy < d->m || (residual && ldres < d->m)) return QNN_EINVAL;
    st = check_image(*d, image, image_bytes);
    if (st != QNN_OK) return st;
    if (!aligned(x, 2) || !aligned(residual, 2) || !aligned(y, out_f32 ? 4 : 2)) return QNN_EALIGN;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return QNN_EWORKSPACE;
    MatmulArgs a = base_args(*d, image, x, ldx, y, ldy);
    a.residual = residual; a.ldres = ldres; a.out_f32 = out_f32; a.rows = a.x_rows = t;
    return from_cuda(run_product(a, *d, workspace, static_cast<cudaStream_t>(stream)));
}

qnn_status qnn_experts_workspace_size(const qnn_matmul_desc *d, int64_t tokens, int32_t top, int32_t combine,
                                      const void *x, int64_t ldx, size_t *bytes)
{
    if (!bytes || !flag_ok(combine)) return QNN_EINVAL;
    const qnn_status st = check_slots(d, tokens, top);
    if (st != QNN_OK) return st;
    if (ldx < d->k) return QNN_EINVAL;
    const int64_t slots = tokens * top;
    *bytes = staging_bytes(*d, slots, d->experts, !combine, x, ldx);
    if (combine) *bytes += align256(static_cast<size_t>(slots) * combine_ld(*d) * sizeof(float));
    return QNN_OK;
}

qnn_status qnn_experts_dispatch(const qnn_matmul_desc *d, const void *image, size_t image_bytes, int64_t tokens,
                                int32_t top, const int32_t *offsets, const int32_t *order, const void *x, int64_t ldx,
                                void *y, int64_t ldy, void *workspace, size_t workspace_bytes, void *stream)
{
    size_t need = 0;
    qnn_status st = qnn_experts_workspace_size(d, tokens, top, 0, x, ldx, &need);
    if (st != QNN_OK) return st;
    if (!offsets || ldy < d->m || (tokens > 0 && (!order || !x || !y))) return QNN_EINVAL;
    st = check_image(*d, image, image_bytes);
    if (st != QNN_OK) return st;
    if (!aligned(x, 2) || !aligned(y, 2) || !aligned(offsets, 4) || !aligned(order, 4)) return QNN_EALIGN;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return QNN_EWORKSPACE;
    MatmulArgs a = base_args(*d, image, x, ldx, y, ldy);
    a.offsets = offsets; a.order = order; a.top = top; a.gather = 1; a.zero_tail = 1; a.rows = tokens * top;
    a.x_rows = tokens;
    return from_cuda(run_product(a, *d, workspace, static_cast<cudaStream_t>(stream)));
}

qnn_status qnn_experts_combine(const qnn_matmul_desc *d, const void *image, size_t image_bytes, int64_t tokens,
                               int32_t top, const int32_t *offsets, const int32_t *position, const float *weights,
                               const void *x, int64_t ldx, const void *residual, int64_t ldres, void *y, int64_t ldy,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    size_t need = 0;
    qnn_status st = qnn_experts_workspace_size(d, tokens, top, 1, x, ldx, &need);
    if (st != QNN_OK) return st;
    if (!offsets || ldy < d->m || (residual && ldres < d->m)) return QNN_EINVAL;
    if (tokens > 0 && (!position || !weights || !x || !y)) return QNN_EINVAL;
    st = check_image(*d, image, image_bytes);
    if (st != QNN_OK) return st;
    if (!aligned(x, 2) || !aligned(residual, 2) || !aligned(y, 2)) return QNN_EALIGN;
    if (!aligned(offsets, 4) || !aligned(position, 4) || !aligned(weights, 4)) return QNN_EALIGN;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return QNN_EWORKSPACE;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    float *z = static_cast<float *>(workspace);
    MatmulArgs a = base_args(*d, image, x, ldx, z, combine_ld(*d));
    a.offsets = offsets; a.out_f32 = 1; a.rows = a.x_rows = tokens * top; a.top = top;
    const size_t z_bytes = align256(static_cast<size_t>(a.rows) * combine_ld(*d) * sizeof(float));
    const cudaError_t e = run_product(a, *d, static_cast<char *>(workspace) + z_bytes, s);
    if (e != cudaSuccess) return QNN_ECUDA;
    return from_cuda(launch_combine(d->dtype, z, combine_ld(*d), weights, position, tokens, top, d->m, residual, ldres,
                                    y, ldy, s));
}

}  // extern "C"
