// C ABI of the language-model block operators (declared in include/qnn.h): argument validation and dispatch.  Every
// check happens before anything is enqueued; a call that returns an error has launched nothing.
#include <cmath>

#include "block_internal.h"

namespace qnn {
namespace {

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
qnn_status from_cuda(cudaError_t e) { return e == cudaSuccess ? QNN_OK : QNN_ECUDA; }
bool dtype_ok(int32_t t) { return t == QNN_F16 || t == QNN_BF16 || t == QNN_F32; }
uintptr_t dtype_size(int32_t t) { return t == QNN_F32 ? 4 : 2; }
bool flag_ok(int32_t v) { return v == 0 || v == 1; }

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

}  // extern "C"
