// C ABI of a training iteration's operators (see include/pollux.h): argument checks on the host, device check, then the
// launch functions.

#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/pollux.h"
#include "pollux_train.h"

namespace {

bool type_ok(int type) { return type == PX_TYPE_F32 || type == PX_TYPE_BF16 || type == PX_TYPE_F16; }
bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
bool stride_ok(int64_t *stride, int64_t width)
{
    if (*stride == 0) *stride = width;
    return *stride >= width && *stride < (1 << 20);
}
int check_workspace(const void *ws, size_t bytes, size_t need)
{
    return !ws || ((uintptr_t)ws & 255u) != 0 || bytes < need ? PX_E_WORKSPACE : PX_OK;
}

bool loss_dims_ok(const pollux_loss_dims *in, pollux_loss_dims *d)
{
    if (!in) return false;
    *d = *in;
    if (d->N < 0 || d->N > (1 << 20) || d->V < 1 || d->V > (1 << 20) || d->D < 1 || d->D > (1 << 16)) return false;
    if (!type_ok(d->type) || (d->flags & ~(PX_FLAG_TOKENS_I64 | PX_FLAG_ACCUMULATE))) return false;
    return stride_ok(&d->hidden_stride, d->D) && stride_ok(&d->weight_stride, d->D) && stride_ok(&d->hidden_grad_stride, d->D) &&
           stride_ok(&d->weight_grad_stride, d->D);
}

}  // namespace

extern "C" {

int pollux_loss_workspace_size(const pollux_loss_dims *dims, int32_t with_grad, size_t *bytes)
{
    pollux_loss_dims d;
    if (!bytes || !loss_dims_ok(dims, &d) || (with_grad != 0 && with_grad != 1)) return PX_E_INVALID_ARG;
    *bytes = px::loss_plan(d, with_grad).total;
    return PX_OK;
}

int pollux_token_loss(const pollux_loss_dims *dims, const void *hidden, const void *weight, const void *targets, void *workspace,
                      size_t workspace_bytes, float *loss, float *lse, void *hip_stream)
{
    pollux_loss_dims d;
    if (!loss_dims_ok(dims, &d)) return PX_E_INVALID_ARG;
    if (d.N > 0 && (!hidden || !targets || !loss || !lse)) return PX_E_INVALID_ARG;
    if (!weight || !aligned16(hidden) || !aligned16(weight)) return PX_E_INVALID_ARG;
    const px::LossPlan p = px::loss_plan(d, false);
    int rc = check_workspace(workspace, workspace_bytes, p.total);
    if (rc == PX_OK) rc = px::check_device();
    if (rc != PX_OK) return rc;
    return px::launch_token_loss(d, p, hidden, weight, targets, workspace, loss, lse, (hipStream_t)hip_stream);
}

int pollux_token_loss_grad(const pollux_loss_dims *dims, const void *hidden, const void *weight, const void *targets, const float *lse,
                           const float *row_weight, void *workspace, size_t workspace_bytes, void *hidden_grad, void *weight_grad,
                           void *hip_stream)
{
    pollux_loss_dims d;
    if (!loss_dims_ok(dims, &d)) return PX_E_INVALID_ARG;
    if (d.N > 0 && (!hidden || !targets || !lse)) return PX_E_INVALID_ARG;
    if (!weight || !aligned16(hidden) || !aligned16(weight) || !aligned16(hidden_grad) || !aligned16(weight_grad)) return PX_E_INVALID_ARG;
    const px::LossPlan p = px::loss_plan(d, true);
    int rc = check_workspace(workspace, workspace_bytes, p.total);
    if (rc == PX_OK) rc = px::check_device();
    if (rc != PX_OK) return rc;
    return px::launch_token_loss_grad(d, p, hidden, weight, targets, lse, row_weight, workspace, hidden_grad, weight_grad, (hipStream_t)hip_stream);
}

}  // extern "C"
