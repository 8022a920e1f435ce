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

bool embed_dims_ok(const pollux_embed_dims *in, pollux_embed_dims *d)
{
    if (!in) return false;
    *d = *in;
    if (d->N < 0 || d->N > (1 << 20) || d->V < 1 || d->V >= (1 << 20) || d->D < 1 || d->D > (1 << 16)) return false;
    if (!type_ok(d->table_type) || !type_ok(d->rows_type) || (d->flags & ~(PX_FLAG_TOKENS_I64 | PX_FLAG_ACCUMULATE)) || !isfinite(d->scale)) return false;
    return stride_ok(&d->table_stride, d->D) && stride_ok(&d->rows_stride, d->D);
}

bool noise_dims_ok(const pollux_noise_dims *in, pollux_noise_dims *d)
{
    if (!in) return false;
    *d = *in;
    if (d->stride == 0) d->stride = d->n;
    return d->n >= 0 && d->n < (1ll << 40) && d->B >= 2 && d->B <= 65536 && type_ok(d->type) && type_ok(d->mean_type) && d->flags == 0 && d->stride >= d->n &&
           d->stride < (1ll << 40) && isfinite(d->examples) && d->examples > 0.0;
}

bool ortho_dims_ok(const pollux_ortho_dims *in, pollux_ortho_dims *d)
{
    if (!in) return false;
    *d = *in;
    if (d->batch < 0 || d->batch > 65535 || d->rows < 1 || d->cols < 1 || d->rows > (1 << 16) || d->cols > (1 << 16) || (d->rows > (1 << 14) && d->cols > (1 << 14))) return false;
    if (!type_ok(d->type) || d->steps < 0 || d->steps > 64 || d->flags != 0 || !isfinite(d->a) || !isfinite(d->b) || !isfinite(d->c)) return false;
    if ((int64_t)d->batch * d->rows * d->cols >= (1ll << 40)) return false;
    if (!stride_ok(&d->grads_stride, d->cols) || !stride_ok(&d->update_stride, d->cols)) return false;
    auto batch_ok = [&](int64_t *batch_stride, int64_t stride) {
        const int64_t one = (d->rows - 1) * stride + d->cols;
        if (*batch_stride == 0) *batch_stride = d->rows * stride;
        return *batch_stride >= one && *batch_stride < (1ll << 40);
    };
    return batch_ok(&d->grads_batch_stride, d->grads_stride) && batch_ok(&d->update_batch_stride, d->update_stride);
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

int pollux_embed(const pollux_embed_dims *dims, const void *tokens, const void *table, void *rows, int32_t *status, void *hip_stream)
{
    pollux_embed_dims d;
    if (!embed_dims_ok(dims, &d) || !table || (d.N > 0 && (!tokens || !rows))) return PX_E_INVALID_ARG;
    if (!aligned16(table) || !aligned16(rows)) return PX_E_INVALID_ARG;
    const int rc = px::check_device();
    if (rc != PX_OK) return rc;
    return px::launch_embed(d, tokens, table, rows, status, (hipStream_t)hip_stream);
}

int pollux_embed_workspace_size(const pollux_embed_dims *dims, size_t *bytes)
{
    pollux_embed_dims d;
    if (!bytes || !embed_dims_ok(dims, &d)) return PX_E_INVALID_ARG;
    *bytes = px::embed_plan(d).total;
    return PX_OK;
}

int pollux_embed_grad(const pollux_embed_dims *dims, const void *tokens, const void *rows_grad, void *workspace, size_t workspace_bytes, void *table_grad,
                      void *hip_stream)
{
    pollux_embed_dims d;
    if (!embed_dims_ok(dims, &d) || !table_grad || (d.N > 0 && (!tokens || !rows_grad))) return PX_E_INVALID_ARG;
    if (!aligned16(table_grad) || !aligned16(rows_grad)) return PX_E_INVALID_ARG;
    const px::EmbedPlan p = px::embed_plan(d);
    int rc = check_workspace(workspace, workspace_bytes, p.total);
    if (rc == PX_OK) rc = px::check_device();
    if (rc != PX_OK) return rc;
    return px::launch_embed_grad(d, p, tokens, rows_grad, workspace, table_grad, (hipStream_t)hip_stream);
}

int pollux_noise_workspace_size(const pollux_noise_dims *dims, size_t *bytes)
{
    pollux_noise_dims d;
    if (!bytes || !noise_dims_ok(dims, &d)) return PX_E_INVALID_ARG;
    *bytes = px::up256(16 * (size_t)px::noise_blocks(d.n));
    return PX_OK;
}

int pollux_noise_scale(const pollux_noise_dims *dims, const void *grads, const float *precondition, void *workspace, size_t workspace_bytes, void *mean,
                       double *scale, void *hip_stream)
{
    pollux_noise_dims d;
    if (!noise_dims_ok(dims, &d) || !scale || (d.n > 0 && !grads)) return PX_E_INVALID_ARG;
    if (!aligned16(grads) || !aligned16(precondition) || !aligned16(mean)) return PX_E_INVALID_ARG;
    int rc = check_workspace(workspace, workspace_bytes, px::up256(16 * (size_t)px::noise_blocks(d.n)));
    if (rc == PX_OK) rc = px::check_device();
    if (rc != PX_OK) return rc;
    return px::launch_noise_scale(d, grads, precondition, workspace, mean, scale, (hipStream_t)hip_stream);
}

int pollux_ortho_workspace_size(const pollux_ortho_dims *dims, size_t *bytes)
{
    pollux_ortho_dims d;
    if (!bytes || !ortho_dims_ok(dims, &d)) return PX_E_INVALID_ARG;
    *bytes = px::ortho_plan(d).total;
    return PX_OK;
}

int pollux_orthogonalize(const pollux_ortho_dims *dims, const void *grads, void *workspace, size_t workspace_bytes, void *update, void *hip_stream)
{
    pollux_ortho_dims d;
    if (!ortho_dims_ok(dims, &d)) return PX_E_INVALID_ARG;
    if (d.batch > 0 && (!grads || !update)) return PX_E_INVALID_ARG;
    if (!aligned16(grads) || !aligned16(update)) return PX_E_INVALID_ARG;
    const px::OrthoPlan p = px::ortho_plan(d);
    int rc = check_workspace(workspace, workspace_bytes, p.total);
    if (rc == PX_OK) rc = px::check_device();
    if (rc != PX_OK) return rc;
    return px::launch_orthogonalize(d, p, grads, workspace, update, (hipStream_t)hip_stream);
}

}  // extern "C"
