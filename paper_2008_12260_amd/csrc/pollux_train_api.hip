// C ABI of a training iteration's operators and of a residual block's (see include/pollux.h): argument checks on the host, device check, then the
// launch functions.

#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/pollux.h"
#include "pollux_train.h"

namespace {

bool type_ok(int type) { return type == PX_TYPE_F32 || type == PX_TYPE_BF16 || type == PX_TYPE_F16; }
bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
bool aligned(int type, const void *p) { return ((uintptr_t)p & (uintptr_t)(px::size_of_type(type) - 1)) == 0; }
bool aligned8(const void *p) { return ((uintptr_t)p & 7u) == 0; }
// (rows one after the other may be as wide as their width's own limit)
bool stride_ok(int64_t *stride, int64_t width, int64_t most = (1 << 20) - 1)
{
    if (*stride == 0) *stride = width;
    return *stride == width || (*stride > width && *stride <= most);
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

bool form_ok(int form, bool none) { return form == PX_KEPT_I8 || form == PX_KEPT_E4M3 || (none && form == PX_KEPT_NONE); }
bool rows_ok(int64_t N) { return N >= 0 && N <= (1 << 24); }

bool keep_dims_ok(const pollux_keep_dims *in, pollux_keep_dims *d)
{
    if (!in) return false;
    *d = *in;
    return rows_ok(d->N) && d->D >= 1 && d->D <= (1 << 20) && type_ok(d->type) && form_ok(d->form, false) && d->flags == 0 && stride_ok(&d->rows_stride, d->D);
}

bool kept_grad_dims_ok(const pollux_kept_grad_dims *in, pollux_kept_grad_dims *d)
{
    if (!in) return false;
    *d = *in;
    return rows_ok(d->N) && d->D >= 1 && d->D <= (1 << 16) && d->M >= 1 && d->M <= (1 << 20) && type_ok(d->type) && type_ok(d->weight_type) &&
           form_ok(d->form, false) && !(d->flags & ~PX_FLAG_ACCUMULATE) && stride_ok(&d->rows_grad_stride, d->M) && stride_ok(&d->weight_grad_stride, d->D);
}

bool edge_dims_ok(const pollux_edge_dims *in, pollux_edge_dims *d)
{
    if (!in) return false;
    *d = *in;
    if (!rows_ok(d->N) || d->D < 1 || d->D > (1 << 14) || !type_ok(d->x_type) || !type_ok(d->type) || !type_ok(d->weight_type) || !type_ok(d->gate_type)) return false;
    if ((d->x_type != d->type && d->x_type != PX_TYPE_F32) || !form_ok(d->form, true) || (d->flags & ~(PX_EDGE_AFTER | PX_EDGE_BEFORE | PX_EDGE_CENTRED))) return false;
    if (!isfinite(d->eps) || d->eps < 0.f || !isfinite(d->residual) || !isfinite(d->scale) || d->span < 0) return false;
    if (d->span >= d->N) d->span = 0;                     // one row of the gate for all
    for (int64_t *stride : {&d->x_stride, &d->branch_stride, &d->y_stride, &d->rows_stride, &d->x_grad_stride, &d->branch_grad_stride, &d->y_grad_stride, &d->rows_grad_stride})
        if (!stride_ok(stride, d->D)) return false;
    return true;
}

bool gated_dims_ok(const pollux_gated_dims *in, pollux_gated_dims *d)
{
    if (!in) return false;
    *d = *in;
    if (!rows_ok(d->N) || d->F < 1 || d->F > (1 << 19) || !type_ok(d->type) || !form_ok(d->form, true) || d->flags != 0) return false;
    if (d->act != PX_ACT_SILU && d->act != PX_ACT_GELU && d->act != PX_ACT_GELU_TANH) return false;
    for (int64_t *stride : {&d->gate_stride, &d->up_stride, &d->rows_stride, &d->rows_grad_stride, &d->gate_grad_stride, &d->up_grad_stride})
        if (!stride_ok(stride, d->F, 1 << 20)) return false;             // halves of rows of 2 F
    return true;
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

int pollux_keep(const pollux_keep_dims *dims, const void *rows, uint8_t *values, uint8_t *scales, void *hip_stream)
{
    pollux_keep_dims d;
    if (!keep_dims_ok(dims, &d) || (d.N > 0 && (!rows || !values || !scales)) || !aligned(d.type, rows) || !aligned16(values)) return PX_E_INVALID_ARG;
    const int rc = px::check_device();
    return rc != PX_OK ? rc : px::launch_keep(d, rows, values, scales, (hipStream_t)hip_stream);
}

int pollux_restore(const pollux_keep_dims *dims, const uint8_t *values, const uint8_t *scales, void *rows, void *hip_stream)
{
    pollux_keep_dims d;
    if (!keep_dims_ok(dims, &d) || (d.N > 0 && (!rows || !values || !scales)) || !aligned(d.type, rows) || !aligned16(values)) return PX_E_INVALID_ARG;
    const int rc = px::check_device();
    return rc != PX_OK ? rc : px::launch_restore(d, values, scales, rows, (hipStream_t)hip_stream);
}

int pollux_kept_grad_workspace_size(const pollux_kept_grad_dims *dims, size_t *bytes)
{
    pollux_kept_grad_dims d;
    if (!bytes || !kept_grad_dims_ok(dims, &d)) return PX_E_INVALID_ARG;
    *bytes = px::kept_grad_plan(d).total;
    return PX_OK;
}

int pollux_kept_grad(const pollux_kept_grad_dims *dims, const uint8_t *values, const uint8_t *scales, const void *rows_grad, const void *weight, const void *bias,
                     void *workspace, size_t workspace_bytes, void *weight_grad, void *hip_stream)
{
    pollux_kept_grad_dims d;
    if (!kept_grad_dims_ok(dims, &d) || !weight_grad || (d.N > 0 && (!values || !scales || !rows_grad))) return PX_E_INVALID_ARG;
    if (!aligned16(values) || !aligned16(rows_grad) || !aligned(d.weight_type, weight) || !aligned(d.weight_type, bias) || !aligned16(weight_grad)) return PX_E_INVALID_ARG;
    const px::KeptGradPlan p = px::kept_grad_plan(d);
    int rc = check_workspace(workspace, workspace_bytes, p.total);
    if (rc == PX_OK) rc = px::check_device();
    if (rc != PX_OK) return rc;
    return px::launch_kept_grad(d, p, values, scales, rows_grad, weight, bias, workspace, weight_grad, (hipStream_t)hip_stream);
}

int pollux_block_edge(const pollux_edge_dims *dims, const void *x, const void *branch, const void *gate, const void *after_weight, const void *after_bias,
                      const void *before_weight, const void *before_bias, void *y, void *rows, float *y_stats, float *branch_stats, uint8_t *y_values,
                      uint8_t *y_scales, uint8_t *branch_values, uint8_t *branch_scales, void *hip_stream)
{
    pollux_edge_dims d;
    if (!edge_dims_ok(dims, &d)) return PX_E_INVALID_ARG;
    const bool before = d.flags & PX_EDGE_BEFORE, after = d.flags & PX_EDGE_AFTER;
    // nothing to do without a branch and a norm; what belongs to a part that there is none of is not given
    if (d.N > 0 && !branch && (!before || after || y || gate || branch_stats || branch_values)) return PX_E_INVALID_ARG;
    // (backward, a branch whose rows are not read looks like none: x's gradient is residual g there, and y is x here)
    if (d.N > 0 && !branch && d.residual != 1.f) return PX_E_INVALID_ARG;
    if (!after && (after_weight || after_bias || branch_stats)) return PX_E_INVALID_ARG;
    if (!before && (before_weight || before_bias || rows || y_stats || y_values)) return PX_E_INVALID_ARG;
    if (d.N > 0 && (!y_values != !y_scales || !branch_values != !branch_scales || (d.form == PX_KEPT_NONE && (y_values || branch_values)))) return PX_E_INVALID_ARG;
    if (d.N > 0 && (!x || (branch && !y) || (before && !rows))) return PX_E_INVALID_ARG;
    if (!aligned(d.x_type, x) || !aligned(d.x_type, y) || !aligned(d.type, branch) || !aligned(d.type, rows) || !aligned(d.gate_type, gate)) return PX_E_INVALID_ARG;
    for (const void *p : {after_weight, after_bias, before_weight, before_bias})
        if (!aligned(d.weight_type, p)) return PX_E_INVALID_ARG;
    if (!aligned8(y_stats) || !aligned8(branch_stats) || !aligned16(y_values) || !aligned16(branch_values)) return PX_E_INVALID_ARG;
    if (!gate) d.span = 0;
    const int rc = px::check_device();
    if (rc != PX_OK) return rc;
    px::EdgeArgs a = {};
    a.x = x;
    a.branch = branch;
    a.gate = gate;
    a.after_weight = after_weight;
    a.after_bias = after_bias;
    a.before_weight = before_weight;
    a.before_bias = before_bias;
    a.y = y;
    a.rows = rows;
    a.y_stats = y_stats;
    a.branch_stats = branch_stats;
    a.y_values = y_values;
    a.y_scales = y_scales;
    a.branch_values = branch_values;
    a.branch_scales = branch_scales;
    return px::launch_block_edge(d, px::edge_plan(d), a, (hipStream_t)hip_stream);
}

int pollux_block_edge_workspace_size(const pollux_edge_dims *dims, size_t *bytes)
{
    pollux_edge_dims d;
    if (!bytes || !edge_dims_ok(dims, &d)) return PX_E_INVALID_ARG;
    *bytes = px::edge_plan(d).total;
    return PX_OK;
}

int pollux_block_edge_grad(const pollux_edge_dims *dims, const void *y_grad, const void *rows_grad, const void *y, const void *y_scales, const void *branch,
                           const void *branch_scales, const float *y_stats, const float *branch_stats, const void *gate, const void *after_weight,
                           const void *after_bias, const void *before_weight, void *workspace, size_t workspace_bytes, void *x_grad, void *branch_grad,
                           void *gate_grad, void *after_weight_grad, void *after_bias_grad, void *before_weight_grad, void *before_bias_grad, void *hip_stream)
{
    pollux_edge_dims d;
    if (!edge_dims_ok(dims, &d)) return PX_E_INVALID_ARG;
    const bool before = d.flags & PX_EDGE_BEFORE, after = d.flags & PX_EDGE_AFTER, kept = d.form != PX_KEPT_NONE;
    if (d.N > 0 && !branch && branch_scales) return PX_E_INVALID_ARG;
    if (!after && (after_weight || after_bias || after_weight_grad || after_bias_grad)) return PX_E_INVALID_ARG;
    if (!before && (rows_grad || before_weight || before_weight_grad || before_bias_grad)) return PX_E_INVALID_ARG;
    if (!gate && gate_grad) return PX_E_INVALID_ARG;
    // of the branch, only its norm and the gate's gradient are asked
    const bool asked = after || gate_grad;
    if (d.N > 0) {
        if (before && (!rows_grad || !y || !y_stats || !y_scales != !kept)) return PX_E_INVALID_ARG;
        if ((asked && !branch) || (branch && !branch_scales != !kept) || (after && !branch_stats)) return PX_E_INVALID_ARG;
    }
    if (!aligned(d.x_type, y_grad) || !aligned(d.x_type, x_grad) || !aligned(d.type, rows_grad) || !aligned(d.type, branch_grad)) return PX_E_INVALID_ARG;
    if (kept ? !aligned16(y) || !aligned16(branch) : !aligned(d.x_type, y) || !aligned(d.type, branch)) return PX_E_INVALID_ARG;
    if (!aligned(d.gate_type, gate) || !aligned(d.gate_type, gate_grad) || !aligned8(y_stats) || !aligned8(branch_stats)) return PX_E_INVALID_ARG;
    for (const void *p : {after_weight, after_bias, before_weight, (const void *)after_weight_grad, (const void *)after_bias_grad, (const void *)before_weight_grad, (const void *)before_bias_grad})
        if (!aligned(d.weight_type, p)) return PX_E_INVALID_ARG;
    if (!gate) d.span = 0;
    if (d.N == 0 && dims->span > 0) gate_grad = nullptr;  // no rows of a gate
    const px::EdgePlan plan = px::edge_plan(d);
    int rc = check_workspace(workspace, workspace_bytes, plan.total);
    if (rc == PX_OK) rc = px::check_device();
    if (rc != PX_OK) return rc;
    px::EdgeArgs a = {};
    a.y_grad = y_grad;
    a.rows_grad = rows_grad;
    if (kept) {
        a.y_values = (uint8_t *)y;
        a.y_scales = (uint8_t *)y_scales;
        a.branch_values = asked ? (uint8_t *)branch : nullptr;
        a.branch_scales = (uint8_t *)branch_scales;
    } else {
        a.y = (void *)y;
        a.branch = asked ? branch : nullptr;
    }
    a.y_stats = (float *)y_stats;
    a.branch_stats = (float *)branch_stats;
    a.gate = gate;
    a.after_weight = after_weight;
    a.after_bias = after_bias;
    a.before_weight = before_weight;
    a.x_grad = x_grad;
    a.branch_grad = branch_grad;
    a.gate_grad = gate_grad;
    a.after_weight_grad = after_weight_grad;
    a.after_bias_grad = after_bias_grad;
    a.before_weight_grad = before_weight_grad;
    a.before_bias_grad = before_bias_grad;
    a.workspace = (char *)workspace;
    return px::launch_block_edge_grad(d, plan, a, (hipStream_t)hip_stream);
}

int pollux_gated(const pollux_gated_dims *dims, const void *gate, const void *up, void *rows, uint8_t *gate_values, uint8_t *gate_scales, uint8_t *up_values,
                 uint8_t *up_scales, void *hip_stream)
{
    pollux_gated_dims d;
    if (!gated_dims_ok(dims, &d) || (d.N > 0 && (!gate || !rows))) return PX_E_INVALID_ARG;
    const bool kept = d.form != PX_KEPT_NONE;
    if (d.N > 0 && (!gate_values != !kept || !gate_scales != !kept || !up_values != !(kept && up) || !up_scales != !(kept && up))) return PX_E_INVALID_ARG;
    if (!aligned(d.type, gate) || !aligned(d.type, up) || !aligned(d.type, rows) || !aligned16(gate_values) || !aligned16(up_values)) return PX_E_INVALID_ARG;
    const int rc = px::check_device();
    if (rc != PX_OK) return rc;
    return px::launch_gated(d, gate, up, rows, gate_values, gate_scales, up_values, up_scales, (hipStream_t)hip_stream);
}

int pollux_gated_grad(const pollux_gated_dims *dims, const void *rows_grad, const void *gate, const void *gate_scales, const void *up, const void *up_scales,
                      void *gate_grad, void *up_grad, void *rows, void *hip_stream)
{
    pollux_gated_dims d;
    if (!gated_dims_ok(dims, &d) || (d.N > 0 && (!rows_grad || !gate || (!up && up_grad)))) return PX_E_INVALID_ARG;
    const bool kept = d.form != PX_KEPT_NONE;
    if (d.N > 0 && (!gate_scales != !kept || !up_scales != !(kept && up))) return PX_E_INVALID_ARG;
    if (kept ? !aligned16(gate) || !aligned16(up) : !aligned(d.type, gate) || !aligned(d.type, up)) return PX_E_INVALID_ARG;
    if (!aligned(d.type, rows_grad) || !aligned(d.type, gate_grad) || !aligned(d.type, up_grad) || !aligned(d.type, rows)) return PX_E_INVALID_ARG;
    const int rc = px::check_device();
    if (rc != PX_OK) return rc;
    return px::launch_gated_grad(d, rows_grad, gate, up, (const uint8_t *)gate_scales, (const uint8_t *)up_scales, gate_grad, up_grad, rows, (hipStream_t)hip_stream);
}

}  // extern "C"
