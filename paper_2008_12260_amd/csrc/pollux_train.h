// Host-side declarations of a training iteration's operators (lookup, loss, noise scale, orthogonalised update), shared by
// their translation units: argument structures as checked, workspace layouts, launch functions.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/pollux.h"

namespace px {

int check_device(int *device = nullptr);

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int status_of(hipError_t e) { return e == hipSuccess ? PX_OK : PX_E_HIP; }
inline int size_of_type(int type) { return type == PX_TYPE_F32 ? 4 : 2; }

// A token, or target: -1 where there is none or it is no entry of the vocabulary (then `bad`).
__device__ __forceinline__ int token_at(const void *tokens, int64_t n, bool i64, int V, bool &bad)
{
    const int64_t y = i64 ? ((const int64_t *)tokens)[n] : (int64_t)((const int32_t *)tokens)[n];
    bad = y < -1 || y >= V;
    return y < 0 || y >= V ? -1 : (int)y;
}

// ---- loss ----------------------------------------------------------------------------------------------------------

// How a loss call cuts the vocabulary, and the byte offsets of its workspace's sections.  Lengths of rows in the workspace are
// padded to whole 16-byte groups, the padding holding zeros.
struct LossPlan {
    bool pack_hidden, pack_weight;      // rows that 16-byte loads cannot take are copied to aligned ones first
    int tiles;                          // which shape of tile the logits are formed in (kShape)
    int grad_tiles;                     // and the gradients
    int piece;                          // vocabulary entries taken at a time, a multiple of 256
    int pieces;
    int tokens;                         // forward: taken at a time
    int slices;                         // workgroups that share one tile of the hidden rows' gradient, each a part of a piece
    int64_t d_pad, v_pad;               // padded width, piece
    size_t status, top;                 // int32 [64]; float [64]: the scale of q (fp16)
    size_t parts;                       // float2 [vocabulary tiles, tokens]: largest logit and sum of exponentials
    size_t picked;                      // float [tokens]: the target's logit
    size_t hidden, weight;              // packed copies [N, d_pad] (of the gradients, with zeros for rows that do not count), [piece, d_pad]
    size_t q;                           // q [N, v_pad]
    size_t rest;                        // float [N] (16 bits): what rounding took from the target's q
    size_t sums;                        // float [slices, N, D]: the hidden rows' gradient so far
    size_t total;
};
LossPlan loss_plan(const pollux_loss_dims &d, bool grad);
int launch_token_loss(const pollux_loss_dims &d, const LossPlan &p, const void *hidden, const void *weight, const void *targets,
                      void *workspace, float *loss, float *lse, hipStream_t stream);
int launch_token_loss_grad(const pollux_loss_dims &d, const LossPlan &p, const void *hidden, const void *weight, const void *targets,
                           const float *lse, const float *row_weight, void *workspace, void *hidden_grad, void *weight_grad,
                           hipStream_t stream);

// ---- lookup --------------------------------------------------------------------------------------------------------

struct EmbedPlan {
    int bits;                   // of a pass of the sort
    int passes;                 // 0: few tokens, ranked by one workgroup
    int blocks, per_block;      // workgroups of a pass, tokens of each
    int window, windows;        // places in sorted order that are summed together, and how many such
    size_t status;
    size_t counts;              // int32 [2][blocks][1 << bits]: a workgroup's tokens by digit, for both passes
    size_t keys[2], places[2];  // int32 [N]: tokens and their positions, before and after the last pass
    size_t partial;             // float [2][windows][D]: sums of the runs that a window's first and last place cut
    size_t total;
};
EmbedPlan embed_plan(const pollux_embed_dims &d);
int launch_embed(const pollux_embed_dims &d, const void *tokens, const void *table, void *rows, int32_t *status, hipStream_t stream);
int launch_embed_grad(const pollux_embed_dims &d, const EmbedPlan &p, const void *tokens, const void *rows_grad, void *workspace, void *table_grad,
                      hipStream_t stream);

// ---- noise scale ---------------------------------------------------------------------------------------------------

unsigned noise_blocks(int64_t n);
int launch_noise_scale(const pollux_noise_dims &d, const void *grads, const float *precondition, void *workspace, void *mean, double *scale,
                       hipStream_t stream);

// ---- orthogonalised update -----------------------------------------------------------------------------------------

struct StepShape {
    int shape;                  // of tiles
    bool half;                  // of a symmetric product, only the tiles on one side of the diagonal
};
struct OrthoPlan {
    int m, n;                   // the smaller and the larger side
    bool tall;                  // the gradients have more rows than columns
    int64_t m_pad, x_pad;       // m and cols in whole 16-byte groups
    StepShape shape_gram, shape_square, shape_wide;       // of the products X X', A A and B X
    int norm_blocks;            // a matrix
    double unit;                // X is held times this power of two
    size_t norms;               // double [batch, norm_blocks]
    size_t x[2];                // _Float16 [batch, rows, x_pad]: before and after a step
    size_t low;                 // _Float16 [batch, rows, x_pad]: what rounding left of X, times 2^11
    size_t gram, poly;          // _Float16 [batch, m, m_pad]: X X', b X X' + c (X X')^2
    size_t total;
};
OrthoPlan ortho_plan(const pollux_ortho_dims &d);
int launch_orthogonalize(const pollux_ortho_dims &d, const OrthoPlan &p, const void *grads, void *workspace, void *update, hipStream_t stream);

// ---- residual blocks -----------------------------------------------------------------------------------------------

int launch_keep(const pollux_keep_dims &d, const void *rows, uint8_t *values, uint8_t *scales, hipStream_t stream);
int launch_restore(const pollux_keep_dims &d, const uint8_t *values, const uint8_t *scales, void *rows, hipStream_t stream);
int launch_gated(const pollux_gated_dims &d, const void *gate, const void *up, void *rows, uint8_t *gate_values, uint8_t *gate_scales, uint8_t *up_values,
                 uint8_t *up_scales, hipStream_t stream);
int launch_gated_grad(const pollux_gated_dims &d, const void *rows_grad, const void *gate, const void *up, const uint8_t *gate_scales, const uint8_t *up_scales,
                      void *gate_grad, void *up_grad, void *rows, hipStream_t stream);

struct KeptGradPlan {
    bool pack;                  // rows of rows_grad that 16-byte loads cannot take are copied to aligned ones first
    int tiles;                  // shape of tile
    int slices;                 // workgroups that share a tile, each a part of the rows
    int64_t slice;              // rows of a slice, whole stages
    int64_t m_pad;              // padded row of rows_grad
    int sum_blocks;             // bias: parts of the rows whose sums are joined
    size_t rows;                // packed copy [N, m_pad]
    size_t parts, sums;         // bias: float [sum_blocks, M], [M]: sums of rows_grad over the rows
    size_t slices_at;           // float [slices, M, D]
    size_t total;
};
KeptGradPlan kept_grad_plan(const pollux_kept_grad_dims &d);
int launch_kept_grad(const pollux_kept_grad_dims &d, const KeptGradPlan &p, const uint8_t *values, const uint8_t *scales, const void *rows_grad, const void *weight,
                     const void *bias, void *workspace, void *weight_grad, hipStream_t stream);

// How an edge's rows are shared out: `team` threads have a row between them, eight elements or twice eight each.
struct EdgePlan {
    int vectors;                // of eight elements, a thread
    int team, teams;            // threads of a row; rows that a workgroup has under way at a time
    int chunk;                  // backward: the most rows that a team sums over; neighbours with a gate for each span of rows, else as far apart as there are teams
    int blocks;                 // backward
    size_t parts;               // float [4][blocks][D]: sums over a workgroup's rows
    size_t ends;                // float [blocks * teams][2][D]: the gate's gradient of the spans that a team's first and last row cut
    size_t total;
};
EdgePlan edge_plan(const pollux_edge_dims &d);
struct EdgeArgs;
int launch_block_edge(const pollux_edge_dims &d, const EdgePlan &p, const EdgeArgs &a, hipStream_t stream);
int launch_block_edge_grad(const pollux_edge_dims &d, const EdgePlan &p, const EdgeArgs &a, hipStream_t stream);

// A call's pointers.
struct EdgeArgs {
    const void *x, *branch, *gate, *after_weight, *after_bias, *before_weight, *before_bias;
    void *y, *rows;
    float *y_stats, *branch_stats;
    uint8_t *y_values, *y_scales, *branch_values, *branch_scales;
    // backward
    const void *y_grad, *rows_grad;
    void *x_grad, *branch_grad, *gate_grad, *after_weight_grad, *after_bias_grad, *before_weight_grad, *before_bias_grad;
    char *workspace;
};

}  // namespace px
