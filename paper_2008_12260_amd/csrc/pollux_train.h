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

}  // namespace px
