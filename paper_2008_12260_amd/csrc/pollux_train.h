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
inline int size_of_type(int type) { return type == PX_TYPE_F32 ? 4 : 2; }

// ---- loss ----------------------------------------------------------------------------------------------------------

// How a loss call cuts the vocabulary, and the byte offsets of its workspace's sections.  Lengths of rows in the workspace are
// padded to whole stages of the matrix kernels (128 bytes), the padding holding zeros.
struct LossPlan {
    bool grad;
    bool pack_hidden, pack_weight;      // rows that 16-byte loads cannot take are copied to aligned ones first
    int tiles;                          // which shape of tile the logits are formed in (loss_tiles_shape)
    int grad_tiles;                     // and the gradients
    int piece;                          // vocabulary entries taken at a time, a multiple of 256
    int pieces;
    int slices;                         // workgroups that share one tile of the hidden rows' gradient, each a part of a piece
    int64_t n_pad, d_pad, v_pad;        // padded tokens, width, piece
    size_t status, top;                 // int32 [64]; float [64]: the scale of q (fp16)
    size_t parts;                       // float2 [vocabulary tiles, N]: largest logit and sum of exponentials
    size_t picked;                      // float [N]: the target's logit
    size_t hidden, weight;              // packed copies [N, d_pad], [piece, d_pad]
    size_t q, qt;                       // q [N, v_pad], its transpose [piece, n_pad]
    size_t ht, wt;                      // transposes: hidden [D, n_pad], a piece of the weights [D, v_pad]
    size_t sums;                        // float [slices, N, D]: the hidden rows' gradient so far
    size_t total;
};
LossPlan loss_plan(const pollux_loss_dims &d, bool grad);
int launch_token_loss(const pollux_loss_dims &d, const LossPlan &p, const void *hidden, const void *weight, const void *targets,
                      void *workspace, float *loss, float *lse, hipStream_t stream);
int launch_token_loss_grad(const pollux_loss_dims &d, const LossPlan &p, const void *hidden, const void *weight, const void *targets,
                           const float *lse, const float *row_weight, void *workspace, void *hidden_grad, void *weight_grad,
                           hipStream_t stream);

}  // namespace px
