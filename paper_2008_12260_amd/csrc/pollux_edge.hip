// The edge between two blocks: a norm of the block's result, its gate, the scaled residual and the norm before the next block, in one pass.
//
//   b = n(z) w_a + b_a,  y = residual x + scale gate b,  h = n(y) w_b + b_b,   n(v) = (v - mean) r,  r = 1 / sqrt(mean((v - mean)^2) + eps)
//
// x and z are read once and y and h written once; each norm's sums are formed from registers (the mean first, then the squares of what is left, so that rows
// far from 0 keep their precision).  The normalised rows are kept in 8 bits on the way.  Bound by memory.

#include <type_traits>

#include "pollux_edge.h"

#include <algorithm>

namespace px {
namespace {

template <class X, class E, int C, int R, bool BRANCH>
__global__ __launch_bounds__(1024) void edge_rows(const EdgeKernelArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    __shared__ float shared[2][kMostWaves][8];
    const pollux_edge_dims &d = A.d;
    const int team = A.team, D = d.D, mine = threadIdx.x & (team <= 64 ? team - 1 : ~0), teams = blockDim.x / team, first = threadIdx.x / team;
    const bool after = d.flags & PX_EDGE_AFTER, before = d.flags & PX_EDGE_BEFORE, centred = d.flags & PX_EDGE_CENTRED;
    const int64_t width = kept_width(D);
    const float over = 1.f / D;
    int parity = 0, c[C], left[C];
    f32x8 w_a[C], w_b[C], gate[C];
#pragma unroll
    for (int k = 0; k < C; ++k) {
        c[k] = (k * team + mine) * kVec;
        left[k] = D - c[k];
        w_a[k] = parameters(after ? A.p.after_weight : nullptr, d.weight_type, c[k], left[k], 1.f);
        w_b[k] = parameters(A.p.before_weight, d.weight_type, c[k], left[k], 1.f);
        gate[k] = parameters(d.span ? nullptr : A.p.gate, d.gate_type, c[k], left[k], 1.f) * d.scale;
    }
    const int N = (int)d.N, step = gridDim.x * teams * R;
    // (of several wavefronts a row, one team a workgroup: all threads come to every barrier)
    for (int row0 = (blockIdx.x * teams + first) * R; row0 < N; row0 += step) {
        f32x8 y[R][C], z[R][C];
        int64_t row[R];
#pragma unroll
        for (int r = 0; r < R; ++r) row[r] = min(row0 + r, N - 1);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (BRANCH) z[r][k] = load8f((const E *)A.p.branch + row[r] * d.branch_stride + c[k], left[k]);
                y[r][k] = load8f((const X *)A.p.x + row[r] * d.x_stride + c[k], left[k]);
            }
        // each row of v becomes n(v); [mean, r] of it
        auto normalise = [&](f32x8(&v)[R][C], float(&mean)[R], float(&spread)[R]) {
#pragma unroll
            for (int r = 0; r < R; ++r) mean[r] = 0.f;
            if (centred) {
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int k = 0; k < C; ++k) mean[r] += sum8(v[r][k]);
                over_team(mean, team, shared, parity);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    mean[r] *= over;
#pragma unroll
                    for (int k = 0; k < C; ++k) {
                        v[r][k] -= mean[r];
                        if (A.ragged) v[r][k] = within(v[r][k], left[k]);
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                spread[r] = 0.f;
#pragma unroll
                for (int k = 0; k < C; ++k) spread[r] += squares8(v[r][k]);
            }
            over_team(spread, team, shared, parity);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                spread[r] = 1.f / sqrtf(fmaf(spread[r], over, d.eps));
#pragma unroll
                for (int k = 0; k < C; ++k) v[r][k] *= spread[r];
            }
        };
        auto leave = [&](const f32x8(&v)[R][C], uint8_t *values, uint8_t *scales) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    const int64_t to = row[r] * width + c[k];
                    keep8(d.form, v[r][k], values + to, scales + to / kKeptGroup, row0 + r < N && c[k] < width);
                }
        };
        float mean[R], spread[R];
        if (BRANCH) {
            if (after) {
                normalise(z, mean, spread);
                if (A.p.branch_stats && mine == 0)
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        if (row0 + r < N) ((float2 *)A.p.branch_stats)[row[r]] = make_float2(mean[r], spread[r]);
            }
            if (A.p.branch_values) leave(z, A.p.branch_values, A.p.branch_scales);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    f32x8 b = z[r][k], g = gate[k];
                    if (d.span) g = parameters(A.p.gate, d.gate_type, (int64_t)((uint32_t)row[r] / (uint32_t)d.span) * D + c[k], left[k], 1.f) * d.scale;
                    if (after) {
                        b *= w_a[k];
                        if (A.p.after_bias) b += parameters(A.p.after_bias, d.weight_type, c[k], left[k], 0.f);
                    }
#pragma unroll
                    for (int i = 0; i < kVec; ++i) y[r][k][i] = fmaf(g[i], b[i], d.residual * y[r][k][i]);
                    if (row0 + r < N) store8f((X *)A.p.y + row[r] * d.y_stride + c[k], left[k], y[r][k]);
                }
        }
        if (!before) continue;
        normalise(y, mean, spread);
        if (A.p.y_stats && mine == 0)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (row0 + r < N) ((float2 *)A.p.y_stats)[row[r]] = make_float2(mean[r], spread[r]);
        if (A.p.y_values) leave(y, A.p.y_values, A.p.y_scales);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int k = 0; k < C; ++k) {
                f32x8 h = y[r][k] * w_b[k];
                if (A.p.before_bias) h += parameters(A.p.before_bias, d.weight_type, c[k], left[k], 0.f);
                if (row0 + r < N) store8f((E *)A.p.rows + row[r] * d.rows_stride + c[k], left[k], h);
            }
    }
#endif
}

template <class X, class E>
void launch_rows(const EdgePlan &p, const EdgeKernelArgs &a, hipStream_t stream)
{
    const dim3 threads(p.team * p.teams);
    auto launch = [&](auto kernel, int rows) {
        // four workgroups a compute unit of 256 threads and up to 16 wavefronts in all: more would each load the parameters again
        const int64_t batches = (a.d.N + (int64_t)rows * p.teams - 1) / ((int64_t)rows * p.teams), most = 256 * std::max(1, 1024 / (p.team * p.teams)) * 2;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(batches, most)), threads, 0, stream, a);
    };
    const bool branch = a.p.branch;
    if (p.vectors == 2) branch ? launch(edge_rows<X, E, 2, 1, true>, 1) : launch(edge_rows<X, E, 2, 1, false>, 1);
    else if (a.d.N <= 1024) branch ? launch(edge_rows<X, E, 1, 1, true>, 1) : launch(edge_rows<X, E, 1, 1, false>, 1);
    else branch ? launch(edge_rows<X, E, 1, 2, true>, 2) : launch(edge_rows<X, E, 1, 2, false>, 2);
}

}  // namespace

EdgePlan edge_plan(const pollux_edge_dims &d)
{
    EdgePlan p = {};
    const int eights = (d.D + kVec - 1) / kVec;
    p.vectors = eights > 1024 ? 2 : 1;
    if (eights <= 64) {
        p.team = 4;
        while (p.team < eights) p.team *= 2;
        p.teams = 256 / p.team;
    } else {
        p.team = ((eights + p.vectors - 1) / p.vectors + 63) / 64 * 64;
        p.teams = 1;
    }
    // Backward: 16 wavefronts a compute unit, but rows enough a team that what it writes of sums, 8 to 16 bytes a column, is little beside the rows.
    const int64_t teams = 4096 * 64 / p.team, least = p.team > 64 ? 8 : 4;
    p.chunk = (int)std::max<int64_t>(least, (d.N + teams - 1) / teams);
    p.chunk = (p.chunk + 1) / 2 * 2;
    p.blocks = (int)((d.N + (int64_t)p.chunk * p.teams - 1) / ((int64_t)p.chunk * p.teams));
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o = up256(o + bytes); return at; };
    p.parts = take(4 * (size_t)p.blocks * d.D * 4);
    if (d.span) p.ends = take((size_t)p.blocks * p.teams * 2 * d.D * 4);
    p.total = std::max<size_t>(o, 256);
    return p;
}

int launch_block_edge(const pollux_edge_dims &d, const EdgePlan &p, const EdgeArgs &args, hipStream_t stream)
{
    if (d.N == 0) return PX_OK;
    EdgeKernelArgs a = {};
    a.d = d;
    a.p = args;
    a.team = p.team;
    a.ragged = p.team * p.vectors * kVec != d.D;
    switch (d.type) {
        case PX_TYPE_F32: launch_rows<float, float>(p, a, stream); break;
        case PX_TYPE_BF16: d.x_type == PX_TYPE_F32 ? launch_rows<float, __bf16>(p, a, stream) : launch_rows<__bf16, __bf16>(p, a, stream); break;
        default: d.x_type == PX_TYPE_F32 ? launch_rows<float, _Float16>(p, a, stream) : launch_rows<_Float16, _Float16>(p, a, stream); break;
    }
    return status_of(hipGetLastError());
}

}  // namespace px
