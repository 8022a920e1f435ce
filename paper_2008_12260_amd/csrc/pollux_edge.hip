// The edge between two blocks: a norm of the block's result, its gate, the scaled residual and the norm before the next block, in one pass.
//
//   b = n(z) w_a + b_a,  y = residual x + scale gate b,  h = n(y) w_b + b_b,   n(v) = (v - mean) r,  r = 1 / sqrt(mean((v - mean)^2) + eps)
//
// x and z are read once and y and h written once; each norm's sums are formed from registers (the mean first, then the squares of what is left, so that rows
// far from 0 keep their precision).  The normalised rows are kept in 8 bits on the way.  Bound by memory: 16384 x 4096 in bfloat16 98 us, 5.5 TB/s,
// with both kept 139, 4.8 TB/s.  Norms with means and biases have twice the sums, one after the other: 182.
// Rows of more than 8192 from an fp32 residual stream have more than registers hold, 30 of which (58 with biases; all in fp32 5 and 106) go by way of scratch memory: 6000 x 9216 beside 16 bits 144 us (floor 100); 4096 x 16384 in bfloat16, without, both kept, 159 (101).

#include <type_traits>

#include "pollux_edge.h"

#include <algorithm>

namespace px {
namespace {

// BIASED: a norm has biases.
template <class X, class E, int C, bool BRANCH, bool BIASED>
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
    f32x8 w_a[C], w_b[C], b_a[C], b_b[C], gate[C];
    auto gate_of = [&](int k, int64_t row) { return parameters(A.p.gate, d.gate_type, row * D + c[k], left[k], 1.f) * d.scale; };
#pragma unroll
    for (int k = 0; k < C; ++k) {
        c[k] = (k * team + mine) * kVec;
        left[k] = D - c[k];
        w_a[k] = parameters(after ? A.p.after_weight : nullptr, d.weight_type, c[k], left[k], 1.f);
        w_b[k] = parameters(A.p.before_weight, d.weight_type, c[k], left[k], 1.f);
        if (BIASED) {
            b_a[k] = parameters(after ? A.p.after_bias : nullptr, d.weight_type, c[k], left[k], 0.f);
            b_b[k] = parameters(A.p.before_bias, d.weight_type, c[k], left[k], 0.f);
        }
        if (!d.span) gate[k] = gate_of(k, 0);
    }
    const int N = (int)d.N, step = gridDim.x * teams;
    // a row as it comes from memory; the next one's loads are under way while one is worked on
    constexpr bool kAhead = C == 1;
    struct Row {
        Loaded<X> x[C];
        Loaded<E> z[C];
    } next;
    auto load = [&](int64_t row) {
#pragma unroll
        for (int k = 0; k < C; ++k) {
            if (BRANCH) next.z[k].rows((const E *)A.p.branch + row * d.branch_stride + c[k], left[k]);
            next.x[k].rows((const X *)A.p.x + row * d.x_stride + c[k], left[k]);
        }
    };
    int row = blockIdx.x * teams + first;
    if (kAhead && row < N) load(row);
    // (of several wavefronts a row, one team a workgroup: all threads come to every barrier)
    for (; row < N; row += step) {
        if (!kAhead) load(row);
        const Row w = next;
        if (BRANCH && d.span)
#pragma unroll
            for (int k = 0; k < C; ++k) gate[k] = gate_of(k, (uint32_t)row / (uint32_t)d.span);
        if (kAhead && row + step < N) load(row + step);
        // v becomes n(v), its (mean, r) is left
        auto normalise = [&](f32x8(&v)[C], float *stats) {
            float mean[1] = {0.f}, spread[1] = {0.f};
            if (centred) {
#pragma unroll
                for (int k = 0; k < C; ++k) mean[0] += sum8(v[k]);
                over_team(mean, team, shared, parity);
                mean[0] *= over;
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    v[k] -= mean[0];
                    if (A.ragged) v[k] = within(v[k], left[k]);
                }
            }
#pragma unroll
            for (int k = 0; k < C; ++k) spread[0] += squares8(v[k]);
            over_team(spread, team, shared, parity);
            const float r = 1.f / sqrtf(fmaf(spread[0], over, d.eps));
#pragma unroll
            for (int k = 0; k < C; ++k) v[k] *= r;
            if (stats && mine == 0) ((float2 *)stats)[row] = make_float2(mean[0], r);
        };
        auto leave = [&](const f32x8(&v)[C], uint8_t *values, uint8_t *scales) {
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int64_t to = row * width + c[k];
                keep8(d.form, v[k], values + to, scales + to / kKeptGroup, c[k] < width);
            }
        };
        f32x8 y[C], z[C];
        if (BRANCH) {
#pragma unroll
            for (int k = 0; k < C; ++k) z[k] = w.z[k].of_rows();
            if (after) normalise(z, A.p.branch_stats);
            if (A.p.branch_values) leave(z, A.p.branch_values, A.p.branch_scales);
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (after) {
                    z[k] *= w_a[k];
                    if (BIASED) z[k] += b_a[k];
                }
                y[k] = fma8(gate[k], z[k], w.x[k].of_rows() * d.residual);
                store8f((X *)A.p.y + row * d.y_stride + c[k], left[k], y[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < C; ++k) y[k] = w.x[k].of_rows();
        }
        if (!before) continue;
        normalise(y, A.p.y_stats);
        if (A.p.y_values) leave(y, A.p.y_values, A.p.y_scales);
#pragma unroll
        for (int k = 0; k < C; ++k) {
            f32x8 h = y[k] * w_b[k];
            if (BIASED) h += b_b[k];
            store8f((E *)A.p.rows + row * d.rows_stride + c[k], left[k], h);
        }
    }
#endif
}

template <class X, class E, int C>
void launch_rows_of(const EdgePlan &p, const EdgeKernelArgs &a, hipStream_t stream)
{
    const int threads = p.team * p.teams;
    auto launch = [&](auto kernel) {
        // some 16 to 20 wavefronts a compute unit, each of which goes through its rows: 16384 x 4096 in bfloat16 98 us, with twice as many 115, with eight times 102
        const int64_t rows = (a.d.N + p.teams - 1) / p.teams, most = 256 * std::max(1, 1280 / threads);
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(rows, most)), dim3(threads), 0, stream, a);
    };
    const bool biased = a.p.after_bias || a.p.before_bias;
    if (a.p.branch) biased ? launch(edge_rows<X, E, C, true, true>) : launch(edge_rows<X, E, C, true, false>);
    else biased ? launch(edge_rows<X, E, C, false, true>) : launch(edge_rows<X, E, C, false, false>);
}

template <class X, class E>
void launch_rows(const EdgePlan &p, const EdgeKernelArgs &a, hipStream_t stream)
{
    if (p.vectors == 2) launch_rows_of<X, E, 2>(p, a, stream);
    else launch_rows_of<X, E, 1>(p, a, stream);
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
    // Backward: 16 wavefronts a compute unit, which is what its registers hold (20 of rows of 4104 to 5120, two workgroups of ten), but rows enough a team that what it writes of sums, 8 to 16 bytes a
    // column, is little beside the rows.
    const int threads = p.team * p.teams;
    const int64_t teams = 256 * (threads > 512 ? std::max(1, 1280 / threads) : 1024 / threads) * p.teams, least = 4;
    p.chunk = (int)std::max<int64_t>(least, (d.N + teams - 1) / teams);
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
