// Gradients of the edge between two blocks.
//
//   g  = y_grad + r_y (p - [mean p] - n_y mean(p n_y)),  p = rows_grad w_b          x_grad = residual g
//   t  = scale gate g,  q = t w_a,   branch_grad = r_z (q - [mean q] - n_z mean(q n_z))
//   w_b' = sum rows_grad n_y,  b_b' = sum rows_grad,  w_a' = sum t n_z,  b_a' = sum t,  gate' = scale (w_a sum g n_z + b_a sum g) over the rows of its span
//
// A team goes through neighbouring rows (a chunk) and holds the sums over them in registers, fp32; a workgroup's go out once, and a second launch adds the
// workgroups' in order.  With one gate for all rows, sums of g n_z and g are all that the last three need.  With a gate for each span of rows, they are taken over a
// span, weighted with its gate at its end, and are the gate's gradient there, or, where the chunk's first or last row cuts the span, parts of it.  Bound by memory: 4 rows read, 2 written, 10 bytes
// an element of 16 bits with the normalised rows kept in 8.

#include <type_traits>

#include "pollux_edge.h"

#include <algorithm>

namespace px {
namespace {

enum Part { kBeforeWeight, kBeforeBias, kAfterWeight, kAfterBias, kParts };

template <class X, class E, int C, int R, bool BRANCH, bool SPANS>
__global__ __launch_bounds__(1024) void edge_grads(const EdgeKernelArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    __shared__ float shared[2][kMostWaves][8];
    const pollux_edge_dims &d = A.d;
    const int team = A.team, D = d.D, mine = threadIdx.x & (team <= 64 ? team - 1 : ~0), teams = blockDim.x / team, first = threadIdx.x / team;
    const bool after = d.flags & PX_EDGE_AFTER, before = d.flags & PX_EDGE_BEFORE, centred = d.flags & PX_EDGE_CENTRED;
    const int64_t width = kept_width(D);
    const float over = 1.f / D;
    int parity = 0, c[C], left[C];
    f32x8 w_a[C], w_b[C], gate[C], sum_pn[C], sum_p[C], sum_tn[C], sum_t[C], span_gn[C], span_g[C];
    const f32x8 zeros = {};
#pragma unroll
    for (int k = 0; k < C; ++k) {
        c[k] = (k * team + mine) * kVec;
        left[k] = D - c[k];
        w_a[k] = parameters(after ? A.p.after_weight : nullptr, d.weight_type, c[k], left[k], 1.f);
        w_b[k] = parameters(A.p.before_weight, d.weight_type, c[k], left[k], 1.f);
        gate[k] = parameters(SPANS ? nullptr : A.p.gate, d.gate_type, c[k], left[k], 1.f) * d.scale;
        sum_pn[k] = sum_p[k] = sum_tn[k] = sum_t[k] = span_gn[k] = span_g[k] = zeros;
    }
    const int N = (int)d.N, chunk = blockIdx.x * teams + first;
    const int begin = (int)min((int64_t)chunk * A.chunk, (int64_t)N), end = min(begin + A.chunk, N);
    const bool has_z = A.p.branch || A.p.branch_values;
    const bool after_sums = BRANCH && (A.p.after_weight_grad || A.p.after_bias_grad || A.p.gate_grad), before_sums = before && (A.p.before_weight_grad || A.p.before_bias_grad);
    int span = 0, count;
    for (int row0 = begin; row0 < end; row0 += count) {
        count = min(R, end - row0);
        if (SPANS) {
            const int at = (uint32_t)row0 / (uint32_t)d.span;
            count = (int)min((int64_t)count, (at + 1) * d.span - row0);
            if (row0 == begin || at != span) {
                span = at;
#pragma unroll
                for (int k = 0; k < C; ++k) gate[k] = parameters(A.p.gate, d.gate_type, (int64_t)span * D + c[k], left[k], 1.f) * d.scale;
            }
        }
        int64_t row[R];
#pragma unroll
        for (int r = 0; r < R; ++r) row[r] = row0 + min(r, count - 1);
        f32x8 g[R][C], n_y[R][C], p[R][C], n_z[R][C];
        float2 stats_y[R], stats_z[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (before) stats_y[r] = ((const float2 *)A.p.y_stats)[row[r]];
            if (BRANCH && after) stats_z[r] = ((const float2 *)A.p.branch_stats)[row[r]];
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int64_t kept = min(row[r] * width + c[k], row[r] * width + width - kVec);
                g[r][k] = A.p.y_grad ? load8f((const X *)A.p.y_grad + row[r] * d.y_grad_stride + c[k], left[k]) : zeros;
                if (before) {
                    p[r][k] = load8f((const E *)A.p.rows_grad + row[r] * d.rows_grad_stride + c[k], left[k]);
                    if (d.form) n_y[r][k] = decode8(d.form, *(const u32x2 *)(A.p.y_values + kept), kept_scale(A.p.y_scales[kept / kKeptGroup]));
                    else n_y[r][k] = load8f((const X *)A.p.y + row[r] * d.y_stride + c[k], left[k]);
                }
                if (BRANCH) {
                    if (!has_z) n_z[r][k] = zeros;
                    else if (d.form) n_z[r][k] = decode8(d.form, *(const u32x2 *)(A.p.branch_values + kept), kept_scale(A.p.branch_scales[kept / kKeptGroup]));
                    else n_z[r][k] = load8f((const E *)A.p.branch + row[r] * d.branch_stride + c[k], left[k]);
                }
            }
        }
        if (!d.form)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    if (before) n_y[r][k] = (n_y[r][k] - stats_y[r].x) * stats_y[r].y;
                    if (BRANCH && after) n_z[r][k] = (n_z[r][k] - stats_z[r].x) * stats_z[r].y;
                }
        // v - [mean v] - n mean(v n), times r: the gradient through a norm
        auto through = [&](f32x8(&v)[R][C], const f32x8(&n)[R][C], const float2(&stats)[R]) {
            float along[R], mean[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                along[r] = mean[r] = 0.f;
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        const bool in = !A.ragged || i < left[k];
                        along[r] = fmaf(in ? v[r][k][i] : 0.f, in ? n[r][k][i] : 0.f, along[r]);
                        mean[r] += in ? v[r][k][i] : 0.f;
                    }
            }
            over_team(along, team, shared, parity);
            if (centred) over_team(mean, team, shared, parity);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float a = along[r] * over, m = centred ? mean[r] * over : 0.f;
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) v[r][k][i] = (fmaf(-a, n[r][k][i], v[r][k][i]) - m) * stats[r].y;
            }
        };
        if (before) {
            if (before_sums)
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (r < count)
#pragma unroll
                        for (int k = 0; k < C; ++k) {
#pragma unroll
                            for (int i = 0; i < kVec; ++i) sum_pn[k][i] = fmaf(p[r][k][i], n_y[r][k][i], sum_pn[k][i]);
                            sum_p[k] += p[r][k];
                        }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < C; ++k) p[r][k] *= w_b[k];
            through(p, n_y, stats_y);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < C; ++k) g[r][k] += p[r][k];
        }
        if (A.p.x_grad)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r < count)
#pragma unroll
                    for (int k = 0; k < C; ++k) store8f((X *)A.p.x_grad + row[r] * d.x_grad_stride + c[k], left[k], g[r][k] * d.residual);
        if (!BRANCH) continue;
        if (after_sums)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r < count)
#pragma unroll
                    for (int k = 0; k < C; ++k) {
                        f32x8 &to = SPANS ? span_gn[k] : sum_tn[k];
#pragma unroll
                        for (int i = 0; i < kVec; ++i) to[i] = fmaf(g[r][k][i], n_z[r][k][i], to[i]);
                        (SPANS ? span_g[k] : sum_t[k]) += g[r][k];
                    }
        if (A.p.branch_grad) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    g[r][k] *= gate[k];
                    if (after) g[r][k] *= w_a[k];
                }
            if (after) through(g, n_z, stats_z);
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r < count)
#pragma unroll
                    for (int k = 0; k < C; ++k) store8f((E *)A.p.branch_grad + row[r] * d.branch_grad_stride + c[k], left[k], g[r][k]);
        }
        if (SPANS && after_sums && (row0 + count == end || row0 + count == (span + 1) * d.span)) {
            // the span's last row here: its sums go to where they belong
            const int64_t from = span * d.span, to = from + d.span;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (A.p.gate_grad) {
                    f32x8 v = span_gn[k];
                    if (after) {
                        v *= w_a[k];
                        if (A.p.after_bias) v += span_g[k] * parameters(A.p.after_bias, d.weight_type, c[k], left[k], 0.f);
                    }
                    v *= d.scale;
                    if (from >= begin && min(to, (int64_t)N) <= end) store_parameters(A.p.gate_grad, d.gate_type, (int64_t)span * D + c[k], left[k], v);
                    else store8f(A.ends + ((int64_t)chunk * 2 + (from >= begin ? 1 : 0)) * D + c[k], left[k], v);
                }
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    sum_tn[k][i] = fmaf(gate[k][i], span_gn[k][i], sum_tn[k][i]);
                    sum_t[k][i] = fmaf(gate[k][i], span_g[k][i], sum_t[k][i]);
                }
                span_gn[k] = span_g[k] = zeros;
            }
        }
    }
    // the workgroup's sums: of teams within a wavefront by way of LDS, in their order
    __shared__ float rows[256][kVec + 1];
    auto leave = [&](f32x8(&v)[C], int part) {
        if (team <= 64) {                                 // (C is 1)
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kVec; ++i) rows[threadIdx.x & 255][i] = v[0][i];
            __syncthreads();
            if ((int)threadIdx.x >= team) return;
            for (int t = 1; t < teams; ++t)
#pragma unroll
                for (int i = 0; i < kVec; ++i) v[0][i] += rows[t * team + threadIdx.x][i];
        }
#pragma unroll
        for (int k = 0; k < C; ++k) store8f(A.parts + ((int64_t)part * gridDim.x + blockIdx.x) * D + c[k], left[k], v[k]);
    };
    if (before && A.p.before_weight_grad) leave(sum_pn, kBeforeWeight);
    if (before && A.p.before_bias_grad) leave(sum_p, kBeforeBias);
    if (after_sums) {
        leave(sum_tn, kAfterWeight);
        leave(sum_t, kAfterBias);
    }
#endif
}

// The workgroups' sums added in their order: 64 columns by 16 parts of the list; blockIdx.y: of the norm before, or of the rest.
constexpr int kJoinColumns = 64, kJoinParts = 16;
__global__ __launch_bounds__(kJoinColumns *kJoinParts) void edge_join(const EdgeKernelArgs A, int blocks)
{
#ifdef __HIP_DEVICE_COMPILE__
    __shared__ float shared[kJoinParts][kJoinColumns];
    const pollux_edge_dims &d = A.d;
    const int column = threadIdx.x % kJoinColumns, part = threadIdx.x / kJoinColumns, c = blockIdx.x * kJoinColumns + column;
    auto total = [&](int which) {
        const float *from = A.parts + (int64_t)which * blocks * d.D + c;
        float v = 0.f;
        const int each = (blocks + kJoinParts - 1) / kJoinParts, first = part * each, last = min(first + each, blocks);
        if (c < d.D)
#pragma unroll 8
            for (int b = first; b < last; ++b) v += from[(int64_t)b * d.D];
        __syncthreads();
        shared[part][column] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int k = 0; k < kJoinParts; ++k) v += shared[k][column];
        return v;
    };
    auto put = [&](void *to, int type, float v) {
        if (part != 0 || c >= d.D) return;
        if (type == PX_TYPE_F32) ((float *)to)[c] = v;
        else if (type == PX_TYPE_BF16) ((__bf16 *)to)[c] = (__bf16)v;
        else ((_Float16 *)to)[c] = (_Float16)v;
    };
    auto one = [&](const void *p, int type, float none) {
        if (!p || c >= d.D) return none;
        return type == PX_TYPE_F32 ? ((const float *)p)[c] : type == PX_TYPE_BF16 ? (float)((const __bf16 *)p)[c] : (float)((const _Float16 *)p)[c];
    };
    if (blockIdx.y == 0) {
        if (A.p.before_weight_grad) put(A.p.before_weight_grad, d.weight_type, total(kBeforeWeight));
        if (A.p.before_bias_grad) put(A.p.before_bias_grad, d.weight_type, total(kBeforeBias));
        return;
    }
    const bool shared_gate = d.span == 0;
    const float tn = total(kAfterWeight), t = total(kAfterBias), by = shared_gate ? d.scale * one(A.p.gate, d.gate_type, 1.f) : 1.f;
    if (A.p.after_weight_grad) put(A.p.after_weight_grad, d.weight_type, tn * by);
    if (A.p.after_bias_grad) put(A.p.after_bias_grad, d.weight_type, t * by);
    if (shared_gate && A.p.gate_grad) {
        const bool after = d.flags & PX_EDGE_AFTER;
        const float w = one(after ? A.p.after_weight : nullptr, d.weight_type, 1.f), b = one(after ? A.p.after_bias : nullptr, d.weight_type, 0.f);
        put(A.p.gate_grad, d.gate_type, d.scale * fmaf(w, tn, b == 0.f ? 0.f : b * t));
    }
#endif
}

// Gates of spans that chunks cut: their parts added in order.  A thread a column, a workgroup 256 columns of a span.
__global__ __launch_bounds__(256) void gate_join(const EdgeKernelArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    const pollux_edge_dims &d = A.d;
    const int64_t spans = (d.N + d.span - 1) / d.span;
    const int c = blockIdx.y * 256 + threadIdx.x;
    if (c >= d.D) return;
    for (int64_t s = blockIdx.x; s < spans; s += gridDim.x) {
        const int64_t from = s * d.span, to = min(from + d.span, d.N);
        const int64_t first = from / A.chunk, last = (to - 1) / A.chunk;
        if (first == last) continue;
        float v = A.ends[(first * 2 + 1) * d.D + c];
#pragma unroll 8
        for (int64_t k = first + 1; k <= last; ++k) v += A.ends[k * 2 * d.D + c];
        if (d.gate_type == PX_TYPE_F32) ((float *)A.p.gate_grad)[s * d.D + c] = v;
        else if (d.gate_type == PX_TYPE_BF16) ((__bf16 *)A.p.gate_grad)[s * d.D + c] = (__bf16)v;
        else ((_Float16 *)A.p.gate_grad)[s * d.D + c] = (_Float16)v;
    }
#endif
}

template <class X, class E, int C, int R>
void launch_grads(const EdgePlan &p, const EdgeKernelArgs &a, hipStream_t stream)
{
    const dim3 grid(p.blocks), threads(p.team * p.teams);
    if (!a.p.branch && !a.p.branch_values && !a.p.branch_grad) hipLaunchKernelGGL((edge_grads<X, E, C, R, false, false>), grid, threads, 0, stream, a);
    else if (a.d.span == 0) hipLaunchKernelGGL((edge_grads<X, E, C, R, true, false>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((edge_grads<X, E, C, R, true, true>), grid, threads, 0, stream, a);
}

template <class X, class E>
void launch_grads(const EdgePlan &p, const EdgeKernelArgs &a, hipStream_t stream)
{
    if (p.vectors == 2) launch_grads<X, E, 2, 1>(p, a, stream);
    else launch_grads<X, E, 1, 1>(p, a, stream);
}

}  // namespace

int launch_block_edge_grad(const pollux_edge_dims &d, const EdgePlan &p, const EdgeArgs &args, hipStream_t stream)
{
    EdgeKernelArgs a = {};
    a.d = d;
    a.p = args;
    a.team = p.team;
    a.chunk = p.chunk;
    a.ragged = p.team * p.vectors * kVec != d.D;
    a.parts = (float *)(args.workspace + p.parts);
    a.ends = (float *)(args.workspace + p.ends);
    // (with no rows the sums over them are zeros)
    if (d.N > 0) switch (d.type) {
        case PX_TYPE_F32: launch_grads<float, float>(p, a, stream); break;
        case PX_TYPE_BF16: d.x_type == PX_TYPE_F32 ? launch_grads<float, __bf16>(p, a, stream) : launch_grads<__bf16, __bf16>(p, a, stream); break;
        default: d.x_type == PX_TYPE_F32 ? launch_grads<float, _Float16>(p, a, stream) : launch_grads<_Float16, _Float16>(p, a, stream); break;
    }
    const bool spans = d.span != 0, before = a.p.before_weight_grad || a.p.before_bias_grad, rest = a.p.after_weight_grad || a.p.after_bias_grad || (!spans && a.p.gate_grad);
    if (before || rest) {
        const int columns = (d.D + kJoinColumns - 1) / kJoinColumns;
        hipLaunchKernelGGL(edge_join, dim3(columns, rest ? 2 : 1), dim3(kJoinColumns * kJoinParts), 0, stream, a, d.N > 0 ? p.blocks : 0);
    }
    if (spans && a.p.gate_grad && d.N > 0 && d.span > 1 && (d.N > p.chunk))
        hipLaunchKernelGGL(gate_join, dim3((unsigned)std::min<int64_t>((d.N + d.span - 1) / d.span, 4096), (d.D + 255) / 256), dim3(256), 0, stream, a);
    return status_of(hipGetLastError());
}

}  // namespace px
