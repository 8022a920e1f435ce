// Gradients of the edge between two blocks.
//
//   g  = y_grad + r_y (p - [mean p] - n_y mean(p n_y)),  p = rows_grad w_b          x_grad = residual g
//   t  = scale gate g,  q = t w_a,   branch_grad = r_z (q - [mean q] - n_z mean(q n_z))
//   w_b' = sum rows_grad n_y,  b_b' = sum rows_grad,  w_a' = sum t n_z,  b_a' = sum t,  gate' = scale (w_a sum g n_z + b_a sum g) over the rows of its span
//
// A team goes through some of the rows and holds the sums over them in registers, fp32; a workgroup's go out once, and a second launch adds the
// workgroups' in order.  With one gate for all rows, sums of g n_z and g are all that the last three need.  With a gate for each span of rows, they are taken over a
// span, weighted with its gate at its end, and are the gate's gradient there, or, where the team's first or last row cuts the span, parts of it.  Bound by memory: 4 rows read, 2 written, 10 bytes
// an element of 16 bits with the normalised rows kept in 8: 16384 x 4096 145 us, 4.6 TB/s (a copy moves 4.6 to 4.8), and 6 for the join; from rows of 16 bits 170.  Rows of more than 8192 have
// more sums than registers: two of them wait in LDS, and some of the rest goes by way of scratch memory: 4096 x 16384 306 us (364 without LDS), with a gate a sequence 418 (1344).

#include <type_traits>

#include "pollux_edge.h"

#include <algorithm>

namespace px {
namespace {

enum Part { kBeforeWeight, kBeforeBias, kAfterWeight, kAfterBias, kParts };

// MOST: threads of a workgroup; with spans, whose sums need the most registers, 512 where rows allow it (3003 x 1000 with biases 64 us within the registers of 1024).
// PLAIN: sums of gradients themselves are wanted too (for biases), not only of their products with normalised rows.
template <class X, class E, int C, bool BRANCH, bool SPANS, bool PLAIN, int MOST>
__global__ __launch_bounds__(MOST) void edge_grads(const EdgeKernelArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    __shared__ float shared[2][kMostWaves][8];
    const pollux_edge_dims &d = A.d;
    const int team = A.team, D = d.D, mine = threadIdx.x & (team <= 64 ? team - 1 : ~0), teams = blockDim.x / team, first = threadIdx.x / team;
    const bool after = d.flags & PX_EDGE_AFTER, before = d.flags & PX_EDGE_BEFORE, centred = d.flags & PX_EDGE_CENTRED;
    const int64_t width = kept_width(D);
    const float over = 1.f / D;
    int parity = 0, c[C], left[C];
    // by: what g is multiplied with on its way to the branch's norm, 0 beyond the row's end; so is rows_grad, which is what keeps both out of the rows' sums
    // (read again for every row where they would not fit beside the sums)
    constexpr bool kReload = C > 1;
    f32x8 w_b[C], by[C], sum_pn[C], sum_p[C], sum_tn[C], sum_t[C], span_gn[C], span_g[C];
    const f32x8 zeros = {};
    // (and the sums of products wait in LDS: 64 bytes a sum and thread, in and out once a row, beside 160 from memory)
    constexpr bool kHeld = C > 1;
    extern __shared__ float4 held[];
    auto recall = [&](int which, int k) {
        const float4 a = held[(which * C + k) * 2 * blockDim.x + threadIdx.x], b = held[((which * C + k) * 2 + 1) * blockDim.x + threadIdx.x];
        return f32x8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    };
    auto hold = [&](int which, int k, f32x8 v) {
        held[(which * C + k) * 2 * blockDim.x + threadIdx.x] = make_float4(v[0], v[1], v[2], v[3]);
        held[((which * C + k) * 2 + 1) * blockDim.x + threadIdx.x] = make_float4(v[4], v[5], v[6], v[7]);
    };
    auto gate_of = [&](int k, int64_t row) { return parameters(A.p.gate, d.gate_type, row * D + c[k], left[k], 1.f) * d.scale; };
    auto after_weight = [&](int k) { return within(parameters(after ? A.p.after_weight : nullptr, d.weight_type, c[k], left[k], 1.f), left[k]); };
#pragma unroll
    for (int k = 0; k < C; ++k) {
        c[k] = (k * team + mine) * kVec;
        left[k] = D - c[k];
        if (!kReload) w_b[k] = parameters(A.p.before_weight, d.weight_type, c[k], left[k], 1.f);
        if (!kReload && BRANCH && !SPANS) by[k] = gate_of(k, 0) * after_weight(k);
        sum_pn[k] = sum_p[k] = sum_tn[k] = sum_t[k] = span_gn[k] = span_g[k] = zeros;
        if (kHeld) {
            hold(0, k, zeros);
            hold(1, k, zeros);
        }
    }
    // with spans a team's rows are neighbours, else as far apart as there are teams: the chip is then at neighbouring rows at any time
    const int N = (int)d.N, chunk = blockIdx.x * teams + first, step = SPANS ? 1 : gridDim.x * teams;
    const int begin = SPANS ? (int)min((int64_t)chunk * A.chunk, (int64_t)N) : chunk, end = SPANS ? min(begin + A.chunk, N) : N;
    const bool has_z = A.p.branch || A.p.branch_values;
    const bool after_sums = BRANCH && (A.p.after_weight_grad || A.p.after_bias_grad || A.p.gate_grad), before_sums = before && (A.p.before_weight_grad || A.p.before_bias_grad);
    // a row as it comes from memory; the next one's loads are under way while one is worked on, where registers hold both: 8192 x 8192 from i8 146 us (164
    // without), 4096 x 16384 752 (372)
    constexpr bool kAhead = C == 1 && !SPANS && sizeof(X) == 2;
    struct Row {
        Loaded<X> dy[C], y[C];
        Loaded<E> dh[C], z[C];
        float2 stats_y, stats_z;
    };
    auto load = [&](Row &w, int at) {
        const int64_t row = at;
        if (before) w.stats_y = ((const float2 *)A.p.y_stats)[row];
        w.stats_z = BRANCH && after ? ((const float2 *)A.p.branch_stats)[row] : make_float2(0.f, 1.f);
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int64_t kept = row * width + min((int64_t)c[k], width - kVec);
            if (before) {
                w.dh[k].rows((const E *)A.p.rows_grad + row * d.rows_grad_stride + c[k], left[k]);
                if (d.form) w.y[k].kept(A.p.y_values, A.p.y_scales, kept);
                else w.y[k].rows((const X *)A.p.y + row * d.y_stride + c[k], left[k]);
            }
            if (A.p.y_grad) w.dy[k].rows((const X *)A.p.y_grad + row * d.y_grad_stride + c[k], left[k]);
            if (BRANCH && has_z) {
                if (d.form) w.z[k].kept(A.p.branch_values, A.p.branch_scales, kept);
                else w.z[k].rows((const E *)A.p.branch + row * d.branch_stride + c[k], left[k]);
            }
        }
    };
    int span = 0;
    Row next;
    if (kAhead && begin < end) load(next, begin);
    for (int row = begin; row < end; row += step) {
        if (!kAhead) load(next, row);
        const Row w = next;
        if (kAhead && row + step < end) load(next, row + step);
        if (SPANS) {
            const int at = (uint32_t)row / (uint32_t)d.span;
            if (row == begin || at != span) {
                span = at;
#pragma unroll
                for (int k = 0; k < C; ++k)
                    if (!kReload) by[k] = gate_of(k, span) * after_weight(k);
            }
        }
        f32x8 g[C], n[C];
        // v - [mean v] - n mean(v n), times r: the gradient through a norm
        auto through = [&](float2 stats) {
            float sums[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < C; ++k) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) sums[0] = fmaf(g[k][i], n[k][i], sums[0]);
                if (centred) sums[1] += sum8(g[k]);
            }
            if (centred) {
                over_team(sums, team, shared, parity);
            } else {
                float along[1] = {sums[0]};
                over_team(along, team, shared, parity);
                sums[0] = along[0];
            }
            const float a = -sums[0] * over, m = sums[1] * over;
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int i = 0; i < kVec; ++i) g[k][i] = (fmaf(a, n[k][i], g[k][i]) - m) * stats.y;
        };
        if (before) {
#pragma unroll
            for (int k = 0; k < C; ++k) {
                g[k] = w.dh[k].of_rows();
                n[k] = w.y[k].normalised(d.form, w.stats_y);
                if (before_sums) {
                    if (kHeld) hold(0, k, fma8(g[k], n[k], recall(0, k)));
                    else sum_pn[k] = fma8(g[k], n[k], sum_pn[k]);
                    if (PLAIN) sum_p[k] += g[k];
                }
                g[k] *= kReload ? parameters(A.p.before_weight, d.weight_type, c[k], left[k], 1.f) : w_b[k];
            }
            through(w.stats_y);
        }
#pragma unroll
        for (int k = 0; k < C; ++k) {
            if (!before) g[k] = zeros;
            if (A.p.y_grad) g[k] += w.dy[k].of_rows();
            if (A.p.x_grad) store8f((X *)A.p.x_grad + row * d.x_grad_stride + c[k], left[k], g[k] * d.residual);
        }
        if (!BRANCH) continue;
#pragma unroll
        for (int k = 0; k < C; ++k) {
            n[k] = has_z ? w.z[k].normalised(d.form, w.stats_z) : zeros;
            if (after_sums) {
                if (SPANS) span_gn[k] = fma8(g[k], n[k], span_gn[k]);
                else if (kHeld) hold(1, k, fma8(g[k], n[k], recall(1, k)));
                else sum_tn[k] = fma8(g[k], n[k], sum_tn[k]);
                if (PLAIN) (SPANS ? span_g[k] : sum_t[k]) += g[k];
            }
            g[k] *= kReload ? gate_of(k, SPANS ? span : 0) * after_weight(k) : by[k];
        }
        if (A.p.branch_grad) {
            if (after) through(w.stats_z);
#pragma unroll
            for (int k = 0; k < C; ++k) store8f((E *)A.p.branch_grad + row * d.branch_grad_stride + c[k], left[k], g[k]);
        }
        if (SPANS && after_sums && (row + 1 == end || row + 1 == (span + 1) * d.span)) {
            // the span's last row here: its sums go to where they belong
            const int64_t from = span * d.span, to = from + d.span;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (A.p.gate_grad) {
                    f32x8 v = span_gn[k] * after_weight(k);
                    if (PLAIN && A.p.after_bias) v = fma8(span_g[k], parameters(A.p.after_bias, d.weight_type, c[k], left[k], 0.f), v);
                    v *= d.scale;
                    if (from >= begin && min(to, (int64_t)N) <= end) store_parameters(A.p.gate_grad, d.gate_type, (int64_t)span * D + c[k], left[k], v);
                    else store8f(A.ends + ((int64_t)chunk * 2 + (from >= begin ? 1 : 0)) * D + c[k], left[k], v);
                }
                const f32x8 gate = gate_of(k, span);
                if (kHeld) hold(1, k, fma8(gate, span_gn[k], recall(1, k)));
                else sum_tn[k] = fma8(gate, span_gn[k], sum_tn[k]);
                if (PLAIN) sum_t[k] = fma8(gate, span_g[k], sum_t[k]);
                span_gn[k] = span_g[k] = zeros;
            }
        }
    }
    if (kHeld)
#pragma unroll
        for (int k = 0; k < C; ++k) {
            sum_pn[k] = recall(0, k);
            sum_tn[k] = recall(1, k);
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
    if (PLAIN && before && A.p.before_bias_grad) leave(sum_p, kBeforeBias);
    if (after_sums) {
        leave(sum_tn, kAfterWeight);
        if (PLAIN) leave(sum_t, kAfterBias);
    }
#endif
}

// The workgroups' sums added in their order: 64 columns by 16 parts of a list.  blockIdx.y: of the norm before, of the rest, and from 2 on of the gates of spans that chunks cut, `cuts` of them.
constexpr int kJoinColumns = 64, kJoinParts = 16;
__global__ __launch_bounds__(kJoinColumns *kJoinParts) void edge_join(const EdgeKernelArgs A, int blocks, int chunks, bool rest, int cuts)
{
#ifdef __HIP_DEVICE_COMPILE__
    __shared__ float shared[kJoinParts][kJoinColumns];
    const pollux_edge_dims &d = A.d;
    const int column = threadIdx.x % kJoinColumns, part = threadIdx.x / kJoinColumns, c = blockIdx.x * kJoinColumns + column;
    // of `count` rows of D, `step` elements apart
    auto total = [&](const float *from, int count, int64_t step) {
        float v = 0.f;
        const int each = (count + kJoinParts - 1) / kJoinParts, first = part * each, last = min(first + each, count);
        if (c < d.D)
#pragma unroll 8
            for (int b = first; b < last; ++b) v += from[b * step + c];
        __syncthreads();
        shared[part][column] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int k = 0; k < kJoinParts; ++k) v += shared[k][column];
        return v;
    };
    auto put = [&](void *to, int type, int64_t at, float v) {
        if (part != 0 || c >= d.D) return;
        if (type == PX_TYPE_F32) ((float *)to)[at + c] = v;
        else if (type == PX_TYPE_BF16) ((__bf16 *)to)[at + c] = (__bf16)v;
        else ((_Float16 *)to)[at + c] = (_Float16)v;
    };
    auto one = [&](const void *p, int type, float none) {
        if (!p || c >= d.D) return none;
        return type == PX_TYPE_F32 ? ((const float *)p)[c] : type == PX_TYPE_BF16 ? (float)((const __bf16 *)p)[c] : (float)((const _Float16 *)p)[c];
    };
    auto sum = [&](int which) { return total(A.parts + (int64_t)which * blocks * d.D, blocks, d.D); };
    if (blockIdx.y == 0) {
        if (A.p.before_weight_grad) put(A.p.before_weight_grad, d.weight_type, 0, sum(kBeforeWeight));
        if (A.p.before_bias_grad) put(A.p.before_bias_grad, d.weight_type, 0, sum(kBeforeBias));
        return;
    }
    if (blockIdx.y == 1) {
        if (!rest) return;
        const bool shared_gate = d.span == 0, plain = A.p.after_bias || A.p.after_bias_grad;
        const float tn = sum(kAfterWeight), t = plain ? sum(kAfterBias) : 0.f, by = shared_gate ? d.scale * one(A.p.gate, d.gate_type, 1.f) : 1.f;
        if (A.p.after_weight_grad) put(A.p.after_weight_grad, d.weight_type, 0, tn * by);
        if (A.p.after_bias_grad) put(A.p.after_bias_grad, d.weight_type, 0, t * by);
        if (shared_gate && A.p.gate_grad) {
            const bool after = d.flags & PX_EDGE_AFTER;
            const float w = one(after ? A.p.after_weight : nullptr, d.weight_type, 1.f), b = one(after ? A.p.after_bias : nullptr, d.weight_type, 0.f);
            put(A.p.gate_grad, d.gate_type, 0, d.scale * fmaf(w, tn, b == 0.f ? 0.f : b * t));
        }
        return;
    }
    // one a span, or, of more spans than borders of chunks, one a border: the span that it cuts, if it is the first to
    const int64_t spans = (d.N + d.span - 1) / d.span;
    for (int k = blockIdx.y - 2; k < cuts; k += gridDim.y - 2) {
        const int64_t s = spans <= chunks - 1 ? k : ((int64_t)(k + 1) * A.chunk - 1) / d.span;
        const int64_t from = s * d.span, to = min(from + d.span, d.N), first = from / A.chunk, last = (to - 1) / A.chunk;
        if (first == last || (spans > chunks - 1 && first != k)) continue;
        // the first chunk's last span, the others' first
        const float head = c < d.D ? A.ends[(first * 2 + 1) * d.D + c] : 0.f;
        put(A.p.gate_grad, d.gate_type, s * d.D, head + total(A.ends + (first + 1) * 2 * d.D, (int)(last - first), 2 * d.D));
    }
#endif
}

template <class X, class E, int C>
void launch_grads_of(const EdgePlan &p, const EdgeKernelArgs &a, hipStream_t stream)
{
    const bool plain = a.p.before_bias_grad || a.p.after_bias || a.p.after_bias_grad, branch = a.p.branch || a.p.branch_values || a.p.branch_grad;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(p.blocks), dim3(p.team * p.teams), C > 1 ? 2 * C * kVec * 4 * p.team : 0, stream, a); };
    if (branch && a.d.span && C == 1 && p.team <= 512) plain ? launch(edge_grads<X, E, 1, true, true, true, 512>) : launch(edge_grads<X, E, 1, true, true, false, 512>);
    else if (branch && a.d.span) plain ? launch(edge_grads<X, E, C, true, true, true, 1024>) : launch(edge_grads<X, E, C, true, true, false, 1024>);
    else if (branch) plain ? launch(edge_grads<X, E, C, true, false, true, 1024>) : launch(edge_grads<X, E, C, true, false, false, 1024>);
    else plain ? launch(edge_grads<X, E, C, false, false, true, 1024>) : launch(edge_grads<X, E, C, false, false, false, 1024>);
}

template <class X, class E>
void launch_grads(const EdgePlan &p, const EdgeKernelArgs &a, hipStream_t stream)
{
    if (p.vectors == 2) launch_grads_of<X, E, 2>(p, a, stream);
    else launch_grads_of<X, E, 1>(p, a, stream);
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
    const int chunks = (int)((d.N + p.chunk - 1) / p.chunk);
    const int cuts = spans && d.span > 1 && a.p.gate_grad && d.N > 0 ? (int)std::min<int64_t>((d.N + d.span - 1) / d.span, chunks - 1) : 0;
    if (before || rest || cuts > 0)
        hipLaunchKernelGGL(edge_join, dim3((d.D + kJoinColumns - 1) / kJoinColumns, cuts > 0 ? 2 + std::min(cuts, 4096) : rest ? 2 : 1), dim3(kJoinColumns * kJoinParts), 0, stream, a,
                           d.N > 0 ? p.blocks : 0, chunks, rest, cuts);
    return status_of(hipGetLastError());
}

}  // namespace px
