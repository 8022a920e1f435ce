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

#ifdef __HIP_DEVICE_COMPILE__
// Eight elements as they came from memory: of rows (T), or codes and their scale's byte.
template <class T>
struct Loaded {
    static constexpr int kWords = sizeof(T) * 2;
    uint32_t words[kWords];
    __device__ __forceinline__ void rows(const T *from, int left)
    {
        typedef uint32_t whole __attribute__((ext_vector_type(kWords)));
        const whole v = __builtin_bit_cast(whole, load8(from, left));
#pragma unroll
        for (int i = 0; i < kWords; ++i) words[i] = v[i];
    }
    __device__ __forceinline__ void kept(const uint8_t *values, const uint8_t *scales, int64_t at)
    {
        const u32x2 codes = *(const u32x2 *)(values + at);
        words[0] = codes[0];
        words[1] = codes[1];
        words[2] = scales[at / kKeptGroup];
    }
    __device__ __forceinline__ f32x8 of_rows() const
    {
        typedef uint32_t whole __attribute__((ext_vector_type(kWords)));
        whole v;
#pragma unroll
        for (int i = 0; i < kWords; ++i) v[i] = words[i];
        return __builtin_convertvector(__builtin_bit_cast(typename Eight<T>::type, v), f32x8);
    }
    // The normalised rows: kept, or formed again.
    __device__ __forceinline__ f32x8 normalised(int form, float2 stats) const
    {
        return form ? decode8(form, u32x2{words[0], words[1]}, kept_scale(words[2])) : (of_rows() - stats.x) * stats.y;
    }
};
__device__ __forceinline__ f32x8 fma8(f32x8 a, f32x8 b, f32x8 c)
{
#pragma unroll
    for (int i = 0; i < kVec; ++i) c[i] = fmaf(a[i], b[i], c[i]);
    return c;
}
#endif

// PLAIN: sums of gradients themselves are wanted too (for biases), not only of their products with normalised rows.
template <class X, class E, int C, int R, bool BRANCH, bool SPANS, bool PLAIN>
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
    // by: what g is multiplied with on its way to the branch's norm, 0 beyond the row's end; so is rows_grad, which is what keeps both out of the rows' sums
    // (read again for every row where they would not fit beside the sums)
    constexpr bool kReload = C > 1;
    f32x8 w_b[C], by[C], sum_pn[C], sum_p[C], sum_tn[C], sum_t[C], span_gn[C], span_g[C];
    const f32x8 zeros = {};
    auto gate_of = [&](int k, int64_t row) { return parameters(A.p.gate, d.gate_type, row * D + c[k], left[k], 1.f) * d.scale; };
    auto after_weight = [&](int k) { return within(parameters(after ? A.p.after_weight : nullptr, d.weight_type, c[k], left[k], 1.f), left[k]); };
#pragma unroll
    for (int k = 0; k < C; ++k) {
        c[k] = (k * team + mine) * kVec;
        left[k] = D - c[k];
        if (!kReload) w_b[k] = parameters(A.p.before_weight, d.weight_type, c[k], left[k], 1.f);
        if (!kReload && BRANCH && !SPANS) by[k] = gate_of(k, 0) * after_weight(k);
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
                for (int k = 0; k < C; ++k)
                    if (!kReload) by[k] = gate_of(k, span) * after_weight(k);
            }
        }
        int64_t row[R];
        Loaded<X> dy[R][C], y[R][C];
        Loaded<E> dh[R][C], z[R][C];
        float2 stats_y[R], stats_z[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            row[r] = row0 + min(r, count - 1);
            if (before) stats_y[r] = ((const float2 *)A.p.y_stats)[row[r]];
            if (BRANCH && after) stats_z[r] = ((const float2 *)A.p.branch_stats)[row[r]];
            else stats_z[r] = make_float2(0.f, 1.f);
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int64_t kept = row[r] * width + min((int64_t)c[k], width - kVec);
                if (before) {
                    dh[r][k].rows((const E *)A.p.rows_grad + row[r] * d.rows_grad_stride + c[k], left[k]);
                    if (d.form) y[r][k].kept(A.p.y_values, A.p.y_scales, kept);
                    else y[r][k].rows((const X *)A.p.y + row[r] * d.y_stride + c[k], left[k]);
                }
                if (A.p.y_grad) dy[r][k].rows((const X *)A.p.y_grad + row[r] * d.y_grad_stride + c[k], left[k]);
                if (BRANCH && has_z) {
                    if (d.form) z[r][k].kept(A.p.branch_values, A.p.branch_scales, kept);
                    else z[r][k].rows((const E *)A.p.branch + row[r] * d.branch_stride + c[k], left[k]);
                }
            }
        }
        f32x8 g[R][C], n[R][C];
        // v - [mean v] - n mean(v n), times r: the gradient through a norm
        auto through = [&](const float2(&stats)[R]) {
            float sums[2 * R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                sums[r] = sums[R + r] = 0.f;
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) sums[r] = fmaf(g[r][k][i], n[r][k][i], sums[r]);
            }
            if (centred) {
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int k = 0; k < C; ++k) sums[R + r] += sum8(g[r][k]);
                over_team(sums, team, shared, parity);
            } else {
                float along[R];
#pragma unroll
                for (int r = 0; r < R; ++r) along[r] = sums[r];
                over_team(along, team, shared, parity);
#pragma unroll
                for (int r = 0; r < R; ++r) sums[r] = along[r];
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float a = -sums[r] * over, m = sums[R + r] * over;
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) g[r][k][i] = (fmaf(a, n[r][k][i], g[r][k][i]) - m) * stats[r].y;
            }
        };
        if (before) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    g[r][k] = dh[r][k].of_rows();
                    n[r][k] = y[r][k].normalised(d.form, stats_y[r]);
                    if (before_sums && r < count) {
                        sum_pn[k] = fma8(g[r][k], n[r][k], sum_pn[k]);
                        if (PLAIN) sum_p[k] += g[r][k];
                    }
                    g[r][k] *= kReload ? parameters(A.p.before_weight, d.weight_type, c[k], left[k], 1.f) : w_b[k];
                }
            through(stats_y);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (!before) g[r][k] = zeros;
                if (A.p.y_grad) g[r][k] += dy[r][k].of_rows();
                if (A.p.x_grad && r < count) store8f((X *)A.p.x_grad + row[r] * d.x_grad_stride + c[k], left[k], g[r][k] * d.residual);
            }
        if (!BRANCH) continue;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int k = 0; k < C; ++k) {
                n[r][k] = has_z ? z[r][k].normalised(d.form, stats_z[r]) : zeros;
                if (after_sums && r < count) {
                    f32x8 &to = SPANS ? span_gn[k] : sum_tn[k];
                    to = fma8(g[r][k], n[r][k], to);
                    if (PLAIN) (SPANS ? span_g[k] : sum_t[k]) += g[r][k];
                }
                g[r][k] *= kReload ? gate_of(k, SPANS ? span : 0) * after_weight(k) : by[k];
            }
        if (A.p.branch_grad) {
            if (after) through(stats_z);
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
                    f32x8 v = span_gn[k] * after_weight(k);
                    if (PLAIN && A.p.after_bias) v = fma8(span_g[k], parameters(A.p.after_bias, d.weight_type, c[k], left[k], 0.f), v);
                    v *= d.scale;
                    if (from >= begin && min(to, (int64_t)N) <= end) store_parameters(A.p.gate_grad, d.gate_type, (int64_t)span * D + c[k], left[k], v);
                    else store8f(A.ends + ((int64_t)chunk * 2 + (from >= begin ? 1 : 0)) * D + c[k], left[k], v);
                }
                const f32x8 gate = gate_of(k, span);
                sum_tn[k] = fma8(gate, span_gn[k], sum_tn[k]);
                if (PLAIN) sum_t[k] = fma8(gate, span_g[k], sum_t[k]);
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
    if (PLAIN && before && A.p.before_bias_grad) leave(sum_p, kBeforeBias);
    if (after_sums) {
        leave(sum_tn, kAfterWeight);
        if (PLAIN) leave(sum_t, kAfterBias);
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
    const bool plain = A.p.after_bias || A.p.after_bias_grad;
    const float tn = total(kAfterWeight), t = plain ? total(kAfterBias) : 0.f, by = shared_gate ? d.scale * one(A.p.gate, d.gate_type, 1.f) : 1.f;
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

template <class X, class E, int C, bool PLAIN>
void launch_grads(const EdgePlan &p, const EdgeKernelArgs &a, hipStream_t stream)
{
    const dim3 grid(p.blocks), threads(p.team * p.teams);
    constexpr int R = C == 1 && sizeof(X) == 2 ? 2 : 1;
    if (!a.p.branch && !a.p.branch_values && !a.p.branch_grad) hipLaunchKernelGGL((edge_grads<X, E, C, R, false, false, PLAIN>), grid, threads, 0, stream, a);
    else if (a.d.span == 0) hipLaunchKernelGGL((edge_grads<X, E, C, 1, true, false, PLAIN>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((edge_grads<X, E, C, 1, true, true, PLAIN>), grid, threads, 0, stream, a);
}

template <class X, class E>
void launch_grads(const EdgePlan &p, const EdgeKernelArgs &a, hipStream_t stream)
{
    const bool plain = a.p.before_bias_grad || a.p.after_bias || a.p.after_bias_grad;
    if (p.vectors == 2) plain ? launch_grads<X, E, 2, true>(p, a, stream) : launch_grads<X, E, 2, false>(p, a, stream);
    else plain ? launch_grads<X, E, 1, true>(p, a, stream) : launch_grads<X, E, 1, false>(p, a, stream);
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
