// Rows kept in 8 bits and restored, and gated activations with their gradients: every element is read once and written once, with a few
// tens of operations between.
//
//   a = act(g) u;   dg = da u act'(g),  du = da act(g),  with g and u as they are or as 8 bits hold them
//
// Eight neighbouring elements a thread, four threads a group of 32; the threads of a launch walk the rows' groups of eight in order, whatever the
// rows' length, so that short rows fill wavefronts as long ones do.  All are bound by memory: in bfloat16 16384 x 8192 kept as i8 in 72 to 87 us and restored in 66 (4.7 to 5.7 and 6.2 TB/s), 8192 x 16384
// of any of the three activations 147 us, with both inputs kept 210 (5.5 and 5.1 TB/s), gradients and rows from what is kept 257 (5.2).

#include "pollux_host.h"
#include "pollux_kept.h"
#include "pollux_rows.h"
#include "pollux_train.h"

#include <algorithm>

namespace px {
namespace {

constexpr int kThreads = 256;

#ifdef __HIP_DEVICE_COMPILE__
// Row and column of the thread's next eight elements, of rows cut in `groups` eights: one division a thread.
struct Walk {
    int64_t row, rows, by_row;
    int group, groups, by_group;
    __device__ __forceinline__ Walk(int64_t rows_, int groups_) : rows(rows_), groups(groups_)
    {
        const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x, step = (int64_t)gridDim.x * kThreads;
        row = at / groups;
        group = (int)(at - row * groups);
        by_row = step / groups;
        by_group = (int)(step - by_row * groups);
    }
    // (of four threads of a group, all or none)
    __device__ __forceinline__ bool there() const { return row < rows; }
    __device__ __forceinline__ void next()
    {
        row += by_row;
        group += by_group;
        if (group >= groups) group -= groups, ++row;
    }
};
#endif

template <class E>
__global__ __launch_bounds__(kThreads) void keep_rows(const E *rows, int64_t ld, int64_t N, int D, int form, uint8_t *values, uint8_t *scales)
{
#ifdef __HIP_DEVICE_COMPILE__
    const int64_t width = kept_width(D);
    for (Walk at(N, (int)(width / kVec)); at.there(); at.next()) {
        const int c = at.group * kVec;
        keep_loaded(form, load8(rows + at.row * ld + c, D - c), values + at.row * width + c, scales + (at.row * width + c) / kKeptGroup);
    }
#endif
}

template <class E>
__global__ __launch_bounds__(kThreads) void restore_rows(const uint8_t *values, const uint8_t *scales, int64_t N, int D, int form, E *rows, int64_t ld)
{
#ifdef __HIP_DEVICE_COMPILE__
    const int64_t width = kept_width(D);
    for (Walk at(N, (int)((D + kVec - 1) / kVec)); at.there(); at.next()) {
        const int c = at.group * kVec;
        const int64_t from = at.row * width + c;
        store8f(rows + at.row * ld + c, D - c, decode8(form, *(const u32x2 *)(values + from), kept_scale(scales[from / kKeptGroup])));
    }
#endif
}

#ifdef __HIP_DEVICE_COMPILE__
// exp(x) and 1 / x.  Of results of 16 bits by the hardware's functions as they are, within 2^-23 of themselves and 2^-24 |x| for x's product with log2 e: vector operations bound these kernels otherwise (8192 x 16384
// in bfloat16 with both inputs kept, silu 229 us and gelu 262 with the library's, vector units 0.97 busy).
template <class E>
__device__ __forceinline__ float exp_of(float x)
{
    return sizeof(E) == 2 ? __builtin_amdgcn_exp2f(x * 1.44269504088896340736f) : expf(x);
}
template <class E>
__device__ __forceinline__ float over(float x)
{
    return sizeof(E) == 2 ? __builtin_amdgcn_rcpf(x) : 1.f / x;
}

// a b, 0 where either is 0.
__device__ __forceinline__ float times(float a, float b)
{
    float c;
    asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(c) : "v"(a), "v"(b));
    return c;
}

// An activation and its derivative.  Each is g p with p from 0 to 1; where p, or what is left of 1, is 0, so are the products with it, whatever g is.
struct Activated {
    float value, slope;
};
template <class E, int ACT>
__device__ __forceinline__ Activated activated(float g)
{
    Activated a;
    if constexpr (ACT == PX_ACT_GELU) {
        // p = Phi(g) from the side on which it is small: erfc(z) = t exp(P(t)) exp(-z^2), t = 1 / (1 + z / 2), P the Chebyshev fit of Numerical Recipes (second edition, 6.2), within 1.2e-7 of itself for
        // every z >= 0;  z^2 = g^2 / 2 is the density's exponent too
        constexpr float c[10] = {-1.26551223f, 1.00002368f, 0.37409196f, 0.09678418f, -0.18628806f, 0.27886807f, -1.13520398f, 1.48851587f, -0.82215223f, 0.17087277f};
        const float z = fabsf(g) * 0.70710678118654752440f, t = over<E>(fmaf(z, 0.5f, 1.f));
        float fit = c[9];
#pragma unroll
        for (int i = 8; i >= 0; --i) fit = fmaf(fit, t, c[i]);
        const float bell = exp_of<E>(-0.5f * g * g), tail = 0.5f * t * exp_of<E>(fit) * bell, density = bell * 0.39894228040143267794f;
        const float p = g < 0.f ? tail : 1.f - tail;
        a.value = times(g, p);
        a.slope = p + times(g, density);
    } else {
        float inner = g, by = 1.f;
        if constexpr (ACT == PX_ACT_GELU_TANH) {
            // 1/2 (1 + tanh t) = 1 / (1 + exp(-2 t)),  t = sqrt(2 / pi) (g + 0.044715 g^3)
            constexpr float k = 1.59576912160573071176f;
            const float square = g * g;
            inner = k * g * fmaf(0.044715f, square, 1.f);
            by = k * fmaf(3 * 0.044715f, square, 1.f);
        }
        const float e = exp_of<E>(-fabsf(inner)), r = over<E>(1.f + e), small = e * r;           // both sides of p from what is below 1
        const float p = inner < 0.f ? small : r;
        float more = times(g, r * small);
        if constexpr (ACT == PX_ACT_GELU_TANH) more = times(more, by);
        a.value = times(g, p);
        a.slope = p + more;
    }
    return a;
}
#endif

struct GatedArgs {
    int64_t N;
    int F;
    int form;
    const void *gate, *up;                          // rows, or null where codes are given; up: null for an activation alone
    int64_t gate_stride, up_stride;
    uint8_t *gate_values, *gate_scales, *up_values, *up_scales;
    const void *rows_grad;                          // backward
    void *rows, *gate_grad, *up_grad;
    int64_t rows_grad_stride, rows_stride, gate_grad_stride, up_grad_stride;
};

template <class E, int ACT>
__global__ __launch_bounds__(kThreads) void gated_rows(const GatedArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    const int64_t width = kept_width(A.F);
    for (Walk at(A.N, (int)(width / kVec)); at.there(); at.next()) {
        const int c = at.group * kVec, left = A.F - c;
        const auto gate = load8((const E *)A.gate + at.row * A.gate_stride + c, left);
        typename Eight<E>::type up = {};
        if (A.up) up = load8((const E *)A.up + at.row * A.up_stride + c, left);
        const f32x8 g = __builtin_convertvector(gate, f32x8), u = __builtin_convertvector(up, f32x8);
        f32x8 a;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float v = activated<E, ACT>(g[i]).value;
            a[i] = A.up ? v * u[i] : v;
        }
        store8f((E *)A.rows + at.row * A.rows_stride + c, left, a);
        if (A.form) {
            const int64_t to = at.row * width + c;
            keep_loaded(A.form, gate, A.gate_values + to, A.gate_scales + to / kKeptGroup);
            if (A.up) keep_loaded(A.form, up, A.up_values + to, A.up_scales + to / kKeptGroup);
        }
    }
#endif
}

template <class E, int ACT>
__global__ __launch_bounds__(kThreads) void gated_grads(const GatedArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    const int64_t width = kept_width(A.F);
    const bool has_up = A.up || A.up_values;
    for (Walk at(A.N, (int)((A.F + kVec - 1) / kVec)); at.there(); at.next()) {
        const int c = at.group * kVec, left = A.F - c;
        const f32x8 d = load8f((const E *)A.rows_grad + at.row * A.rows_grad_stride + c, left);
        f32x8 g, u = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        if (A.form) {
            const int64_t from = at.row * width + c;
            const u32x2 codes = *(const u32x2 *)(A.gate_values + from);
            const uint32_t byte = A.gate_scales[from / kKeptGroup];
            if (has_up) u = decode8(A.form, *(const u32x2 *)(A.up_values + from), kept_scale(A.up_scales[from / kKeptGroup]));
            g = decode8(A.form, codes, kept_scale(byte));
        } else {
            g = load8f((const E *)A.gate + at.row * A.gate_stride + c, left);
            if (has_up) u = load8f((const E *)A.up + at.row * A.up_stride + c, left);
        }
        f32x8 dg, du, a;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const Activated v = activated<E, ACT>(g[i]);
            dg[i] = d[i] * u[i] * v.slope;
            du[i] = d[i] * v.value;
            a[i] = v.value * u[i];
        }
        if (A.gate_grad) store8f((E *)A.gate_grad + at.row * A.gate_grad_stride + c, left, dg);
        if (has_up && A.up_grad) store8f((E *)A.up_grad + at.row * A.up_grad_stride + c, left, du);
        if (A.rows) store8f((E *)A.rows + at.row * A.rows_stride + c, left, a);
    }
#endif
}

unsigned blocks_for(int64_t N, int64_t width) { return (unsigned)std::min<int64_t>((N * (width / kVec) + kThreads - 1) / kThreads, 8192); }

template <class F>
void of_type(int type, F f)
{
    switch (type) {
        case PX_TYPE_F32: f(0.f); break;
        case PX_TYPE_BF16: f((__bf16)0.f); break;
        default: f((_Float16)0.f); break;
    }
}

template <bool GRAD, class E>
void launch_gated_of(int act, const GatedArgs &a, hipStream_t stream)
{
    const dim3 grid(blocks_for(a.N, kept_width(a.F)));
    auto launch = [&](auto forward, auto backward) {
        if constexpr (GRAD) hipLaunchKernelGGL(backward, grid, dim3(kThreads), 0, stream, a);
        else hipLaunchKernelGGL(forward, grid, dim3(kThreads), 0, stream, a);
    };
    switch (act) {
        case PX_ACT_SILU: launch(gated_rows<E, PX_ACT_SILU>, gated_grads<E, PX_ACT_SILU>); break;
        case PX_ACT_GELU: launch(gated_rows<E, PX_ACT_GELU>, gated_grads<E, PX_ACT_GELU>); break;
        default: launch(gated_rows<E, PX_ACT_GELU_TANH>, gated_grads<E, PX_ACT_GELU_TANH>); break;
    }
}

}  // namespace

int launch_keep(const pollux_keep_dims &d, const void *rows, uint8_t *values, uint8_t *scales, hipStream_t stream)
{
    if (d.N == 0) return PX_OK;
    of_type(d.type, [&](auto e) {
        typedef decltype(e) E;
        hipLaunchKernelGGL(keep_rows<E>, dim3(blocks_for(d.N, kept_width(d.D))), dim3(kThreads), 0, stream, (const E *)rows, d.rows_stride, d.N, d.D, d.form, values, scales);
    });
    return status_of(hipGetLastError());
}

int launch_restore(const pollux_keep_dims &d, const uint8_t *values, const uint8_t *scales, void *rows, hipStream_t stream)
{
    if (d.N == 0) return PX_OK;
    of_type(d.type, [&](auto e) {
        typedef decltype(e) E;
        hipLaunchKernelGGL(restore_rows<E>, dim3(blocks_for(d.N, kept_width(d.D))), dim3(kThreads), 0, stream, values, scales, d.N, d.D, d.form, (E *)rows, d.rows_stride);
    });
    return status_of(hipGetLastError());
}

int launch_gated(const pollux_gated_dims &d, const void *gate, const void *up, void *rows, uint8_t *gate_values, uint8_t *gate_scales, uint8_t *up_values,
                 uint8_t *up_scales, hipStream_t stream)
{
    if (d.N == 0) return PX_OK;
    GatedArgs a = {};
    a.N = d.N;
    a.F = d.F;
    a.form = d.form;
    a.gate = gate;
    a.up = up;
    a.gate_stride = d.gate_stride;
    a.up_stride = d.up_stride;
    a.rows = rows;
    a.rows_stride = d.rows_stride;
    a.gate_values = gate_values;
    a.gate_scales = gate_scales;
    a.up_values = up_values;
    a.up_scales = up_scales;
    of_type(d.type, [&](auto e) { launch_gated_of<false, decltype(e)>(d.act, a, stream); });
    return status_of(hipGetLastError());
}

int launch_gated_grad(const pollux_gated_dims &d, const void *rows_grad, const void *gate, const void *up, const uint8_t *gate_scales, const uint8_t *up_scales,
                      void *gate_grad, void *up_grad, void *rows, hipStream_t stream)
{
    if (d.N == 0) return PX_OK;
    GatedArgs a = {};
    a.N = d.N;
    a.F = d.F;
    a.form = d.form;
    if (d.form) {
        a.gate_values = (uint8_t *)gate;
        a.gate_scales = (uint8_t *)gate_scales;
        a.up_values = (uint8_t *)up;
        a.up_scales = (uint8_t *)up_scales;
    } else {
        a.gate = gate;
        a.up = up;
        a.gate_stride = d.gate_stride;
        a.up_stride = d.up_stride;
    }
    a.rows_grad = rows_grad;
    a.rows_grad_stride = d.rows_grad_stride;
    a.gate_grad = gate_grad;
    a.gate_grad_stride = d.gate_grad_stride;
    a.up_grad = up_grad;
    a.up_grad_stride = d.up_grad_stride;
    a.rows = rows;
    a.rows_stride = d.rows_stride;
    of_type(d.type, [&](auto e) { launch_gated_of<true, decltype(e)>(d.act, a, stream); });
    return status_of(hipGetLastError());
}

}  // namespace px
