// The gradient noise scale of several gradients, and their mean, in one pass over them.
//
// Per element, with deviations d_i = g_i - g_0 from the first gradient (exact in fp64 for 16-bit gradients; equal gradients
// then show no noise at all): sum_i (g_i - mean)^2 = sum d_i^2 - (sum d_i)^2 / B and mean = g_0 + sum d_i / B.  Where g_0 is infinite the
// deviations are those from 0, g_0's own among them: the mean is then infinite, or NaN, as the formula's is.  Bound by reading
// the gradients: about five fp64 operations an element hide behind 2 bytes of it.  Workgroups leave fp64 sums in the workspace
// and a second launch adds them up in their order, so that the result depends on nothing but the gradients.

#include "pollux_host.h"
#include "pollux_rows.h"
#include "pollux_train.h"

#include <algorithm>

namespace px {
namespace {

constexpr int kThreads = 256;

#ifdef __HIP_DEVICE_COMPILE__
// A mean in fp32 on its way to 16 bits, where it is rounded: towards 0, the last bit standing for whatever was cut off.  That bit is far below the middle of two
// neighbours of 16 bits, so that rounding it gives what rounding the mean itself would.
__device__ __forceinline__ float to_be_rounded(double m)
{
    const float f = (float)m;
    unsigned u = __float_as_uint(f);
    if ((double)f != m) u = (u - (fabs((double)f) > fabs(m) ? 1u : 0u)) | 1u;
    return __uint_as_float(u);
}
#endif

template <class E, class M>
__global__ __launch_bounds__(kThreads) void noise_sums(const E *grads, int64_t n, int B, int64_t stride, const float *precondition, M *mean, double2 *sums)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int kAhead = 4;
    double trace = 0.0, norm = 0.0;
    const double over_b = 1.0 / B;
    for (int64_t at = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kVec; at < n; at += (int64_t)gridDim.x * kThreads * kVec) {
        const int64_t left = n - at;
        f32x8 g0 = load8f(grads + at, left);
        double s1[kVec], s2[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const bool infinite = fabsf(g0[i]) == __builtin_inff();
            s1[i] = infinite ? (double)g0[i] : 0.0;
            s2[i] = infinite ? (double)__builtin_inff() : 0.0;
            g0[i] = infinite ? 0.f : g0[i];
        }
        for (int b = 1; b < B; b += kAhead) {
            f32x8 g[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (b + k < B) g[k] = load8f(grads + (b + k) * stride + at, left);
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (b + k < B) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        const double d = (double)g[k][i] - (double)g0[i];
                        s1[i] += d;
                        s2[i] = fma(d, d, s2[i]);
                    }
                }
        }
        f32x8 p, out;
        if (precondition) p = load8f(precondition + at, left);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const double m = (double)g0[i] + s1[i] * over_b;
            out[i] = sizeof(M) == 2 ? to_be_rounded(m) : (float)m;
            if (i < left) {
                const double w = precondition ? (double)p[i] * (double)p[i] : 1.0;
                const double v = fma(-s1[i] * over_b, s1[i], s2[i]);
                trace += w * (v < 0.0 ? 0.0 : v);              // (NaN stays)
                norm += w * (m * m);
            }
        }
        if (mean) store8f(mean + at, left, out);
    }
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) {
        trace += __shfl_xor(trace, w);
        norm += __shfl_xor(norm, w);
    }
    __shared__ double2 waves[kThreads / 64];
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = make_double2(trace, norm);
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int i = 1; i < kThreads / 64; ++i) {
        trace += waves[i].x;
        norm += waves[i].y;
    }
    sums[blockIdx.x] = make_double2(trace, norm);
#endif
}

__global__ __launch_bounds__(kThreads) void noise_join(const double2 *sums, int blocks, int B, double examples, double *scale)
{
    __shared__ double2 shared[kThreads];
    double trace = 0.0, norm = 0.0;
    for (int i = threadIdx.x; i < blocks; i += kThreads) {
        trace += sums[i].x;
        norm += sums[i].y;
    }
    shared[threadIdx.x] = make_double2(trace, norm);
    __syncthreads();
    for (int w = kThreads / 2; w > 0; w >>= 1) {
        if (threadIdx.x < w) {
            shared[threadIdx.x].x += shared[threadIdx.x + w].x;
            shared[threadIdx.x].y += shared[threadIdx.x + w].y;
        }
        __syncthreads();
    }
    if (threadIdx.x != 0) return;
    const double t = shared[0].x * (examples / (B - 1)), e = shared[0].y - t / (examples * B);
    scale[0] = t;
    scale[1] = e;
    scale[2] = t / e;
}

}  // namespace

// Workgroups of the pass: eight a compute unit at most, so that there are few sums to add up.
unsigned noise_blocks(int64_t n)
{
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>((n + kThreads * kVec - 1) / (kThreads * kVec), 2048));
}

int launch_noise_scale(const pollux_noise_dims &d, const void *grads, const float *precondition, void *workspace, void *mean, double *scale,
                       hipStream_t stream)
{
    const unsigned blocks = noise_blocks(d.n);
    auto pass = [&](auto e, auto m) {
        typedef decltype(e) E;
        typedef decltype(m) M;
        hipLaunchKernelGGL((noise_sums<E, M>), dim3(blocks), dim3(kThreads), 0, stream, (const E *)grads, d.n, d.B, d.stride, precondition, (M *)mean, (double2 *)workspace);
    };
    auto with_mean = [&](auto e) {
        switch (d.mean_type) {
            case PX_TYPE_F32: pass(e, 0.f); break;
            case PX_TYPE_BF16: pass(e, (__bf16)0.f); break;
            default: pass(e, (_Float16)0.f); break;
        }
    };
    switch (d.type) {
        case PX_TYPE_F32: with_mean(0.f); break;
        case PX_TYPE_BF16: with_mean((__bf16)0.f); break;
        default: with_mean((_Float16)0.f); break;
    }
    hipLaunchKernelGGL(noise_join, dim3(1), dim3(kThreads), 0, stream, (const double2 *)workspace, (int)blocks, d.B, d.examples, scale);
    return status_of(hipGetLastError());
}

}  // namespace px
