// Orthogonalised updates: X = G / |G|_F, then `steps` times  A = X X',  B = b A + c A^2,  X <- a X + B X.
//
// All three products are of the matrix kernels' form (k contiguous in both operands) when X is held both as it is and
// transposed: A[i,j] = <X_i, X_j>; A^2 and B X use that A and B are symmetric, so that a row is a column.  The product that
// forms the next X writes both layouts, the second through turned 4 x 4 blocks.  Three launches a step, for all matrices of the
// batch together.
//
// X is held in fp16, times a power of two near the root of its longer side, so that its elements lie well within fp16's range
// whatever the matrix's shape: an element's rounding is then 2^-11 of it, a quarter of what bfloat16 would leave, and the
// steps (each of which multiplies what is small by up to a) stay below the rounding of the bfloat16 result.  A and B have
// elements of 1 or so.  Sums in fp32, the norm in fp64.

#include "pollux_host.h"
#include "pollux_tiles.h"
#include "pollux_train.h"

#include <algorithm>

namespace px {
namespace {

constexpr int kThreads = 256;

template <class E>
__global__ __launch_bounds__(kThreads) void square_sums(const E *grads, int rows, int cols, int64_t ld, int64_t ld_batch, double *sums)
{
    const E *g = grads + blockIdx.y * ld_batch;
    double sum = 0.0;
    for (int r = blockIdx.x; r < rows; r += gridDim.x)
#pragma unroll 4
        for (int c = threadIdx.x; c < cols; c += kThreads) {
            const double v = (double)(float)g[r * ld + c];
            sum = fma(v, v, sum);
        }
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) sum += __shfl_xor(sum, w);
    __shared__ double waves[kThreads / 64];
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) sums[blockIdx.y * gridDim.x + blockIdx.x] = waves[0] + waves[1] + waves[2] + waves[3];
}

// X and its transpose from the gradients (tall: of their transposes), 64 x 64 at a time, rows padded with zeros.
template <class E>
__global__ __launch_bounds__(kThreads) void normalise(const E *grads, int rows, int cols, int64_t ld, int64_t ld_batch, const double *sums, int parts, double unit, _Float16 *as_is,
                                                      int64_t ld_as, _Float16 *turned_to, int64_t ld_turned)
{
    __shared__ float tile[64][65];
    __shared__ double waves[kThreads / 64];
    const int64_t batch = blockIdx.z;
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) sum += sums[batch * parts + i];
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) sum += __shfl_xor(sum, w);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = waves[0] + waves[1] + waves[2] + waves[3];
    const double by = sum == 0.0 ? 0.0 : unit / sqrt(sum);
    const E *g = grads + batch * ld_batch;
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, x = threadIdx.x & 63, y = threadIdx.x >> 6;
    for (int i = y; i < 64; i += 4) {
        const int r = r0 + i, c = c0 + x;
        const float v = r < rows && c < cols ? (float)((double)(float)g[r * ld + c] * by) : 0.f;
        tile[i][x] = v;
        if (r < rows && c < ld_as) as_is[(batch * rows + r) * ld_as + c] = (_Float16)v;
    }
    __syncthreads();
    for (int i = y; i < 64; i += 4) {
        const int c = c0 + i, r = r0 + x;
        if (c < cols && r < ld_turned) turned_to[(batch * cols + c) * ld_turned + r] = (_Float16)tile[x][i];
    }
}

struct StepArgs {
    Operands o;
    int64_t batch_a, batch_b;           // bytes from matrix to matrix
    int tiles_m, tiles_n, group;
    int cols, rows;                     // m and n of the product
    float by;                           // of the product
    float plus;                         // of `base`
    const _Float16 *base;               // [rows, ld]: added; null: nothing
    _Float16 *out;                      // [rows, ld]
    _Float16 *out_turned;               // [cols, ld_turned], or null
    int64_t ld, ld_turned;              // elements, padded
    __bf16 *last;                       // the update itself in place of `out`: [rows, ld_last]
    int64_t ld_last, batch_last;
};

// out = plus base + by (product), and its transpose; or the update.
template <class S>
__global__ __launch_bounds__(S::kThreads) void step_tiles(const StepArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    extern __shared__ __align__(16) char lds[];
    const Tile t = tile_of(blockIdx.x, A.tiles_m, A.tiles_n, A.group);
    const int64_t batch = blockIdx.y;
    Operands o = A.o;
    o.a += batch * A.batch_a;
    o.b += batch * A.batch_b;
    f32x4 acc[S::FM][S::FN];
    tile_product<S>(o, t, lds, acc);
    const Place<S> at(t);
    const bool whole = (A.ld_last & 3) == 0 && (A.batch_last & 3) == 0 && ((uintptr_t)A.last & 7) == 0;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int n = at.first_n + j * 16;
#pragma unroll
        for (int i = 0; i < S::FM; ++i) {
            const int m = at.first_m + 16 * i;
            f32x4 v = acc[i][j] * A.by;
            const int64_t here = (batch * A.rows + n) * A.ld + m;
            const bool inside = n < A.rows && m < A.ld;
            if (A.base && inside) v += A.plus * __builtin_convertvector(*(const f16x4 *)(A.base + here), f32x4);
            if (A.last) {
                if (n >= A.rows) continue;
                __bf16 *to = A.last + batch * A.batch_last + (int64_t)n * A.ld_last + m;
                if (whole && m + 4 <= A.cols) store4<Bf16>(to, v);
                else
                    for (int r = 0; r < 4; ++r)
                        if (m + r < A.cols) to[r] = (__bf16)v[r];
                continue;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (m + r >= A.cols || n >= A.rows) v[r] = 0.f;
            if (inside) store4<F16>(A.out + here, v);
            if (A.out_turned) {
                const f32x4 w = turned(v);
                const int row = m + (threadIdx.x & 3), col = n & ~3;
                if (row < A.cols && col < A.ld_turned) store4<F16>(A.out_turned + (batch * A.cols + row) * A.ld_turned + col, w);
            }
        }
    }
#endif
}

template <class S>
void launch_step(StepArgs a, int batch, hipStream_t stream)
{
    a.tiles_m = (a.cols + S::BM - 1) / S::BM;
    a.tiles_n = (a.rows + S::BN - 1) / S::BN;
    a.group = 8;
    hipLaunchKernelGGL(step_tiles<S>, dim3((unsigned)(a.tiles_m * a.tiles_n), (unsigned)batch), dim3(S::kThreads), S::kLds, stream, a);
}
void launch_step(int shape, const StepArgs &a, int batch, hipStream_t stream)
{
    switch (shape) {
        case 0: launch_step<Shape0<F16>>(a, batch, stream); break;
        case 1: launch_step<Shape1<F16>>(a, batch, stream); break;
        default: launch_step<Shape2<F16>>(a, batch, stream); break;
    }
}

// The update where no step is taken: X itself.
template <class E>
__global__ __launch_bounds__(kThreads) void normalise_only(const E *grads, int rows, int cols, int64_t ld, int64_t ld_batch, const double *sums, int parts, __bf16 *out, int64_t ld_out,
                                                           int64_t ld_out_batch)
{
    const int64_t batch = blockIdx.z;
    double sum = 0.0;
    for (int i = 0; i < parts; ++i) sum += sums[batch * parts + i];
    const double by = sum == 0.0 ? 0.0 : 1.0 / sqrt(sum);
    for (int r = blockIdx.y; r < rows; r += gridDim.y)
        for (int c = blockIdx.x * kThreads + threadIdx.x; c < cols; c += gridDim.x * kThreads)
            out[batch * ld_out_batch + r * ld_out + c] = (__bf16)(float)((double)(float)grads[batch * ld_batch + r * ld + c] * by);
}

template <class E>
int orthogonalize(const pollux_ortho_dims &d, const OrthoPlan &p, const E *grads, char *ws, __bf16 *update, hipStream_t stream)
{
    double *norms = (double *)(ws + p.norms);
    hipLaunchKernelGGL(square_sums<E>, dim3(p.norm_blocks, d.batch), dim3(kThreads), 0, stream, grads, d.rows, d.cols, d.grads_stride, d.grads_batch_stride, norms);
    if (d.steps == 0) {
        hipLaunchKernelGGL(normalise_only<E>, dim3((unsigned)std::min(16, (d.cols + kThreads - 1) / kThreads), (unsigned)std::min(256, d.rows), (unsigned)d.batch), dim3(kThreads), 0, stream,
                           grads, d.rows, d.cols, d.grads_stride, d.grads_batch_stride, (const double *)norms, p.norm_blocks, update, d.update_stride, d.update_batch_stride);
        return status_of(hipGetLastError());
    }
    _Float16 *x[2] = {(_Float16 *)(ws + p.x[0]), (_Float16 *)(ws + p.x[1])}, *xt[2] = {(_Float16 *)(ws + p.xt[0]), (_Float16 *)(ws + p.xt[1])};
    _Float16 *gram = (_Float16 *)(ws + p.gram), *poly = (_Float16 *)(ws + p.poly);
    // X is [m, n]: the gradients as they are, or, of more rows than columns, transposed
    const int64_t pad_as = p.tall ? p.m_pad : p.n_pad, pad_turned = p.tall ? p.n_pad : p.m_pad;
    hipLaunchKernelGGL(normalise<E>, dim3((unsigned)((pad_as + 63) / 64), (unsigned)((pad_turned + 63) / 64), (unsigned)d.batch), dim3(kThreads), 0, stream, grads, d.rows, d.cols,
                       d.grads_stride, d.grads_batch_stride, (const double *)norms, p.norm_blocks, p.unit, p.tall ? xt[0] : x[0], pad_as, p.tall ? x[0] : xt[0], pad_turned);
    for (int s = 0; s < d.steps; ++s) {
        const _Float16 *from = x[s & 1], *from_t = xt[s & 1];
        StepArgs a = {};
        // gram = X X'
        a.o = {(const char *)from, (const char *)from, p.n_pad * 2, p.n_pad * 2, p.m, p.m, (int)p.n_pad * 2};
        a.batch_a = a.batch_b = p.m * p.n_pad * 2;
        a.cols = a.rows = p.m;
        a.by = (float)(1.0 / (p.unit * p.unit));
        a.out = gram;
        a.ld = p.m_pad;
        launch_step(p.shape_square, a, d.batch, stream);
        // poly = b gram + c gram gram
        a.o = {(const char *)gram, (const char *)gram, p.m_pad * 2, p.m_pad * 2, p.m, p.m, (int)p.m_pad * 2};
        a.batch_a = a.batch_b = p.m * p.m_pad * 2;
        a.by = (float)d.c;
        a.plus = (float)d.b;
        a.base = gram;
        a.out = poly;
        launch_step(p.shape_square, a, d.batch, stream);
        // X = a X + poly X; the last one as the update, in the gradients' own layout
        const bool last = s + 1 == d.steps;
        a.by = 1.f;
        a.plus = (float)d.a;
        if (last) {
            a.by /= (float)p.unit;
            a.plus /= (float)p.unit;
            a.last = update;
            a.ld_last = d.update_stride;
            a.batch_last = d.update_batch_stride;
        }
        if (last && p.tall) {                   // X' [n, m] = a X' + X' poly
            a.o = {(const char *)poly, (const char *)from_t, p.m_pad * 2, p.m_pad * 2, p.m, p.n, (int)p.m_pad * 2};
            a.batch_a = p.m * p.m_pad * 2;
            a.batch_b = p.n * p.m_pad * 2;
            a.cols = p.m;
            a.rows = p.n;
            a.base = from_t;
            a.ld = p.m_pad;
        } else {
            a.o = {(const char *)from_t, (const char *)poly, p.m_pad * 2, p.m_pad * 2, p.n, p.m, (int)p.m_pad * 2};
            a.batch_a = p.n * p.m_pad * 2;
            a.batch_b = p.m * p.m_pad * 2;
            a.cols = p.n;
            a.rows = p.m;
            a.base = from;
            a.out = x[(s + 1) & 1];
            a.ld = p.n_pad;
            a.out_turned = xt[(s + 1) & 1];
            a.ld_turned = p.m_pad;
        }
        launch_step(p.shape_wide, a, d.batch, stream);
    }
    return status_of(hipGetLastError());
}

}  // namespace

OrthoPlan ortho_plan(const pollux_ortho_dims &d)
{
    OrthoPlan p = {};
    p.tall = d.rows > d.cols;
    p.m = std::min(d.rows, d.cols);
    p.n = std::max(d.rows, d.cols);
    p.m_pad = (p.m + 7) / 8 * 8;
    p.n_pad = (p.n + 7) / 8 * 8;
    p.unit = ldexp(1.0, (int)lround(0.5 * log2((double)p.n)));
    p.norm_blocks = (int)std::min<int64_t>(d.rows, std::max<int64_t>(1, std::min<int64_t>(1024 / std::max(d.batch, 1) + 1, (int64_t)d.rows * d.cols / 4096)));
    p.shape_square = std::min(2, shape_for(p.m, p.m, d.batch, false));
    p.shape_wide = std::min(2, shape_for(p.n, p.m, d.batch, false));
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o = up256(o + bytes); return at; };
    p.norms = take(std::max<size_t>(8, 8 * (size_t)d.batch * p.norm_blocks));
    if (d.steps > 0) {
        for (int i = 0; i < (d.steps > 1 ? 2 : 1); ++i) {
            p.x[i] = take(2 * (size_t)d.batch * p.m * p.n_pad);
            p.xt[i] = take(2 * (size_t)d.batch * p.n * p.m_pad);
        }
        p.gram = take(2 * (size_t)d.batch * p.m * p.m_pad);
        p.poly = take(2 * (size_t)d.batch * p.m * p.m_pad);
    }
    p.total = o;
    return p;
}

int launch_orthogonalize(const pollux_ortho_dims &d, const OrthoPlan &p, const void *grads, void *workspace, void *update, hipStream_t stream)
{
    if (d.batch == 0) return PX_OK;
    char *ws = (char *)workspace;
    switch (d.type) {
        case PX_TYPE_F32: return orthogonalize(d, p, (const float *)grads, ws, (__bf16 *)update, stream);
        case PX_TYPE_BF16: return orthogonalize(d, p, (const __bf16 *)grads, ws, (__bf16 *)update, stream);
        default: return orthogonalize(d, p, (const _Float16 *)grads, ws, (__bf16 *)update, stream);
    }
}

}  // namespace px
