// Orthogonalised updates: X = G / |G|_F, then `steps` times  A = X X',  B = b A + c A^2,  X <- a X + B X.
//
// X is held as the gradients lie.  Of at most as many rows as columns: A = X X' takes rows, and B X the columns of X; of more rows
// than columns (the formula on the transposes): A = X' X takes columns, and X B the rows.  A^2, A and B are symmetric, so that a row is
// a column, and where that is less work only the tiles on one side of their diagonals are formed.  Three launches a step, for all matrices of the batch together.
//
// The products take X in fp16, times a power of two near the root of its longer side, so that its elements lie well within fp16's range
// whatever the matrix's shape: an element's rounding is then 2^-11 of it, a quarter of what bfloat16 would leave.  A and B have
// elements of 1 or so.  Sums in fp32, the norm in fp64.  What the roundings of a product's operands leave stays among the directions that X has: B acts
// on X from one side, and what it puts outside X's other side is a slight turn of those directions.  The term a X does not: it multiplies the rounding of X in a direction
// that the gradient has none of by a, in every step (by 485 in five of the default coefficients), and of a gradient of low rank those
// are nearly all.  So beside X stands what its rounding left, in fp16 times 2^11: both together are X to within 2^-22 of each element, and a X is taken from both.
// (1024 x 1024 of rank 1, five steps: off by 1.7e-3 of the update's size, the rounding of the result; 0.15 with X alone.  The rest costs two bytes an element in and out a step:
// 8192 x 4096 2.25 ms and 2.13 without, twelve of 384 x 640 142 us and 133.)

#include "pollux_host.h"
#include "pollux_rows.h"
#include "pollux_tiles.h"
#include "pollux_train.h"

#include <algorithm>

namespace px {
namespace {

constexpr int kThreads = 256;

template <class E>
__global__ __launch_bounds__(kThreads) void square_sums(const E *grads, int rows, int cols, int64_t ld, int64_t ld_batch, double *sums)
{
#ifdef __HIP_DEVICE_COMPILE__
    const E *g = grads + blockIdx.y * ld_batch;
    double sum = 0.0;
    const int groups = (cols + kVec - 1) / kVec;
    const int64_t total = (int64_t)rows * groups;
#pragma unroll 2
    for (int64_t at = blockIdx.x * (int64_t)kThreads + threadIdx.x; at < total; at += gridDim.x * (int64_t)kThreads) {
        const int64_t r = at / groups;
        const int c = (int)(at - r * groups) * kVec;
        const f32x8 v = load8f(g + r * ld + c, cols - c);
#pragma unroll
        for (int i = 0; i < kVec; ++i) sum = fma((double)v[i], (double)v[i], sum);
    }
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) sum += __shfl_xor(sum, w);
    __shared__ double waves[kThreads / 64];
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) sums[blockIdx.y * gridDim.x + blockIdx.x] = waves[0] + waves[1] + waves[2] + waves[3];
#endif
}

// What rounding a value to fp16 left of it, as it is held.
#ifdef __HIP_DEVICE_COMPILE__
constexpr float kLowUnit = 2048.f;
__device__ __forceinline__ _Float16 low_part(float v, _Float16 rounded) { return (_Float16)((v - (float)rounded) * kLowUnit); }
#endif

// X from the gradients, rows padded with zeros.
template <class E>
__global__ __launch_bounds__(kThreads) void normalise(const E *grads, int rows, int cols, int64_t ld, int64_t ld_batch, const double *sums, int parts, double unit, _Float16 *x, _Float16 *low, int64_t ld_x)
{
#ifdef __HIP_DEVICE_COMPILE__
    __shared__ double waves[kThreads / 64];
    const int64_t batch = blockIdx.y;
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) sum += sums[batch * parts + i];
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) sum += __shfl_xor(sum, w);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = waves[0] + waves[1] + waves[2] + waves[3];
    const double by = sum == 0.0 ? 0.0 : unit / sqrt(sum);
    const int groups = (int)(ld_x / 8);
    const int64_t total = (int64_t)rows * groups;
    for (int64_t at = blockIdx.x * (int64_t)kThreads + threadIdx.x; at < total; at += gridDim.x * (int64_t)kThreads) {
        const int64_t r = at / groups;
        const int c = (int)(at - r * groups) * 8;
        const f32x8 g = load8f(grads + batch * ld_batch + r * ld + c, cols - c);
        f16x8 h, l;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = (float)((double)g[i] * by);
            h[i] = (_Float16)v;
            l[i] = low_part(v, h[i]);
        }
        const int64_t to = (batch * rows + r) * ld_x + c;
        *(f16x8 *)(x + to) = h;
        *(f16x8 *)(low + to) = l;
    }
#endif
}

struct StepArgs {
    Operands o;
    int64_t batch_a, batch_b;           // bytes from matrix to matrix
    int tiles_m, tiles_n, group;
    int cols, rows;                     // m and n of the product
    float by;                           // of the product
    float plus;                         // of `base`
    const _Float16 *base;               // [rows, ld]: added; null: nothing
    _Float16 *low;                      // [rows, ld]: what rounding left of `base`, replaced by what it leaves of `out`; null: nothing is kept
    _Float16 *out;                      // [rows, ld]
    int64_t ld;                         // elements, padded
    __bf16 *last;                       // the update itself in place of `out`: [rows, ld_last]
    int64_t ld_last, batch_last;
};

// A wavefront's part of a tile on its way to the other side: rows of n, TM elements and a gap that keeps them on different banks.
template <class S>
constexpr int kTurnRow = S::TM * 2 + 16;
template <class S>
constexpr int kTurnBytes = S::TN * kTurnRow<S>;
template <class S>
constexpr int kStepLds = S::kLds > S::WM * S::WN * kTurnBytes<S> ? S::kLds : S::WM * S::WN * kTurnBytes<S>;

// out = plus base + by (product); or the update.  SYMMETRIC: the product is, and its tiles on one side of the diagonal are formed and
// stored on both sides (4096 x 4096 over 8192: 143 us, 217 with all tiles).
template <class S, bool SYMMETRIC>
__global__ __launch_bounds__(S::kThreads) void step_tiles(const StepArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    extern __shared__ __align__(16) char lds[];
    const Tile t = SYMMETRIC ? triangle_of(blockIdx.x, A.tiles_m) : tile_of(blockIdx.x, A.tiles_m, A.tiles_n, A.group);
    const int64_t batch = blockIdx.y;
    Operands o = A.o;
    o.a += batch * A.batch_a;
    o.b += batch * A.batch_b;
    f32x4 acc[S::FM][S::FN];
    tile_product<S>(o, t, lds, acc);
    const Place<S> at(t);
    const bool whole = (A.ld_last & 7) == 0 && (A.batch_last & 7) == 0 && ((uintptr_t)A.last & 15) == 0;
    static_assert(S::FM % 2 == 0, "tiles in pairs");
    const Pair pair;
    const int wave_m = at.first_m - (threadIdx.x >> 4 & 3) * 4;
    const bool both = SYMMETRIC && t.m != t.n;
    lds_char *const turn = (lds_char *)lds + (threadIdx.x >> 6) * kTurnBytes<S>;
    typedef __attribute__((address_space(3))) f16x8 lds_f16x8;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int n = at.first_n + j * 16;
#pragma unroll
        for (int i = 0; i < S::FM; i += 2) {
            float v[8];
            paired32(acc[i][j], acc[i + 1][j], v);
            const int m = wave_m + 16 * (i + pair.tile) + pair.row;
            const bool there = n < A.rows && m < A.ld;
            const int64_t here = (batch * A.rows + n) * A.ld + m;
            f16x8 base = {}, low = {};
            if (A.base && there) base = *(const f16x8 *)(A.base + here);
            if (A.low && there) low = *(const f16x8 *)(A.low + here);
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = v[r] * A.by + A.plus * fmaf((float)low[r], 1.f / kLowUnit, (float)base[r]);
            if (A.last) {
                __bf16 *to = A.last + batch * A.batch_last + (int64_t)n * A.ld_last + m;
                if (!there) {
                } else if (whole && m + 8 <= A.cols) {
                    bf16x8 t;
#pragma unroll
                    for (int r = 0; r < 8; ++r) t[r] = (__bf16)v[r];
                    *(bf16x8 *)to = t;
                } else {
                    for (int r = 0; r < 8; ++r)
                        if (m + r < A.cols) to[r] = (__bf16)v[r];
                }
            } else {
                f16x8 t;
#pragma unroll
                for (int r = 0; r < 8; ++r) t[r] = (_Float16)(there && m + r < A.cols ? v[r] : 0.f);
                if (there) *(f16x8 *)(A.out + here) = t;
                if (A.low && there) {
#pragma unroll
                    for (int r = 0; r < 8; ++r) low[r] = m + r < A.cols ? low_part(v[r], t[r]) : (_Float16)0.f;
                    *(f16x8 *)(A.low + here) = low;
                }
                if (both) *(lds_f16x8 *)(turn + (j * 16 + (threadIdx.x & 15)) * kTurnRow<S> + (16 * (i + pair.tile) + pair.row) * 2) = t;
            }
        }
    }
    if (!both) return;
    // The wavefront's part turned, sixteen rows m of eight n at a time by sixteen lanes: C[m, n .. n + 7].
    asm volatile("" ::: "memory");         // (a wavefront's own accesses to LDS keep their order)
    __builtin_amdgcn_wave_barrier();
    constexpr int kAcross = S::TN / 8, kUnits = S::TM / 16 * kAcross;
    const int wave = threadIdx.x >> 6, r = threadIdx.x & 15;
    static_assert(kUnits % 4 == 0, "four at a time");
    for (int u = threadIdx.x >> 4 & 3; u < kUnits; u += 4) {
        const int m = u / kAcross * 16, n = u % kAcross * 8;
        const lds_char *from = turn + (n + (r >> 2)) * kTurnRow<S> + (m + (r & 3) * 4) * 2;
        const s16x4 low = read_turned((lds_s16x4 *)from), high = read_turned((lds_s16x4 *)(from + 4 * kTurnRow<S>));
        const int row = t.m * S::BM + wave / S::WN * S::TM + m + r, col = t.n * S::BN + wave % S::WN * S::TN + n;
        if (row < A.rows && col < A.ld)
            *(s16x8 *)(A.out + (batch * A.rows + row) * A.ld + col) = (s16x8)__builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
    }
#endif
}

template <bool SYMMETRIC, class S>
void launch_step(StepArgs a, int batch, hipStream_t stream)
{
    a.tiles_m = (a.cols + S::BM - 1) / S::BM;
    a.tiles_n = (a.rows + S::BN - 1) / S::BN;
    a.group = 8;
    const int tiles = SYMMETRIC ? a.tiles_m * (a.tiles_m + 1) / 2 : a.tiles_m * a.tiles_n;
    hipLaunchKernelGGL((step_tiles<S, SYMMETRIC>), dim3((unsigned)tiles, (unsigned)batch), dim3(S::kThreads), SYMMETRIC ? kStepLds<S> : S::kLds, stream, a);
}
template <bool SYMMETRIC, bool COLS_A, bool COLS_B>
void launch_step(int shape, const StepArgs &a, int batch, hipStream_t stream)
{
    switch (shape) {
        case 0: launch_step<SYMMETRIC, Shape0<F16, COLS_A, COLS_B>>(a, batch, stream); break;
        case 1: launch_step<SYMMETRIC, Shape1<F16, COLS_A, COLS_B>>(a, batch, stream); break;
        case 2: launch_step<SYMMETRIC, Shape2<F16, COLS_A, COLS_B>>(a, batch, stream); break;
        case 3:                             // (not square)
            if constexpr (!SYMMETRIC) launch_step<SYMMETRIC, Shape3<F16, COLS_A, COLS_B>>(a, batch, stream);
            break;
        case 4: launch_step<SYMMETRIC, Shape4<F16, COLS_A, COLS_B>>(a, batch, stream); break;
        default: launch_step<SYMMETRIC, Shape5<F16, COLS_A, COLS_B>>(a, batch, stream); break;
    }
}

template <bool COLS_A, bool COLS_B>
void launch_step(StepShape shape, const StepArgs &a, int batch, hipStream_t stream)
{
    if (shape.half) launch_step<true, COLS_A, COLS_B>(shape.shape, a, batch, stream);
    else launch_step<false, COLS_A, COLS_B>(shape.shape, a, batch, stream);
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
    _Float16 *x[2] = {(_Float16 *)(ws + p.x[0]), (_Float16 *)(ws + p.x[1])}, *gram = (_Float16 *)(ws + p.gram), *poly = (_Float16 *)(ws + p.poly), *low = (_Float16 *)(ws + p.low);
    const unsigned blocks = (unsigned)std::min<int64_t>(std::max<int64_t>(2048 / d.batch, 16), ((int64_t)d.rows * (p.x_pad / 8) + kThreads - 1) / kThreads);
    hipLaunchKernelGGL(normalise<E>, dim3(blocks, (unsigned)d.batch), dim3(kThreads), 0, stream, grads, d.rows, d.cols, d.grads_stride, d.grads_batch_stride, (const double *)norms,
                       p.norm_blocks, p.unit, x[0], low, p.x_pad);
    const int64_t ld_x = p.x_pad * 2, ld_m = p.m_pad * 2, batch_x = d.rows * ld_x, batch_m = p.m * ld_m;      // bytes
    for (int s = 0; s < d.steps; ++s) {
        const char *from = (const char *)x[s & 1];
        StepArgs a = {};
        // gram = X X'
        a.o = {from, from, ld_x, ld_x, p.m, p.m, p.n};
        a.batch_a = a.batch_b = batch_x;
        a.cols = a.rows = p.m;
        a.by = (float)(1.0 / (p.unit * p.unit));
        a.out = gram;
        a.ld = p.m_pad;
        if (p.tall) launch_step<true, true>(p.shape_gram, a, d.batch, stream);
        else launch_step<false, false>(p.shape_gram, a, d.batch, stream);
        // poly = b gram + c gram gram
        a.o = {(const char *)gram, (const char *)gram, ld_m, ld_m, p.m, p.m, p.m};
        a.batch_a = a.batch_b = batch_m;
        a.by = (float)d.c;
        a.plus = (float)d.b;
        a.base = gram;
        a.out = poly;
        launch_step<false, false>(p.shape_square, a, d.batch, stream);
        // X = a X + poly X (tall: + X poly); the last one as the update
        a.by = 1.f;
        a.plus = (float)d.a;
        a.base = x[s & 1];
        a.low = low;
        a.out = x[(s + 1) & 1];
        a.ld = p.x_pad;
        a.cols = d.cols;
        a.rows = d.rows;
        if (s + 1 == d.steps) {
            a.by /= (float)p.unit;
            a.plus /= (float)p.unit;
            a.last = update;
            a.ld_last = d.update_stride;
            a.batch_last = d.update_batch_stride;
        }
        if (p.tall) {
            a.o = {(const char *)poly, from, ld_m, ld_x, d.cols, d.rows, p.m};
            a.batch_a = batch_m;
            a.batch_b = batch_x;
            launch_step<false, false, false>(p.shape_wide.shape, a, d.batch, stream);
        } else {
            a.o = {from, (const char *)poly, ld_x, ld_m, d.cols, d.rows, p.m};
            a.batch_a = batch_x;
            a.batch_b = batch_m;
            launch_step<false, true, false>(p.shape_wide.shape, a, d.batch, stream);
        }
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
    p.x_pad = (d.cols + 7) / 8 * 8;
    p.unit = ldexp(1.0, (int)lround(0.5 * log2((double)p.n)));
    p.norm_blocks = (int)std::max<int64_t>(1, std::min<int64_t>(2048 / std::max(d.batch, 1), (int64_t)d.rows * d.cols / 8192));
    p.shape_gram = step_shape_for(p.m, p.m, p.n, d.batch, true);
    p.shape_square = step_shape_for(p.m, p.m, p.m, d.batch, true);
    p.shape_wide = step_shape_for(d.cols, d.rows, p.m, d.batch, false);
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o = up256(o + bytes); return at; };
    p.norms = take(std::max<size_t>(8, 8 * (size_t)d.batch * p.norm_blocks));
    if (d.steps > 0) {
        for (int i = 0; i < (d.steps > 1 ? 2 : 1); ++i) p.x[i] = take(2 * (size_t)d.batch * d.rows * p.x_pad);
        p.low = take(2 * (size_t)d.batch * d.rows * p.x_pad);
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
