// The gradient of a layer's weights from its input kept in 8 bits:
//
//   dW[m,k] = w[k] sum_n dY[n,m] X[n,k] + b[k] sum_n dY[n,m]
//
// A product over the rows n, of which both operands are columns in memory: tiles of dW, k in registers (a lane's four values are neighbours of a row of dW).  X is turned into dY's type on its way to
// LDS and is nowhere in memory in more than 8 bits.  Scales differ from row to row, which is what the product sums over, so that they cannot wait until after it;
// a norm's weights w can, and are multiplied in where tiles are stored.  Few tiles: the rows are cut in slices, whose sums are joined in order.
// Bound by the matrix units, and by the power that they and the codes' turning take together: 16384 x 4096 x 16384 in bfloat16, in turn on one card three times from cold on, from i8
// 1.14, 1.21 and 1.23 PFLOP/s, from e4m3 1.18 to 1.19 (a code of i8 takes two and a half operations, one of e4m3 half a one), a library product of 16 bits 1.09, 1.18 and 1.19.

#include "pollux_host.h"
#include "pollux_kept.h"
#include "pollux_rows.h"
#include "pollux_tiles.h"
#include "pollux_train.h"

#include <math.h>

#include <algorithm>

namespace px {
namespace {

constexpr int kThreads = 256;

struct KeptGradArgs {
    Operands o;
    int tiles_m, tiles_n;
    int64_t N, slice;
    int D, M;
    const void *weight, *bias;
    int weight_type;
    const float *sums;          // [M] of rows_grad over the rows, with a bias
    void *out;                  // weight_grad, or the slices' sums
    int64_t ld;
    int slices;
    bool add;
};

#ifdef __HIP_DEVICE_COMPILE__
__device__ __forceinline__ float parameter(const void *p, int type, int at, float none)
{
    if (!p) return none;
    return type == PX_TYPE_F32 ? ((const float *)p)[at] : type == PX_TYPE_BF16 ? (float)((const __bf16 *)p)[at] : (float)((const _Float16 *)p)[at];
}
#endif

template <class S>
__global__ __launch_bounds__(S::kThreads) void kept_tiles(const KeptGradArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    typedef typename S::element::type type;
    extern __shared__ __align__(16) char lds[];
    const Tile t = tile_of(blockIdx.x, A.tiles_m, A.tiles_n, 8);
    Operands o = A.o;
    const int64_t row = blockIdx.y * A.slice;
    o.a += row * o.lda;
    o.scales += row * (o.lda / kKeptGroup);
    o.b += row * o.ldb;
    o.k = __builtin_amdgcn_readfirstlane((int)max((int64_t)0, min(A.slice, A.N - row)));
    f32x4 acc[S::FM][S::FN];
    tile_product<S>(o, t, lds, acc);
    const Place<S> at(t);
    constexpr bool kPairs = sizeof(type) == 2 && S::FM % 2 == 0;
    const Pair pair;
    const int wave_m = at.first_m - (threadIdx.x >> 4 & 3) * 4;
    const bool sums = A.slices > 1;
    const int group = sums || !kPairs ? 3 : 7;
    const bool whole = sums ? (A.D & 3) == 0 : (A.ld & group) == 0;
    if (!sums && (A.weight || A.bias)) {
        // (a lane's columns are its rows' all alike)
        float rows[S::FN];
#pragma unroll
        for (int j = 0; j < S::FN; ++j) rows[j] = A.bias && at.first_n + j * 16 < A.M ? A.sums[at.first_n + j * 16] : 0.f;
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int m = min(at.first_m + 16 * i + r, A.D - 1);
                const float w = parameter(A.weight, A.weight_type, m, 1.f), b = parameter(A.bias, A.weight_type, m, 0.f);
#pragma unroll
                for (int j = 0; j < S::FN; ++j) acc[i][j][r] = A.bias ? fmaf(rows[j], b, acc[i][j][r] * w) : acc[i][j][r] * w;
            }
    }
    const bool plain = whole && !sums && !A.add && (t.m + 1) * S::BM <= A.D;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int n = at.first_n + j * 16;
        if (sums) {
            if (n >= A.M) continue;
            float *const to = (float *)A.out + ((int64_t)blockIdx.y * A.M + n) * A.D;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int m = at.first_m + 16 * i;
                const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                put<F32>(to + m, v, A.D - m, whole, false);
            }
            continue;
        }
        type *const to = (type *)A.out + (int64_t)n * A.ld;
        if constexpr (kPairs) {
#pragma unroll
            for (int i = 0; i < S::FM; i += 2) {
                const int m = wave_m + 16 * (i + pair.tile) + pair.row;
                // (lanes change places, those past the last row too)
                if (plain) {
                    const auto both = paired<typename S::element>(acc[i][j], acc[i + 1][j]);
                    if (n < A.M) *(typename S::element::piece *)(to + m) = both;
                } else {
                    float both[8];
                    paired32(acc[i][j], acc[i + 1][j], both);
                    if constexpr (S::BM < 256) {
                        // (at any alignment: 300 x 4100 x 4200 34 us where single elements take 62; tiles of 256 have no registers left for it)
                        f32x8 v = {both[0], both[1], both[2], both[3], both[4], both[5], both[6], both[7]};
                        if (n < A.M && m < A.D) {
                            if (A.add) v += load8f(to + m, A.D - m);
                            store8f(to + m, A.D - m, v);
                        }
                    } else if (n < A.M) {
                        put<typename S::element>(to + m, both, A.D - m, whole, A.add);
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int m = at.first_m + 16 * i;
                const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                if (n < A.M) put<typename S::element>(to + m, v, A.D - m, whole, A.add);
            }
        }
    }
#endif
}

// The slices' sums, added in their order, weighted and rounded.
template <class T>
__global__ __launch_bounds__(kThreads) void join_slices(const KeptGradArgs A, const float *slices)
{
#ifdef __HIP_DEVICE_COMPILE__
    typedef typename T::type type;
    const int groups = (A.D + kVec - 1) / kVec;
    const int64_t total = (int64_t)A.M * groups, one = (int64_t)A.M * A.D;
    for (int64_t at = blockIdx.x * (int64_t)kThreads + threadIdx.x; at < total; at += gridDim.x * (int64_t)kThreads) {
        const int64_t n = at / groups;
        const int c = (int)(at - n * groups) * kVec, left = A.D - c;
        const float *from = slices + n * A.D + c;
        f32x8 v = load8f(from, left);
#pragma unroll 4
        for (int s = 1; s < A.slices; ++s) v += load8f(from + s * one, left);
        if (A.weight || A.bias) {
            const float rows = A.bias ? A.sums[n] : 0.f;
            v *= parameters(A.weight, A.weight_type, c, left, 1.f);
            if (A.bias) {
                const f32x8 b = parameters(A.bias, A.weight_type, c, left, 0.f);
#pragma unroll
                for (int i = 0; i < kVec; ++i) v[i] = fmaf(rows, b[i], v[i]);
            }
        }
        type *const to = (type *)A.out + n * A.ld + c;
        if (A.add) v += load8f(to, left);
        store8f(to, left, v);
    }
#endif
}

// Sums of rows_grad over the rows: of a part of them, eight columns a thread, by `down` threads that each take every down-th row; then of the parts in order.  to: the rows are copied there
// on the way, padded with zeros to ld_to.
template <class E, bool SUMS>
__global__ __launch_bounds__(kThreads) void sum_rows(const E *rows, int64_t ld, int64_t N, int M, int across, float *parts, E *to, int64_t ld_to)
{
#ifdef __HIP_DEVICE_COMPILE__
    __shared__ float shared[SUMS ? kThreads : 1][kVec + 1];
    const int down = kThreads / across, mine = threadIdx.x % across, from = threadIdx.x / across;
    const int c = (blockIdx.x * across + mine) * kVec, left = M - c;
    const int64_t each = (N + gridDim.y - 1) / gridDim.y, first = blockIdx.y * each, last = min(first + each, N);
    f32x8 v = {};
#pragma unroll 4
    for (int64_t n = first + from; n < last; n += down) {
        const auto row = load8(rows + n * ld + c, left);
        if (to) store8(to + n * ld_to + c, ld_to - c, row);
        if (SUMS) v += __builtin_convertvector(row, f32x8);
    }
    if (!SUMS) return;
#pragma unroll
    for (int i = 0; i < kVec; ++i) shared[threadIdx.x][i] = v[i];
    __syncthreads();
    if (from != 0) return;
    for (int k = 1; k < down; ++k)
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] += shared[k * across + mine][i];
    store8f(parts + (int64_t)blockIdx.y * M + c, left, v);
#endif
}
__global__ __launch_bounds__(kThreads) void sum_parts(const float *parts, int count, int M, float *sums)
{
    const int m = blockIdx.x * kThreads + threadIdx.x;
    if (m >= M) return;
    float v = 0.f;
#pragma unroll 16
    for (int k = 0; k < count; ++k) v += parts[(int64_t)k * M + m];
    sums[m] = v;
}

unsigned blocks_for(int64_t groups) { return (unsigned)std::min<int64_t>((groups + kThreads - 1) / kThreads, 8192); }

template <class T, int FORM>
void launch_tiles(int shape, KeptGradArgs a, hipStream_t stream)
{
    auto launch = [&](auto s) {
        typedef decltype(s) S;
        a.tiles_m = (a.D + S::BM - 1) / S::BM;
        a.tiles_n = (a.M + S::BN - 1) / S::BN;
        hipLaunchKernelGGL(kept_tiles<S>, dim3((unsigned)(a.tiles_m * a.tiles_n), (unsigned)a.slices), dim3(S::kThreads), S::kLds, stream, a);
    };
    switch (shape) {
        case 0:
            if constexpr (!std::is_same<T, F32>::value) launch(TileShape<T, 256, 256, 2, 4, 2, true, true, FORM>());
            break;
        case 1: launch(TileShape<T, 128, 128, 2, 2, 2, true, true, FORM>()); break;
        default: launch(TileShape<T, 64, 64, 2, 2, 2, true, true, FORM>()); break;
    }
}

template <class T>
int kept_grad(const pollux_kept_grad_dims &d, const KeptGradPlan &p, const uint8_t *values, const uint8_t *scales, const char *rows_grad, const void *weight,
              const void *bias, char *ws, void *weight_grad, hipStream_t stream)
{
    typedef typename T::type type;
    constexpr int e = sizeof(type);
    KeptGradArgs a = {};
    a.N = d.N;
    a.D = d.D;
    a.M = d.M;
    a.weight = weight;
    a.bias = bias;
    a.weight_type = d.weight_type;
    a.sums = (const float *)(ws + p.sums);
    a.add = d.flags & PX_FLAG_ACCUMULATE;
    a.slice = p.slice;
    a.slices = p.slices;
    a.ld = d.weight_grad_stride;
    int64_t ld = d.rows_grad_stride;
    if (bias || (p.pack && d.N > 0)) {
        // (32 threads across: 512 bytes a row, and eight rows under way a workgroup)
        int across = 1;
        while (across < 32 && across * kVec < d.M) across *= 2;
        const dim3 grid((unsigned)((d.M + across * kVec - 1) / (across * kVec)), (unsigned)p.sum_blocks);
        type *const to = p.pack ? (type *)(ws + p.rows) : nullptr;
        auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, (const type *)rows_grad, ld, d.N, d.M, across, (float *)(ws + p.parts), to, p.m_pad); };
        bias ? launch(sum_rows<type, true>) : launch(sum_rows<type, false>);
        if (bias) hipLaunchKernelGGL(sum_parts, dim3((unsigned)((d.M + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, (const float *)(ws + p.parts), p.sum_blocks, d.M, (float *)(ws + p.sums));
        if (to) {
            rows_grad = ws + p.rows;
            ld = p.m_pad;
        }
    }
    const int64_t width = kept_width(d.D);
    a.o = {(const char *)values, rows_grad, width, ld * e, d.D, d.M, 0, scales};
    a.out = p.slices > 1 ? (void *)(ws + p.slices_at) : weight_grad;
    if (d.form == PX_KEPT_I8) launch_tiles<T, PX_KEPT_I8>(p.tiles, a, stream);
    else launch_tiles<T, PX_KEPT_E4M3>(p.tiles, a, stream);
    if (p.slices > 1) {
        a.out = weight_grad;
        hipLaunchKernelGGL(join_slices<T>, dim3(blocks_for((int64_t)d.M * ((d.D + kVec - 1) / kVec))), dim3(kThreads), 0, stream, a, (const float *)(ws + p.slices_at));
    }
    return status_of(hipGetLastError());
}

}  // namespace

// What shapes of tile take (pollux_tiles.h) where one operand's codes are turned on their way to LDS: i8 in 16-bit products of 300 to 65536 rows x 128 to 4096 x 128 to 4096 and in fp32, within some 15 %:
// 8192 x 2048 x 2048 in one slice 220, 130, 158 us, in four 88, 117, 162; 65536 x 128 x 128 in 32 slices 67, 43, 33; fp32 4096 x 2048 x 4096 253 and 557.
constexpr ShapeOf kKeptShape[3] = {{256, 256, 1, 1.64, 1.64, 0.00, 0.00, 8.7}, {128, 128, 2, 0.93, 1.38, 1.27, 1.93, 6.0}, {64, 64, 4, 0.62, 1.20, 0.75, 2.14, 4.5}};

KeptGradPlan kept_grad_plan(const pollux_kept_grad_dims &d)
{
    KeptGradPlan p = {};
    const int e = size_of_type(d.type), pad = 16 / e, depth = kRowBytes / e;
    const bool f32 = e == 4;
    p.m_pad = ((int64_t)d.M + pad - 1) / pad * pad;
    p.pack = d.rows_grad_stride % pad != 0 || d.M % pad != 0;
    const int64_t stages = std::max<int64_t>(1, (d.N + depth - 1) / depth);
    // in as many slices of the rows as takes least, their sums being written and read at some 8 TB/s each, out of the caches
    double least = 1e300;
    for (int slices = 1; slices <= 128; slices += slices < 8 ? 1 : slices / 4) {
        if (slices > 1 && (stages < 4 * slices || (int64_t)slices * d.M * d.D * 4 > (512ll << 20))) break;
        for (int s = f32 ? 1 : 0; s < 3; ++s) {
            double cost = shape_cost(kKeptShape[s], d.D, d.M, (double)d.N / slices, slices, f32);
            if (slices > 1) cost += 4.0 + 4.0 * slices * d.M * d.D / 4.2e6;
            // (tiles of 256 store rows that begin anywhere an element at a time)
            else if (s == 0 && d.weight_grad_stride % 8 != 0) cost += 25.0 * ceil(ceil(d.D / 256.0) * ceil(d.M / 256.0) / 256);
            if (cost < least) least = cost, p.slices = slices, p.tiles = s;
        }
    }
    p.slice = (stages + p.slices - 1) / p.slices * depth;
    p.sum_blocks = (int)std::max<int64_t>(1, std::min<int64_t>(64, d.N / 32));
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o = up256(o + bytes); return at; };
    p.parts = take((size_t)p.sum_blocks * d.M * 4);
    p.sums = take((size_t)d.M * 4);
    if (p.pack) p.rows = take((size_t)d.N * p.m_pad * e);
    if (p.slices > 1) p.slices_at = take((size_t)p.slices * d.M * d.D * 4);
    p.total = o;
    return p;
}

int launch_kept_grad(const pollux_kept_grad_dims &d, const KeptGradPlan &p, const uint8_t *values, const uint8_t *scales, const void *rows_grad, const void *weight,
                     const void *bias, void *workspace, void *weight_grad, hipStream_t stream)
{
    const char *rows = (const char *)rows_grad;
    char *ws = (char *)workspace;
    switch (d.type) {
        case PX_TYPE_F32: return kept_grad<F32>(d, p, values, scales, rows, weight, bias, ws, weight_grad, stream);
        case PX_TYPE_BF16: return kept_grad<Bf16>(d, p, values, scales, rows, weight, bias, ws, weight_grad, stream);
        default: return kept_grad<F16>(d, p, values, scales, rows, weight, bias, ws, weight_grad, stream);
    }
}

}  // namespace px
