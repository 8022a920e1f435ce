// Cross entropy of tokens over a large vocabulary, from hidden rows and the projection's weights, and its gradients, in pieces
// of the vocabulary: the logits of all tokens over all entries are never in memory.
//
//   l[n,v] = <h_n, w_v>     lse_n = max_v l + log sum_v exp(l - max)     loss_n = lse_n - l[n, y_n]
//   q[n,v] = g_n (exp(l[n,v] - lse_n) - [v = y_n])      dH = q W      dW = q' H
//
// Forward: a tile of logits is reduced, as it leaves the matrix units, to each token's largest logit and sum of exponentials
// over the tile's entries (loss_tiles); a second launch joins a token's tiles (loss_join).
// Backward: for each piece of the vocabulary the logits are formed again, q of the piece is written once (q_tiles), and both
// gradients are products with it (grad_tiles): of the hidden rows' the weights lie as columns, of the weights' both operands.  The hidden rows'
// gradient is summed over pieces in fp32 (and over slices of a piece where few tiles would leave the chip idle), in a
// fixed order, and rounded once (join_slices).
//
// q is rounded to the type of the inputs because the matrix units take it so: half a step of that type per element.  A token's
// largest q by far is its target's, as large as all others together: what its rounding leaves is kept in fp32 (`rest`) and multiplied with the target's weights
// where the hidden rows' gradient is rounded, which brings that gradient's error from 1.35 times that of its own rounding to what the rounding leaves.
// fp16 has too few exponents for q (a mean over 10^4 tokens of probabilities of 10^-6): there q is
// scaled by the power of two that brings the largest row weight to 2^13, and the gradients are scaled back in fp32.

#include "pollux_host.h"
#include "pollux_rows.h"
#include "pollux_tiles.h"
#include "pollux_train.h"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace px {
namespace {

#ifdef __HIP_DEVICE_COMPILE__
__device__ __forceinline__ int target_of(const void *targets, int64_t n, bool i64, int V)
{
    bool bad;
    return token_at(targets, n, i64, V, bad);
}
#endif

constexpr float kLog2e = 1.44269504088896340736f;

// A maximum to subtract: 0 stands in for one that is infinite, so that inf - inf is never formed.
__device__ __forceinline__ float finite_or_zero(float m) { return fabsf(m) < __builtin_inff() ? m : 0.f; }

// (largest logit, sum of exponentials from it) of two sets as that of both.  The sum from a maximum of -inf is 0, or NaN.
__device__ __forceinline__ float2 joined(float2 a, float2 b)
{
    const float top = fmaxf(a.x, b.x), from = finite_or_zero(top);
    auto part = [&](float2 p) {
        return p.y == __builtin_inff() || p.x == -__builtin_inff() ? p.y : p.y * __builtin_amdgcn_exp2f((finite_or_zero(p.x) - from) * kLog2e);
    };
    return make_float2(top, part(a) + part(b));
}

struct LogitArgs {
    Operands o;                 // a: weights of the piece, b: hidden rows
    int first, V, N;            // the piece's first vocabulary entry
    int tiles_m, tiles_n, group;
    const void *targets;
    bool i64;
    // forward
    float2 *parts;              // of the piece's first tile
    float *picked;
    int32_t *status;            // of the first piece, else null: forward, the first workgroup clears it; backward, the first tiles report
    // backward
    const float *lse, *row_weight, *scale;
    void *q;
    float *rest;                // [N]: the target's q less what it was rounded to; null (fp32): nothing is lost
    int64_t ld_q;               // elements
    int rows;                   // entries of the piece
};

// One tile of logits -> per token (largest logit, sum of exponentials from it) over the tile's entries, and the target's logit
// where the tile holds it.  A lane has one token and 4 FM entries of it; four lanes share a token in a wavefront, WM wavefronts
// in the workgroup.
template <class S>
__global__ __launch_bounds__(S::kThreads) void loss_tiles(const LogitArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    extern __shared__ __align__(16) char lds[];
    const Tile t = tile_of(blockIdx.x, A.tiles_m, A.tiles_n, A.group);
    if (A.status && blockIdx.x == 0 && threadIdx.x < kStatusWords) A.status[threadIdx.x] = 0;
    f32x4 acc[S::FM][S::FN];
    tile_product<S>(A.o, t, lds, acc);
    const Place<S> at(t);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, left = A.o.m;
    const bool edge = (t.m + 1) * S::BM > left;
    float2 *const shared = (float2 *)lds;        // [WM][BN]
    __syncthreads();
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int n = at.first_n + j * 16;
        const int y = n < A.N ? target_of(A.targets, n, A.i64, A.V) - A.first : -1;
        float top = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < S::FM; ++i) {
            const int v = at.first_m + 16 * i;
            if (edge)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (v + r >= left) acc[i][j][r] = -__builtin_inff();
            if (y >= v && y < min(v + 4, left)) A.picked[n] = y == v ? acc[i][j][0] : y == v + 1 ? acc[i][j][1] : y == v + 2 ? acc[i][j][2] : acc[i][j][3];
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, acc[i][j][r]);
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float from = finite_or_zero(top);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f((acc[i][j][r] - from) * kLog2e);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16) shared[wave / S::WN * S::BN + wave % S::WN * S::TN + j * 16 + lane] = make_float2(top, sum);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < S::BN; c += S::kThreads) {
        const int n = t.n * S::BN + c;
        if (n >= A.N) break;
        float2 all = shared[c];
#pragma unroll
        for (int w = 1; w < S::WM; ++w) all = joined(all, shared[w * S::BN + c]);
        A.parts[(int64_t)t.m * A.N + n] = all;
    }
#endif
}

// Each token's tiles joined: TOKENS neighbouring tokens (a line of a tile's values) by 256 / TOKENS parts of the list.
constexpr int kJoinThreads = 256;
template <int TOKENS>
__global__ __launch_bounds__(kJoinThreads) void loss_join(const float2 *parts, int tiles, int N, const float *picked, const void *targets, bool i64, int V, float *loss,
                                                          float *lse, int32_t *status)
{
    constexpr int kParts = kJoinThreads / TOKENS, kAhead = 4;
    __shared__ float2 shared[kJoinThreads / 64][TOKENS];
    const int c = threadIdx.x % TOKENS, k = threadIdx.x / TOKENS, n = blockIdx.x * TOKENS + c;
    const float2 none = make_float2(-__builtin_inff(), 0.f);
    float2 all = none;
    if (n < N)
        for (int t0 = k; t0 < tiles; t0 += kParts * kAhead) {
            float2 p[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) p[i] = t0 + i * kParts < tiles ? parts[(int64_t)(t0 + i * kParts) * N + n] : none;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) all = joined(all, p[i]);
        }
#pragma unroll
    for (int w = TOKENS; w < 64; w <<= 1) all = joined(all, make_float2(__shfl_xor(all.x, w), __shfl_xor(all.y, w)));
    if ((threadIdx.x & 63) < TOKENS) shared[threadIdx.x >> 6][c] = all;
    __syncthreads();
    if (threadIdx.x >= TOKENS || n >= N) return;
#pragma unroll
    for (int i = 1; i < kJoinThreads / 64; ++i) all = joined(all, shared[i][c]);
    const float from = finite_or_zero(all.x), sum = all.y;
    const float whole = from + logf(sum);
    lse[n] = whole;
    bool bad;
    const int y = token_at(targets, n, i64, V, bad);
    loss[n] = y < 0 ? 0.f : whole - picked[n];
    if (bad) atomicOr(status, PX_ST_BAD_TOKEN);
}

// ---- backward ------------------------------------------------------------------------------------------------------

// Clears the status word where nothing else is launched.
__global__ void clear_status(int32_t *status)
{
    if (threadIdx.x < kStatusWords) status[threadIdx.x] = 0;
}

#ifdef __HIP_DEVICE_COMPILE__
// For fp16, by one workgroup of 256: the power of two that q is scaled by: scale[0] that, scale[1] its inverse.
__device__ __forceinline__ void find_scale(const void *targets, bool i64, int V, int64_t N, const float *row_weight, float *scale)
{
    __shared__ float tops[4];
    float top = 0.f;
#pragma unroll 8
    for (int64_t n = threadIdx.x; n < N; n += 256) {
        const float g = target_of(targets, n, i64, V) < 0 ? 0.f : row_weight ? fabsf(row_weight[n]) : 1.f;
        if (g < __builtin_inff()) top = fmaxf(top, g);
    }
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) top = fmaxf(top, __shfl_xor(top, w));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int i = 0; i < 4; ++i) top = fmaxf(top, tops[i]);
    const int e = top > 0.f ? min(100, max(-100, 13 - ilogbf(top))) : 0;
    scale[0] = ldexpf(1.f, e);
    scale[1] = ldexpf(1.f, -e);
}
#endif

// One tile of q from the logits' tile.  A token without a target, or of weight 0, has a row of zeros,
// whatever its logits are.
template <class S>
__global__ __launch_bounds__(S::kThreads) void q_tiles(const LogitArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    typedef typename S::element::type type;
    extern __shared__ __align__(16) char lds[];
    const Tile t = tile_of(blockIdx.x, A.tiles_m, A.tiles_n, A.group);
    f32x4 acc[S::FM][S::FN];
    tile_product<S>(A.o, t, lds, acc);
    const Place<S> at(t);
    const float scale = A.scale ? A.scale[0] : 1.f;
    const bool edge = (t.m + 1) * S::BM > A.rows;
    const Pair pair;
    const int wave_m = at.first_m - (threadIdx.x >> 4 & 3) * 4;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int n = at.first_n + j * 16;
        bool bad = false;
        const int y = n < A.N ? token_at(A.targets, n, A.i64, A.V, bad) : -1;
        if (bad && A.status && t.m == 0) atomicOr(A.status, PX_ST_BAD_TOKEN);
        const float g = y < 0 ? 0.f : (A.row_weight ? A.row_weight[n] : 1.f) * scale;
        const float lse = g == 0.f ? 0.f : A.lse[n];
        const int hit = y - A.first;
        auto value = [&](int i) {
            const int v = at.first_m + 16 * i;
            f32x4 q;
#pragma unroll
            for (int r = 0; r < 4; ++r) q[r] = __builtin_amdgcn_exp2f((acc[i][j][r] - lse) * kLog2e) * g;
            if (hit >= v && hit < v + 4)
#pragma unroll
                for (int r = 0; r < 4; ++r) q[r] -= v + r == hit ? g : 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) q[r] = g != 0.f && (!edge || v + r < A.rows) ? q[r] : 0.f;
            if constexpr (sizeof(type) == 2)
                if (hit >= v && hit < v + 4) {
                    const float whole = hit == v ? q[0] : hit == v + 1 ? q[1] : hit == v + 2 ? q[2] : q[3], lost = whole - (float)(type)whole;
                    A.rest[n] = fabsf(lost) < __builtin_inff() ? lost : 0.f;
                }
            return q;
        };
        type *const row = (type *)A.q + (int64_t)n * A.ld_q;
        if constexpr (sizeof(type) == 2 && S::FM % 2 == 0) {
#pragma unroll
            for (int i = 0; i < S::FM; i += 2) {
                const auto both = paired<typename S::element>(value(i), value(i + 1));
                const int v = wave_m + 16 * (i + pair.tile) + pair.row;
                if (n < A.N && v < A.ld_q) *(typename S::element::piece *)(row + v) = both;
            }
        } else {
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int v = at.first_m + 16 * i;
                if (n < A.N && v < A.ld_q) store4<typename S::element>(row + v, value(i));
            }
        }
    }
#endif
}

struct GradArgs {
    Operands o;
    int tiles_m, tiles_n, group;
    int slice_k;                // k that a slice (blockIdx.y) takes
    int cols, rows;             // m and n
    void *out;                  // [rows, ld]: the gradient, or fp32 sums [slices, rows, cols]
    int64_t ld;                 // elements
    int sums;                   // 0: the gradient itself; 1: sums begin; 2: sums go on
    bool add;                   // what `out` holds is added to
    const float *scale;
    const void *targets;        // rows without a target, or of weight 0, are zeros; null: no such rows
    const float *row_weight;
    bool i64;
    int V;
    const float *rest;          // [N], and the weights it multiplies (elements from row to row); null: nothing
    const void *weight;
    int64_t ld_weight;
};

#ifdef __HIP_DEVICE_COMPILE__
// v += rest * the target's weights, of which `left` remain in the row.  (An infinite weight has made its logit, and the row, what it is already.)
template <class E, class V>
__device__ __forceinline__ void add_rest(V &v, float rest, const E *weight, int64_t left)
{
    const f32x8 w = load8f(weight, left);
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const float more = rest * w[r];
        v[r] += fabsf(more) < __builtin_inff() ? more : 0.f;
    }
}
#endif

template <class S>
__global__ __launch_bounds__(S::kThreads) void grad_tiles(const GradArgs A)
{
#ifdef __HIP_DEVICE_COMPILE__
    typedef typename S::element::type type;
    extern __shared__ __align__(16) char lds[];
    const Tile t = tile_of(blockIdx.x, A.tiles_m, A.tiles_n, A.group);
    Operands o = A.o;
    const int k0 = blockIdx.y * A.slice_k;
    o.a += S::COLS_A ? k0 * o.lda : k0 * (int64_t)sizeof(type);
    o.b += S::COLS_B ? k0 * o.ldb : k0 * (int64_t)sizeof(type);
    o.k = max(0, min(A.slice_k, A.o.k - k0));
    f32x4 acc[S::FM][S::FN];
    tile_product<S>(o, t, lds, acc);
    const Place<S> at(t);
    const float scale = A.scale ? A.scale[1] : 1.f;
    constexpr bool kPairs = sizeof(type) == 2 && S::FM % 2 == 0;
    const Pair pair;
    const int wave_m = at.first_m - (threadIdx.x >> 4 & 3) * 4;
    const int group = A.sums || !kPairs ? 3 : 7;
    const bool whole = A.sums ? (A.cols & group) == 0 : (A.ld & group) == 0 && ((uintptr_t)A.out & 15) == 0;
    const bool plain = whole && !A.add && !A.rest && (t.m + 1) * S::BM <= A.cols;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int n = at.first_n + j * 16;
        if (n >= A.rows) continue;
        bool none = false;
        int y = -1;
        if (A.targets && !A.sums) {
            y = target_of(A.targets, n, A.i64, A.V);
            none = y < 0 || (A.row_weight && A.row_weight[n] == 0.f);
        }
        if (A.sums) {
            float *const row = (float *)A.out + ((int64_t)blockIdx.y * A.rows + n) * A.cols;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int m = at.first_m + 16 * i;
                const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                put<F32>(row + m, v, A.cols - m, whole, A.sums == 2);
            }
            continue;
        }
        type *const row = (type *)A.out + (int64_t)n * A.ld;
        auto value = [&](int i, int r) { return none ? 0.f : acc[i][j][r] * scale; };
        if constexpr (kPairs) {
            const float rest = A.rest && !none ? A.rest[n] * scale : 0.f;
            const type *const target = (const type *)A.weight + (int64_t)max(y, 0) * A.ld_weight;
#pragma unroll
            for (int i = 0; i < S::FM; i += 2) {
                const f32x4 first = {value(i, 0), value(i, 1), value(i, 2), value(i, 3)}, second = {value(i + 1, 0), value(i + 1, 1), value(i + 1, 2), value(i + 1, 3)};
                const int m = wave_m + 16 * (i + pair.tile) + pair.row;
                if (plain) {                               // (the same for all lanes, which change places)
                    *(typename S::element::piece *)(row + m) = paired<typename S::element>(first, second);
                } else {
                    float v[8];
                    paired32(first, second, v);
                    if (rest != 0.f && m < A.cols) add_rest(v, rest, target + m, A.cols - m);
                    put<typename S::element>(row + m, v, A.cols - m, whole, A.add);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int m = at.first_m + 16 * i;
                const float v[4] = {value(i, 0), value(i, 1), value(i, 2), value(i, 3)};
                put<typename S::element>(row + m, v, A.cols - m, whole, A.add);
            }
        }
    }
#endif
}

// The slices' sums, added in their order, and the targets' rests; rounded.
template <class T>
__global__ __launch_bounds__(256) void join_slices(const GradArgs A, const float *sums, int slices, int64_t N, int D)
{
#ifdef __HIP_DEVICE_COMPILE__
    typedef typename T::type type;
    const int groups = (D + kVec - 1) / kVec;
    const int64_t total = N * groups;
    for (int64_t at = blockIdx.x * 256ll + threadIdx.x; at < total; at += gridDim.x * 256ll) {
        const int64_t n = at / groups;
        const int c = (int)(at - n * groups) * kVec;
        const float *from = sums + n * D + c;
        f32x8 v = load8f(from, D - c);
#pragma unroll 4
        for (int s = 1; s < slices; ++s) v += load8f(from + s * N * D, D - c);
        const int y = target_of(A.targets, n, A.i64, A.V);
        const bool none = y < 0 || (A.row_weight && A.row_weight[n] == 0.f);
        if (A.rest && !none) add_rest(v, A.rest[n], (const type *)A.weight + y * A.ld_weight + c, D - c);
        const f32x8 zeros = {};
        store8f((type *)A.out + n * A.ld + c, D - c, none ? zeros : v * (A.scale ? A.scale[1] : 1.f));
    }
#endif
}

// Rows copied to aligned ones, `cols` padded with zeros to ld_to; rows without a target, or of weight 0, are copied as zeros.  scale: one more
// workgroup finds it (a launch of its own took 5 us).
template <class E>
__global__ __launch_bounds__(256) void pack_rows(const E *from, int64_t ld_from, int64_t rows, int cols, E *to, int64_t ld_to, const void *targets, const float *row_weight,
                                                 bool i64, int V, int32_t *status, float *scale)
{
#ifdef __HIP_DEVICE_COMPILE__
    const unsigned blocks = gridDim.x - (scale ? 1 : 0);
    if (blockIdx.x == blocks) {
        find_scale(targets, i64, V, rows, row_weight, scale);
        return;
    }
    if (status && blockIdx.x == 0 && threadIdx.x < kStatusWords) status[threadIdx.x] = 0;
    const int groups = (int)((ld_to + kVec - 1) / kVec);
    const int64_t total = rows * groups;
    for (int64_t at = blockIdx.x * 256ll + threadIdx.x; at < total; at += blocks * 256ll) {
        const int64_t n = at / groups;
        const int c = (int)(at - n * groups) * kVec;
        const bool there = !targets || (target_of(targets, n, i64, V) >= 0 && !(row_weight && row_weight[n] == 0.f));
        typename Eight<E>::type v = {};
        if (there && c < cols) v = load8(from + n * ld_from + c, cols - c);
        store8(to + n * ld_to + c, ld_to - c, v);
    }
#endif
}

// ---- host ----------------------------------------------------------------------------------------------------------

enum LogitKind { kLoss, kQ };
template <class S>
void launch_logits(LogitKind kind, LogitArgs a, hipStream_t stream)
{
    a.tiles_m = (a.o.m + S::BM - 1) / S::BM;
    a.tiles_n = (a.N + S::BN - 1) / S::BN;
    a.group = 8;
    const dim3 grid((unsigned)(a.tiles_m * a.tiles_n));
    if (kind == kLoss) hipLaunchKernelGGL(loss_tiles<S>, grid, dim3(S::kThreads), S::kLds, stream, a);
    else hipLaunchKernelGGL(q_tiles<S>, grid, dim3(S::kThreads), S::kLds, stream, a);
}
template <class T>
void launch_logits(int shape, LogitKind kind, const LogitArgs &a, hipStream_t stream)
{
    switch (shape) {
        case 0:
            if constexpr (!std::is_same<T, F32>::value) launch_logits<Shape0<T>>(kind, a, stream);
            break;
        case 1: launch_logits<Shape1<T>>(kind, a, stream); break;
        case 2: launch_logits<Shape2<T>>(kind, a, stream); break;
        case 3: launch_logits<Shape3<T>>(kind, a, stream); break;
        default: launch_logits<Shape4<T>>(kind, a, stream); break;
    }
}
template <class S>
void launch_grad(GradArgs a, int slices, hipStream_t stream)
{
    a.tiles_m = (a.cols + S::BM - 1) / S::BM;
    a.tiles_n = (a.rows + S::BN - 1) / S::BN;
    a.group = 8;
    hipLaunchKernelGGL(grad_tiles<S>, dim3((unsigned)(a.tiles_m * a.tiles_n), (unsigned)slices), dim3(S::kThreads), S::kLds, stream, a);
}
// (the hidden rows': the weights as columns; the weights': both operands)
template <class T, bool COLS_B>
void launch_grad(int shape, const GradArgs &a, int slices, hipStream_t stream)
{
    switch (shape) {
        case 0:
            if constexpr (!std::is_same<T, F32>::value) launch_grad<Shape0<T, true, COLS_B>>(a, slices, stream);
            break;
        case 1: launch_grad<Shape1<T, true, COLS_B>>(a, slices, stream); break;
        case 2: launch_grad<Shape2<T, true, COLS_B>>(a, slices, stream); break;
        case 3: launch_grad<Shape3<T, true, COLS_B>>(a, slices, stream); break;
        default: launch_grad<Shape4<T, true, COLS_B>>(a, slices, stream); break;
    }
}

unsigned blocks_for(int64_t elements) { return (unsigned)std::min<int64_t>((elements + 255) / 256, 8192); }

template <class T>
int token_loss(const pollux_loss_dims &d, const LossPlan &p, const char *hidden, const char *weight, const void *targets, char *ws,
               float *loss, float *lse, hipStream_t stream)
{
    typedef typename T::type type;
    constexpr int e = sizeof(type);
    const int N = (int)d.N;
    const int64_t ld_h = p.pack_hidden ? p.d_pad : d.hidden_stride, ld_w = p.pack_weight ? p.d_pad : d.weight_stride;
    int32_t *status = (int32_t *)(ws + p.status);
    if (N == 0) {
        hipLaunchKernelGGL(clear_status, dim3(1), dim3(64), 0, stream, status);
        return status_of(hipGetLastError());
    }
    if (p.pack_hidden) {
        hipLaunchKernelGGL(pack_rows<type>, dim3(blocks_for(N * ((p.d_pad + kVec - 1) / kVec))), dim3(256), 0, stream, (const type *)hidden, d.hidden_stride, (int64_t)N, d.D, (type *)(ws + p.hidden), p.d_pad, (const void *)nullptr, (const float *)nullptr, false, 0, (int32_t *)nullptr, (float *)nullptr);
        hidden = ws + p.hidden;
    }
    LogitArgs a = {};
    a.i64 = d.flags & PX_FLAG_TOKENS_I64;
    a.V = d.V;
    a.picked = (float *)(ws + p.picked);
    a.o.ldb = ld_h * e;
    a.o.lda = ld_w * e;
    a.o.k = (int)p.d_pad;                  // (where D is padded, both operands are packed)
    for (int first = 0; first < N; first += p.tokens) {
        a.targets = (const char *)targets + (int64_t)first * (a.i64 ? 8 : 4);
        a.N = a.o.n = std::min(p.tokens, N - first);
        a.o.b = hidden + first * a.o.ldb;
        int tiles = 0;
        for (int k = 0; k < p.pieces; ++k) {
            a.first = k * p.piece;
            a.rows = a.o.m = std::min(p.piece, d.V - a.first);
            const char *from = weight + (int64_t)a.first * d.weight_stride * e;
            if (p.pack_weight) {
                if (first == 0 || p.pieces > 1)
                    hipLaunchKernelGGL(pack_rows<type>, dim3(blocks_for(a.rows * ((p.d_pad + kVec - 1) / kVec))), dim3(256), 0, stream, (const type *)from, d.weight_stride, (int64_t)a.rows, d.D, (type *)(ws + p.weight), p.d_pad, (const void *)nullptr, (const float *)nullptr, false, 0, (int32_t *)nullptr, (float *)nullptr);
                from = ws + p.weight;
            }
            a.o.a = from;
            a.parts = (float2 *)(ws + p.parts) + (int64_t)tiles * a.N;
            a.status = first == 0 && k == 0 ? status : nullptr;
            launch_logits<T>(p.tiles, kLoss, a, stream);
            tiles += (a.rows + kShape[p.tiles].bm - 1) / kShape[p.tiles].bm;
        }
        auto join = [&](auto kernel, int tokens) {
            hipLaunchKernelGGL(kernel, dim3((a.N + tokens - 1) / tokens), dim3(kJoinThreads), 0, stream, (const float2 *)(ws + p.parts), tiles, a.N, (const float *)(ws + p.picked), a.targets,
                               a.i64, d.V, loss + first, lse + first, status);
        };
        // (few tokens: as many threads for each; three tokens of 1024 tiles 25 us with sixteen parts)
        if (a.N <= 1024) join(loss_join<2>, 2);
        else join(loss_join<16>, 16);
    }
    return status_of(hipGetLastError());
}

template <class T>
int token_loss_grad(const pollux_loss_dims &d, const LossPlan &p, const char *hidden, const char *weight, const void *targets, const float *lse,
                    const float *row_weight, char *ws, char *hidden_grad, char *weight_grad, hipStream_t stream)
{
    typedef typename T::type type;
    constexpr int e = sizeof(type);
    constexpr bool scaled = std::is_same<T, F16>::value;
    const int N = (int)d.N;
    const bool i64 = d.flags & PX_FLAG_TOKENS_I64;
    int32_t *status = (int32_t *)(ws + p.status);
    float *scale = scaled ? (float *)(ws + p.top) : nullptr;
    if (N == 0) {
        hipLaunchKernelGGL(clear_status, dim3(1), dim3(64), 0, stream, status);
        if (weight_grad && !(d.flags & PX_FLAG_ACCUMULATE)) {      // products over no tokens
            GradArgs g = {};
            g.o.m = g.cols = d.D;
            g.o.n = g.rows = d.V;
            g.out = weight_grad;
            g.ld = d.weight_grad_stride;            // (no scale: the sums are zeros)
            launch_grad<T, true>(1, g, 1, stream);
        }
        return status_of(hipGetLastError());
    }
    // (this clears the status word too; a product with q's zeros would still be NaN where a row that counts for nothing holds one)
    hipLaunchKernelGGL(pack_rows<type>, dim3(blocks_for(N * ((p.d_pad + kVec - 1) / kVec)) + (scaled ? 1 : 0)), dim3(256), 0, stream, (const type *)hidden, d.hidden_stride, (int64_t)N, d.D,
                       (type *)(ws + p.hidden), p.d_pad, targets, row_weight, i64, d.V, status, scale);
    LogitArgs a = {};
    a.targets = targets;
    a.i64 = i64;
    a.V = d.V;
    a.N = N;
    a.lse = lse;
    a.row_weight = row_weight;
    a.scale = scale;
    a.q = ws + p.q;
    a.rest = e == 2 ? (float *)(ws + p.rest) : nullptr;
    a.ld_q = p.v_pad;
    a.o.b = ws + p.hidden;
    a.o.ldb = p.d_pad * e;
    a.o.n = N;
    a.o.lda = (p.pack_weight ? p.d_pad : d.weight_stride) * e;
    a.o.k = (int)p.d_pad;                  // (where D is padded, both operands are packed)
    GradArgs h = {};                       // the hidden rows' gradient
    h.cols = d.D;
    h.rows = N;
    h.scale = scale;
    h.targets = targets;
    h.row_weight = row_weight;
    h.i64 = i64;
    h.V = d.V;
    h.rest = a.rest;
    h.weight = weight;
    h.ld_weight = d.weight_stride;
    h.ld = d.hidden_grad_stride;
    for (int k = 0; k < p.pieces; ++k) {
        a.first = k * p.piece;
        a.rows = a.o.m = std::min(p.piece, d.V - a.first);
        const char *from = weight + (int64_t)a.first * d.weight_stride * e;
        if (p.pack_weight) {
            hipLaunchKernelGGL(pack_rows<type>, dim3(blocks_for(a.rows * ((p.d_pad + kVec - 1) / kVec))), dim3(256), 0, stream, (const type *)from, d.weight_stride, (int64_t)a.rows, d.D, (type *)(ws + p.weight), p.d_pad, (const void *)nullptr, (const float *)nullptr, false, 0, (int32_t *)nullptr, (float *)nullptr);
            from = ws + p.weight;
        }
        a.o.a = from;
        a.status = k == 0 ? status : nullptr;
        launch_logits<T>(p.tiles, kQ, a, stream);
        if (hidden_grad) {
            h.o = {from, ws + p.q, a.o.lda, p.v_pad * e, d.D, N, a.rows};
            const int depth = kRowBytes / e, stages = (a.rows + depth - 1) / depth;
            h.slice_k = (stages + p.slices - 1) / p.slices * depth;
            h.sums = p.slices == 1 && p.pieces == 1 ? 0 : k == 0 ? 1 : 2;
            h.out = h.sums ? (void *)(ws + p.sums) : (void *)hidden_grad;
            launch_grad<T, false>(p.grad_tiles, h, p.slices, stream);
        }
        if (weight_grad) {
            GradArgs g = {};
            g.o = {ws + p.hidden, ws + p.q, p.d_pad * e, p.v_pad * e, d.D, a.rows, N};
            g.cols = d.D;
            g.rows = a.rows;
            g.slice_k = N;
            g.scale = scale;
            g.out = weight_grad + (int64_t)a.first * d.weight_grad_stride * e;
            g.ld = d.weight_grad_stride;
            g.add = d.flags & PX_FLAG_ACCUMULATE;
            launch_grad<T, true>(shape_for(d.D, a.rows, N, 1, e == 4), g, 1, stream);
        }
    }
    if (hidden_grad && (p.slices > 1 || p.pieces > 1)) {
        h.out = hidden_grad;
        hipLaunchKernelGGL(join_slices<T>, dim3(blocks_for((int64_t)N * ((d.D + kVec - 1) / kVec))), dim3(256), 0, stream, h, (const float *)(ws + p.sums), p.slices, (int64_t)N, d.D);
    }
    return status_of(hipGetLastError());
}

}  // namespace

LossPlan loss_plan(const pollux_loss_dims &d, bool grad)
{
    LossPlan p = {};
    const int64_t e = size_of_type(d.type), pad = 16 / e, N = d.N;
    const bool f32 = e == 4;
    auto padded = [&](int64_t x) { return (x + pad - 1) / pad * pad; };
    p.d_pad = padded(d.D);
    p.pack_hidden = d.hidden_stride % pad != 0 || d.D % pad != 0;
    p.pack_weight = d.weight_stride % pad != 0 || d.D % pad != 0;
    // A piece's q is held to 512 MiB, packed weights to 256.  Up to some 2^16 tokens pieces are then large enough to keep the matrix kernels' ends and the sums' passes over
    // memory to a few per cent; of 2^18 in 16 bits a piece has 1024 entries, and reading and writing the hidden rows' sums once a piece takes about as long as the
    // piece's product, of 2^20 (256 entries) several times as long.  There the scratch memory bounds the speed: such a batch is better given in parts.
    int64_t piece = (d.V + 255) / 256 * 256;
    // Forward, tokens are taken so many at a time that no launch has 2^32 threads, whatever its tiles; the lists of tiles are held to 4 GiB by it too.
    p.tokens = 1 << 15;
    if (grad) piece = std::min(piece, std::max<int64_t>(256, ((512ll << 20) / (std::max<int64_t>(N, 1) * e)) / 256 * 256));
    if (p.pack_weight) piece = std::min(piece, std::max<int64_t>(256, ((256ll << 20) / (p.d_pad * e)) / 256 * 256));
    p.pieces = (int)((d.V + piece - 1) / piece);
    // (even shares)
    piece = ((d.V + p.pieces - 1) / p.pieces + 255) / 256 * 256;
    p.piece = (int)piece;
    p.pieces = (int)((d.V + piece - 1) / piece);
    // (rows of q a stage longer than a power of two: those of one tile then begin in different channels of memory)
    p.v_pad = padded(std::min<int64_t>(piece, d.V)) + kRowBytes / e;
    p.tiles = shape_for(std::min<int64_t>(piece, d.V), grad ? N : std::min<int64_t>(N, p.tokens), d.D, 1, f32);
    p.slices = 1;
    if (grad) {
        // the hidden rows' gradient has few tiles and a long sum: in as many slices as takes least, their sums being written and read at some
        // 4 and 3 TB/s (2048 x 32768 x 1024 in one slice 579 us, in eight 117 and 23)
        double least = 1e300;
        for (int slices = 1; slices <= 32; slices *= 2) {
            if (slices > 1 && (p.v_pad * e / kRowBytes < 4 * slices || (int64_t)slices * N * d.D * 4 > (512ll << 20))) break;
            double cost;
            const int shape = shape_for(d.D, N, (double)piece / slices, slices, f32, &cost);
            if (slices > 1) cost += 4.0 + 4.0 * slices * N * d.D * (1 / 4e6 + 1 / 3e6);
            if (cost < least) least = cost, p.slices = slices, p.grad_tiles = shape;
        }
    }
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o = up256(o + bytes); return at; };
    p.status = take(4 * kStatusWords);
    p.top = take(256);
    if (!grad) {
        const size_t tiles = (size_t)p.pieces * ((piece + kShape[p.tiles].bm - 1) / kShape[p.tiles].bm);
        const size_t tokens = (size_t)std::min<int64_t>(N, p.tokens);
        p.parts = take(8 * tiles * tokens);
        p.picked = take(4 * tokens);
    }
    if (grad || p.pack_hidden) p.hidden = take((size_t)N * p.d_pad * e);
    if (p.pack_weight) p.weight = take((size_t)piece * p.d_pad * e);
    if (grad) {
        p.q = take((size_t)N * p.v_pad * e);
        if (!f32) p.rest = take(4 * (size_t)N);
        if (p.slices > 1 || p.pieces > 1) p.sums = take((size_t)p.slices * N * d.D * 4);
    }
    p.total = o;
    return p;
}

int launch_token_loss(const pollux_loss_dims &d, const LossPlan &p, const void *hidden, const void *weight, const void *targets,
                      void *workspace, float *loss, float *lse, hipStream_t stream)
{
    const char *h = (const char *)hidden, *w = (const char *)weight;
    switch (d.type) {
        case PX_TYPE_F32: return token_loss<F32>(d, p, h, w, targets, (char *)workspace, loss, lse, stream);
        case PX_TYPE_BF16: return token_loss<Bf16>(d, p, h, w, targets, (char *)workspace, loss, lse, stream);
        default: return token_loss<F16>(d, p, h, w, targets, (char *)workspace, loss, lse, stream);
    }
}

int launch_token_loss_grad(const pollux_loss_dims &d, const LossPlan &p, const void *hidden, const void *weight, const void *targets,
                           const float *lse, const float *row_weight, void *workspace, void *hidden_grad, void *weight_grad,
                           hipStream_t stream)
{
    const char *h = (const char *)hidden, *w = (const char *)weight;
    char *hg = (char *)hidden_grad, *wg = (char *)weight_grad, *ws = (char *)workspace;
    switch (d.type) {
        case PX_TYPE_F32: return token_loss_grad<F32>(d, p, h, w, targets, lse, row_weight, ws, hg, wg, stream);
        case PX_TYPE_BF16: return token_loss_grad<Bf16>(d, p, h, w, targets, lse, row_weight, ws, hg, wg, stream);
        default: return token_loss_grad<F16>(d, p, h, w, targets, lse, row_weight, ws, hg, wg, stream);
    }
}

}  // namespace px
