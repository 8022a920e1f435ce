// Rows of a table looked up by token, and the table's gradient: the rows' gradients summed by token.
//
// The lookup moves N rows in and out and nothing else.  The gradient is a sum over the places where a token occurs, as uneven as
// words are: a few tokens hold thousands of places, most one or none.  So the tokens are sorted first (stably, so that every
// order below is one), and the sorted places are cut into windows of equal length: each window sums its runs of equal tokens,
// writes those that lie within it, and leaves the sums of the two that its ends may cut (sum_windows); a second launch adds
// up the pieces of the runs that were cut, in their order (join_runs).  Work is even whatever the tokens are, no result depends on
// the order in which atomics arrive.  The sort is a chain of short launches on few compute units; further workgroups of them zero the
// table meanwhile (the few rows that tokens name are written twice, which costs less than telling them apart: 65536 x 2048 in bfloat16 from 16384
// rows 107 us with the others zeroed after the sort).

#include "pollux_host.h"
#include "pollux_rows.h"
#include "pollux_train.h"

#include <algorithm>

namespace px {
namespace {

template <int TYPE>
struct ElementOf;
template <>
struct ElementOf<PX_TYPE_F32> {
    typedef float type;
};
template <>
struct ElementOf<PX_TYPE_BF16> {
    typedef __bf16 type;
};
template <>
struct ElementOf<PX_TYPE_F16> {
    typedef _Float16 type;
};

// A wavefront a row, or, of wide rows, kRowPart columns of one (blockIdx.y).
constexpr int kRowPart = 64 * kVec * 8;
template <class T, class R>
__global__ __launch_bounds__(256) void embed_rows(const void *tokens, bool i64, int64_t N, int V, int D, const T *table, int64_t ld_table, float scale, R *rows,
                                                  int64_t ld_rows, int32_t *status)
{
#ifdef __HIP_DEVICE_COMPILE__
    const int64_t n = blockIdx.x * 4ll + (threadIdx.x >> 6);
    if (n >= N) return;
    bool bad;
    const int v = token_at(tokens, n, i64, V, bad);
    const int first = blockIdx.y * kRowPart, last = min(D, first + kRowPart);
    if (bad && status && blockIdx.y == 0 && (threadIdx.x & 63) == 0) atomicOr(status, PX_ST_BAD_TOKEN);
    const T *from = table + (int64_t)max(v, 0) * ld_table;
    R *to = rows + n * ld_rows;
#pragma unroll 4
    for (int c = first + (threadIdx.x & 63) * kVec; c < last; c += 64 * kVec) {
        f32x8 x = {};
        if (v >= 0) x = load8f(from + c, last - c) * scale;
        store8f(to + c, last - c, x);
    }
#endif
}

// ---- sort ----------------------------------------------------------------------------------------------------------
// Keys are tokens, V for none (sorted last, and dropped).  Up to kFew tokens: one workgroup counts, for every token, those before it
// (265 tokens 17 us in all; 642 30 so, in the passes 25).
// More: two passes, lowest digit first, of ceil(log2(V + 1)) / 2 bits.

// A table's rows from `first` on, `rows` of them, zeroed by the workgroups from `blocks` on, kZeroAhead groups of 16 bytes a thread and turn.
constexpr int kFew = 512, kThreads = 1024, kWaves = kThreads / 64, kMaxBits = 10, kZeroAhead = 4;
struct ZeroArgs {
    char *table;
    int64_t ld;                 // bytes
    int row;                    // bytes of a row, even
    int first, rows;
    int blocks;
    bool past;                  // the stores go past the caches
};
// (two loops for the two kinds of stores: of a branch at each store the compiler makes one of the ordinary kind)
template <bool PAST>
__device__ __forceinline__ void zero_rows(const ZeroArgs &Z, int64_t block, int64_t blocks)
{
#ifdef __HIP_DEVICE_COMPILE__
    const words none = {};
    auto put = [&](char *to, int64_t left) {
        if (left < 16)
            for (int i = 0; i < left; i += 2) *(short *)(to + i) = 0;
        else if constexpr (PAST)
            __builtin_nontemporal_store(none, (at_any *)to);
        else
            *(at_any *)to = none;
    };
    char *const table = Z.table + Z.first * Z.ld;
    if (Z.ld == Z.row) {                     // rows without gaps: one long one
        const int64_t bytes = (int64_t)Z.rows * Z.row, step = kThreads * 16;
        for (int64_t at = block * step * kZeroAhead + threadIdx.x * 16; at < bytes; at += blocks * step * kZeroAhead)
#pragma unroll
            for (int i = 0; i < kZeroAhead; ++i)
                if (at + i * step < bytes) put(table + at + i * step, bytes - at - i * step);
    } else {
        const int64_t groups = (Z.row + 15) / 16, total = groups * Z.rows;
        for (int64_t at = block * kThreads + threadIdx.x; at < total; at += blocks * kThreads) {
            const int64_t r = at / groups, byte = (at - r * groups) * 16;
            put(table + r * Z.ld + byte, Z.row - byte);
        }
    }
#endif
}
__device__ __forceinline__ bool zero_rows(const ZeroArgs &Z)
{
    const int64_t block = (int64_t)blockIdx.x - Z.blocks, blocks = (int64_t)gridDim.x - Z.blocks;
    if (block < 0) return false;
    if (Z.past) zero_rows<true>(Z, block, blocks);
    else zero_rows<false>(Z, block, blocks);
    return true;
}

// `parts` threads a token (a power of two, at most a wavefront), each of which compares it with as great a share of all; a key and its position in one
// number, so that one comparison decides (219 tokens: 7 us of comparing with a thread each and two).
__global__ __launch_bounds__(kThreads) void rank_few(const void *tokens, bool i64, int N, int V, int parts, int32_t *status, int *keys, int *places, const ZeroArgs Z)
{
    if (zero_rows(Z)) return;
    static_assert(kFew <= 1 << 10 && kFew <= kThreads, "positions of 10 bits below keys of 20");
    __shared__ int shared[kFew];
    __shared__ int bad_any;
    const int tid = threadIdx.x;
    if (tid == 0) bad_any = 0;
    if (tid < kStatusWords) status[tid] = 0;
    bool bad = false;
    if (tid < N) {
        const int v = token_at(tokens, tid, i64, V, bad);
        shared[tid] = (v < 0 ? V : v) << 10 | tid;
    }
    __syncthreads();
    if (bad) bad_any = 1;
    const int n = tid / parts, mine = n < N ? shared[n] : 0;
    int before = 0;
#pragma unroll 8
    for (int i = tid % parts; i < N; i += parts) before += shared[i] < mine ? 1 : 0;
    for (int w = 1; w < parts; w <<= 1) before += __shfl_xor(before, w);
    if (n < N && tid % parts == 0) {
        keys[before] = mine >> 10;
        places[before] = n;
    }
    __syncthreads();
    if (tid == 0 && bad_any) *status = PX_ST_BAD_TOKEN;
}

// A workgroup's tokens counted by their lowest digit; the second pass's counts and the status word are cleared.
__global__ __launch_bounds__(kThreads) void count_digits(const void *tokens, bool i64, int N, int V, int per_block, int bits, int *counts, int *counts2, int32_t *status, const ZeroArgs Z)
{
    if (zero_rows(Z)) return;
    __shared__ int bins[1 << kMaxBits];
    const int size = 1 << bits, first = blockIdx.x * per_block, last = min(N, first + per_block);
    for (int i = threadIdx.x; i < size; i += kThreads) bins[i] = 0;
    if (blockIdx.x == 0 && threadIdx.x < kStatusWords) status[threadIdx.x] = 0;
    __syncthreads();
    for (int n = first + threadIdx.x; n < last; n += kThreads) {
        bool bad;
        const int v = token_at(tokens, n, i64, V, bad);
        atomicAdd(&bins[(v < 0 ? V : v) & (size - 1)], 1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < size; i += kThreads) {
        counts[blockIdx.x * size + i] = bins[i];
        counts2[blockIdx.x * size + i] = 0;
    }
}

// One pass: every workgroup finds, from all workgroups' counts, where its tokens of each digit go, and puts them there in their
// order.  The first pass reads the tokens themselves and counts, for the second, the next digits of the places it fills.
template <bool FIRST>
__global__ __launch_bounds__(kThreads) void place_digits(const void *tokens, bool i64, const int *keys_in, const int *places_in, int N, int V, int blocks, int per_block,
                                                         int bits, const int *counts, int *counts2, int *keys, int *places, int32_t *status, const ZeroArgs Z)
{
    if (zero_rows(Z)) return;
    __shared__ int base[1 << kMaxBits];
    __shared__ int in_wave[kWaves][1 << kMaxBits];
    __shared__ int waves[kWaves];
    const int size = 1 << bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // digit `tid`: tokens of it in all workgroups and in those before this one
    int all = 0, before = 0;
    if (tid < size)
#pragma unroll 8
        for (int b = 0; b < blocks; ++b) {
            const int c = counts[b * size + tid];
            all += c;
            before += b < (int)blockIdx.x ? c : 0;
        }
    int sum = all;
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) {
        const int up = __shfl_up(sum, w);
        if (lane >= w) sum += up;
    }
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    int lower = 0;
    for (int w = 0; w < wave; ++w) lower += waves[w];
    if (tid < size) base[tid] = lower + sum - all + before;
    bool bad_seen = false;
    const int first = blockIdx.x * per_block, last = min(N, first + per_block);
    for (int at = first; at < last; at += kThreads) {
        const int n = at + tid;
        const bool there = n < last;
        int key = 0, place = 0;
        if (there) {
            if (FIRST) {
                bool bad;
                const int v = token_at(tokens, n, i64, V, bad);
                bad_seen |= bad;
                key = v < 0 ? V : v;
                place = n;
            } else {
                key = keys_in[n];
                place = places_in[n];
            }
        }
        const int digit = (FIRST ? key : key >> bits) & (size - 1);
        for (int i = tid; i < kWaves * size; i += kThreads) in_wave[i >> bits][i & (size - 1)] = 0;
        __syncthreads();
        // lanes of this wavefront with the same digit
        unsigned long long same = __ballot(there);
        for (int b = 0; b < bits; ++b) {
            const unsigned long long set = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        if (there && rank == 0) in_wave[wave][digit] = __popcll(same);
        __syncthreads();
        int total = 0;
        if (tid < size)
            for (int w = 0; w < kWaves; ++w) {
                const int c = in_wave[w][tid];
                in_wave[w][tid] = total;
                total += c;
            }
        __syncthreads();
        int to = 0;
        if (there) {
            to = base[digit] + in_wave[wave][digit] + rank;
            keys[to] = key;
            places[to] = place;
        }
        if (FIRST) {
            // equal keys go to places in a row, in one of the second pass's workgroups or in two: one lane counts for all that share both
            // (a frequent token is in a wavefront many times, and adding one by one they would wait for each other: 16384 tokens 12 us, 10 so)
            const int high = key >> bits, block = to / per_block;
            for (int b = 0; b < bits; ++b) {
                const unsigned long long set = __ballot((high >> b) & 1);
                same &= (high >> b) & 1 ? set : ~set;
            }
            const unsigned long long odd = __ballot(block & 1);
            same &= block & 1 ? odd : ~odd;
            if (there && (same & ((1ull << lane) - 1)) == 0) atomicAdd(&counts2[block * size + (high & (size - 1))], __popcll(same));
        }
        __syncthreads();
        if (tid < size) base[tid] += total;
        __syncthreads();
    }
    if (FIRST && bad_seen) atomicOr(status, PX_ST_BAD_TOKEN);
}

// ---- sums ----------------------------------------------------------------------------------------------------------

struct SumArgs {
    const int *keys, *places;
    int64_t ld_rows, ld_table;
    float *partial;             // [2][windows][D]: the run cut by a window's first place, by its last
    int N, V, D, window, windows;
    int lanes;                  // threads that share a window, kVec columns each: a power of two
    int groups;                 // 256 / lanes windows a workgroup
    bool add;
    float scale;
};

// WIDE: rows so wide that a wavefront has one window.  Its keys and places then come in one load each, a batch ahead, lane i's
// being the i-th, and are read out of the lanes: a batch's rows wait for no other load (16384 rows of 2048 in bfloat16 26 us with a load for each, one
// behind the other).
template <class R, class T, bool WIDE>
__global__ __launch_bounds__(256) void sum_windows(const SumArgs A, const R *rows, T *table)
{
#ifdef __HIP_DEVICE_COMPILE__
    const int group = threadIdx.x / A.lanes, w = blockIdx.x * A.groups + (WIDE ? __builtin_amdgcn_readfirstlane(group) : group);
    const int c = (blockIdx.y * A.lanes + threadIdx.x % A.lanes) * kVec;
    if (w >= A.windows || (!WIDE && c >= A.D)) return;        // (WIDE: all lanes stay, those past the row's end with nothing to load or store)
    const int first = w * A.window, last = min(A.N, first + A.window), left = A.D - c, lane = threadIdx.x & 63;
    f32x8 sum = {};
    constexpr int kAhead = sizeof(R) == 2 ? 16 : 8;
    int lane_key = 0, lane_place = 0;
    auto fetch = [&](int at) {
        if constexpr (WIDE) {
            const int p = min(at + lane, A.N - 1);
            lane_key = A.keys[p];
            lane_place = A.places[p];
        }
    };
    fetch(first);
    int run = A.keys[first];
    bool cut = first > 0 && A.keys[first - 1] == run;         // by the window's first place
    for (int at = first; at < last; at += kAhead) {
        typename Eight<R>::type x[kAhead];
        int key[kAhead + 1], place[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int p = min(at + i, A.N - 1);
            key[i] = WIDE ? __builtin_amdgcn_readlane(lane_key, i) : A.keys[p];
            place[i] = WIDE ? __builtin_amdgcn_readlane(lane_place, i) : A.places[p];
        }
        key[kAhead] = at + kAhead >= A.N ? -1 : WIDE ? __builtin_amdgcn_readlane(lane_key, kAhead) : A.keys[at + kAhead];
        if (at + kAhead < last) fetch(at + kAhead);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (at + i < last && key[i] < A.V) x[i] = load8(rows + (int64_t)place[i] * A.ld_rows + c, left);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (at + i >= last) break;
            if (key[i] >= A.V) return;                        // from here on no tokens
            if (key[i] != run) {
                run = key[i];
                cut = false;
                sum = f32x8{};
            }
            sum += __builtin_convertvector(x[i], f32x8);
            const bool ends = at + i + 1 >= A.N || key[i + 1] != run, final = at + i + 1 >= last;
            if (!ends && !final) continue;
            if (ends && !cut) {
                T *to = table + (int64_t)run * A.ld_table + c;
                f32x8 out = sum * A.scale;
                if (A.add) out += load8f(to, left);
                store8f(to, left, out);
            } else {
                store8f(A.partial + ((int64_t)(cut ? 0 : A.windows) + w) * A.D + c, left, sum);
            }
        }
    }
#endif
}

// The runs that windows cut: the window in which one begins adds up the pieces, its own and those of the windows after it, a
// quarter of them each of four wavefronts, and these in their order.
template <class T>
__global__ __launch_bounds__(256) void join_runs(const SumArgs A, T *table)
{
#ifdef __HIP_DEVICE_COMPILE__
    __shared__ f32x8 shared[3][64];
    const int w = blockIdx.x, part = threadIdx.x >> 6, c = (blockIdx.y * 64 + (threadIdx.x & 63)) * kVec, left = A.D - c;
    const int first = w * A.window, last = first + A.window, run = A.keys[last - 1];
    if (run >= A.V || A.keys[last] != run) return;            // nothing is cut by this window's end
    if (A.keys[first] == run && first > 0 && A.keys[first - 1] == run) return;      // it began before
    // whole windows that the run fills after this one, 64 looked at together, and the one in which it ends
    int count = 1;
    for (int u = w + 1;; u += 64) {
        const int64_t next = ((int64_t)u + (threadIdx.x & 63) + 1) * A.window;      // the first place after a window
        const unsigned long long over = __ballot(next >= A.N || A.keys[next] != run);
        if (over) {
            count += u - (w + 1) + __ffsll(over) - 1;
            break;
        }
    }
    const int each = (count + 3) >> 2, u0 = w + 1 + part * each, u1 = min(w + 1 + count, u0 + each);
    f32x8 sum = {};
    if (c < A.D) {
        if (part == 0) sum = load8f(A.partial + ((int64_t)A.windows + w) * A.D + c, left);
#pragma unroll 8
        for (int u = u0; u < u1; ++u) sum += load8f(A.partial + (int64_t)u * A.D + c, left);
    }
    if (part > 0) shared[part - 1][threadIdx.x & 63] = sum;
    __syncthreads();
    if (part > 0 || c >= A.D) return;
#pragma unroll
    for (int i = 0; i < 3; ++i) sum += shared[i][threadIdx.x];
    T *to = table + (int64_t)run * A.ld_table + c;
    sum *= A.scale;
    if (A.add) sum += load8f(to, left);
    store8f(to, left, sum);
#endif
}

template <class R, class T>
int embed_grad(const pollux_embed_dims &d, const EmbedPlan &p, const void *tokens, const R *rows, char *ws, T *table, hipStream_t stream)
{
    const int N = (int)d.N;
    const bool i64 = d.flags & PX_FLAG_TOKENS_I64;
    int32_t *status = (int32_t *)(ws + p.status);
    int *keys[2] = {(int *)(ws + p.keys[0]), (int *)(ws + p.keys[1])}, *places[2] = {(int *)(ws + p.places[0]), (int *)(ws + p.places[1])};
    const bool add = d.flags & PX_FLAG_ACCUMULATE;
    // rows [V at / 16, V to / 16) of the table zeroed by a launch whose own workgroups are `blocks`.  Each of the sort's three launches takes about a third, the second,
    // which counts besides, the most: a table that is written for longer than the sort runs keeps all three busy (16384 x 2048 in bfloat16 into 65536 rows 77 us, 91 with all
    // zeros in the first and 85 in the second; 16384 x 4096 into 131072 245, 266, 260), a small one fits any (5003 x 1000 in fp32 into 20011 37, 39, 36; 10^6 x 256 into
    // 200000 369, 374, 365).  Shares of 4, 7, 5 and of 5, 6, 5 sixteenths are within 1 %.
    // (A table that the memory-side cache of 256 MiB holds beside the rows stays there: 29114 x 2048 in fp32 40 us, 54 with stores past the
    // caches; a larger one only pushes the rows out: 65536 x 2048 in bfloat16 from 16384 rows 95 us, 81 past them.)
    const bool past = (int64_t)d.V * d.D * (int64_t)sizeof(T) + (int64_t)N * d.D * (int64_t)sizeof(R) > (256ll << 20);
    auto zero = [&](int at, int to, int blocks) {
        const int first = (int)((int64_t)d.V * at / 16), last = (int)((int64_t)d.V * to / 16);
        return ZeroArgs{(char *)table, d.table_stride * (int64_t)sizeof(T), d.D * (int)sizeof(T), first, add ? 0 : last - first, blocks, past};
    };
    auto grid = [&](const ZeroArgs &z) {
        const int64_t groups = ((int64_t)z.row + 15) / 16 * z.rows, each = kThreads * kZeroAhead;
        return dim3((unsigned)(z.blocks + std::min<int64_t>((groups + each - 1) / each, 512)));
    };
    if (p.passes == 0) {
        const ZeroArgs z = zero(0, 16, 1);
        int parts = 1;
        while (parts < 64 && 2 * parts * N <= kThreads) parts *= 2;
        hipLaunchKernelGGL(rank_few, grid(z), dim3(kThreads), 0, stream, tokens, i64, N, d.V, parts, status, keys[1], places[1], z);
    } else {
        int *counts = (int *)(ws + p.counts), *counts2 = counts + ((size_t)p.blocks << p.bits);
        const ZeroArgs z[3] = {zero(0, 4, p.blocks), zero(4, 11, p.blocks), zero(11, 16, p.blocks)};
        hipLaunchKernelGGL(count_digits, grid(z[0]), dim3(kThreads), 0, stream, tokens, i64, N, d.V, p.per_block, p.bits, counts, counts2, status, z[0]);
        hipLaunchKernelGGL(place_digits<true>, grid(z[1]), dim3(kThreads), 0, stream, tokens, i64, (const int *)nullptr, (const int *)nullptr, N, d.V, p.blocks,
                           p.per_block, p.bits, (const int *)counts, counts2, keys[0], places[0], status, z[1]);
        hipLaunchKernelGGL(place_digits<false>, grid(z[2]), dim3(kThreads), 0, stream, tokens, i64, (const int *)keys[0], (const int *)places[0], N, d.V, p.blocks,
                           p.per_block, p.bits, (const int *)counts2, (int *)nullptr, keys[1], places[1], status, z[2]);
    }
    SumArgs a = {};
    a.keys = keys[1];
    a.places = places[1];
    a.ld_rows = d.rows_stride;
    a.ld_table = d.table_stride;
    a.partial = (float *)(ws + p.partial);
    a.N = N;
    a.V = d.V;
    a.D = d.D;
    a.window = p.window;
    a.windows = p.windows;
    a.lanes = 1;
    while (a.lanes < 256 && a.lanes * kVec < d.D) a.lanes *= 2;
    a.groups = 256 / a.lanes;
    a.add = add;
    a.scale = d.scale;
    const unsigned parts = (unsigned)((d.D + 256 * kVec - 1) / (256 * kVec));
    const dim3 grid_sums((unsigned)((p.windows + a.groups - 1) / a.groups), parts);
    if (p.windows > 0 && a.lanes >= 64) hipLaunchKernelGGL((sum_windows<R, T, true>), grid_sums, dim3(256), 0, stream, a, rows, table);
    else if (p.windows > 0) hipLaunchKernelGGL((sum_windows<R, T, false>), grid_sums, dim3(256), 0, stream, a, rows, table);
    if (p.windows > 1) hipLaunchKernelGGL(join_runs<T>, dim3((unsigned)(p.windows - 1), (unsigned)((d.D + 64 * kVec - 1) / (64 * kVec))), dim3(256), 0, stream, a, table);
    return status_of(hipGetLastError());
}

template <class F>
int with_type(int type, F f)
{
    switch (type) {
        case PX_TYPE_F32: return f(ElementOf<PX_TYPE_F32>());
        case PX_TYPE_BF16: return f(ElementOf<PX_TYPE_BF16>());
        default: return f(ElementOf<PX_TYPE_F16>());
    }
}

}  // namespace

EmbedPlan embed_plan(const pollux_embed_dims &d)
{
    EmbedPlan p = {};
    const int N = (int)d.N;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o = up256(o + bytes); return at; };
    p.status = take(4 * kStatusWords);
    if (N > kFew) {
        int bits = 1;
        while (((int64_t)1 << (2 * bits)) <= d.V) ++bits;       // keys 0 .. V
        p.bits = bits;
        p.passes = 2;
        // at most 64 workgroups: each reads all of their counts
        p.per_block = std::max(kThreads, ((N + 63) / 64 + kThreads - 1) / kThreads * kThreads);
        p.blocks = (N + p.per_block - 1) / p.per_block;
        p.counts = take((size_t)2 * p.blocks * 4 << bits);
        p.keys[0] = take(4 * (size_t)N);
        p.places[0] = take(4 * (size_t)N);
    }
    p.keys[1] = take(4 * (size_t)N);
    p.places[1] = take(4 * (size_t)N);
    // Windows: of few tokens short ones, which give many wavefronts work and end soon; of many long ones, whose cut runs' pieces are fewer to write and join.  With 8, 16, 32, 64,
    // 128 places: 5003 x 1000 in fp32 36, 37, 45, 59, 87 us; 16384 x 2048 in bfloat16 80, 78, 78, 85, 105; 65536 x 1024 92, 79, 72, 72, 84; 131072 x 1024 172, 144, 128, 120,
    // 121; 10^6 x 1024 1185, 943, 829, 760, 733.
    p.window = N <= 1 << 13 ? 8 : N <= 1 << 15 ? 16 : N <= 1 << 17 ? 32 : 128;
    p.windows = (N + p.window - 1) / p.window;
    p.partial = take(2 * (size_t)p.windows * d.D * 4);
    p.total = o;
    return p;
}

int launch_embed(const pollux_embed_dims &d, const void *tokens, const void *table, void *rows, int32_t *status, hipStream_t stream)
{
    if (d.N == 0) return PX_OK;
    return with_type(d.table_type, [&](auto t) {
        return with_type(d.rows_type, [&](auto r) {
            typedef typename decltype(t)::type T;
            typedef typename decltype(r)::type R;
            hipLaunchKernelGGL((embed_rows<T, R>), dim3((unsigned)((d.N + 3) / 4), (unsigned)((d.D + kRowPart - 1) / kRowPart)), dim3(256), 0, stream, tokens,
                               (d.flags & PX_FLAG_TOKENS_I64) != 0, d.N, d.V, d.D, (const T *)table, d.table_stride, d.scale, (R *)rows, d.rows_stride, status);
            return status_of(hipGetLastError());
        });
    });
}

int launch_embed_grad(const pollux_embed_dims &d, const EmbedPlan &p, const void *tokens, const void *rows_grad, void *workspace, void *table_grad,
                      hipStream_t stream)
{
    return with_type(d.table_type, [&](auto t) {
        return with_type(d.rows_type, [&](auto r) {
            typedef typename decltype(t)::type T;
            typedef typename decltype(r)::type R;
            return embed_grad<R, T>(d, p, tokens, (const R *)rows_grad, (char *)workspace, (T *)table_grad, stream);
        });
    });
}

}  // namespace px
