// Matrix products on the matrix units, shared by the loss and the orthogonalised update: one tile of
//   C[m, n] = sum_k A[m, k] B[n, k]
// per workgroup, sums in fp32.  Either operand may lie in memory as its rows (k contiguous) or as its columns (rows of k, m or n
// contiguous): a product with a transposed matrix needs no transposed copy.
//
// A stage of k (128 bytes of a row: 64 elements of 16 bits, 32 of 32 bits) comes into LDS by loads that write LDS directly,
// two stages in turn, three of tiles of 192, five of the smallest tiles, which would otherwise wait for every one.  What a load writes is in the order of its lanes, so it is the address a lane loads from that is permuted:
// * rows: a row's eight 16-byte pieces lie in the order piece ^ (row & 7); the sixteen rows' pieces that a wavefront reads
//   together then touch every bank once.
// * columns: a row of k is BM (BN) elements; its pieces lie in the order piece ^ f(k), which puts the four rows of k that sixteen lanes read
//   together (eight bytes each, turned by the read into four k of one column a lane; in fp32 four reads) on different banks.
// Each lane holds column n = lane & 15 of a 16 x 16 tile and four consecutive rows m: what runs over m (the vocabulary) is
// reduced mostly in registers, and four elements contiguous in m go out in one store.
// 8192 x 8192 x 4096 in bfloat16, tiles of 256 x 256: 1.38 PFLOP/s, where a large library product reaches 1.28 to 1.59.  The matrix units are
// busy 61 to 70 % of the time, at a clock that falls to 1.85 to 1.95 GHz under that load (2.1 GHz at 39 %): what is left is power as much as stalls, and
// tiles streamed through one workgroup a compute unit (the next one's loads under way while one is finished), priorities of wavefronts and other
// orders of loads and reads between the products all took the same time or more.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "pollux_kept.h"
#include "pollux_train.h"

namespace px {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// The element types: what a value is stored as, and the product of 16 bytes of k of sixteen rows with those of sixteen others
// (four lanes share a row).
struct Bf16 {
    typedef __bf16 type;
    typedef bf16x8 piece;
};
struct F16 {
    typedef _Float16 type;
    typedef f16x8 piece;
};
struct F32 {
    typedef float type;
    typedef f32x4 piece;
};

constexpr int kRowBytes = 128;      // of k, a stage

// m, n: rows of A and B.  Rows: the elements between k and the next multiple of 16 bytes are zeros in at least one operand and finite
// in the other.  Columns: rows of k are whole 16-byte groups.  k = 0 gives a tile of zeros.
struct Operands {
    const char *a, *b;
    int64_t lda, ldb;       // bytes from row to row in memory, multiples of 16, as are the pointers
    int m, n, k;
    const uint8_t *scales;  // of a, kept in 8 bits as its columns: rows of lda codes, lda / 32 scales
};

// Workgroup -> tile.  Workgroups go round the eight XCDs, each with a cache of its own: the tiles are cut into eight runs, one
// an XCD, and a run walks `group` tiles of m by all of n, so that the workgroups on an XCD at one time share rows of both
// operands (8192 x 8192 x 4096: 1062, 1242, 1269 TFLOP/s with groups of 4, 8, 16; 4096 x 8192 x 16384: 1294, 1269, 900).
struct Tile {
    int m, n;
};
__device__ __forceinline__ Tile tile_of(int block, int tiles_m, int tiles_n, int group)
{
    const int total = tiles_m * tiles_n, q = total >> 3, r = total & 7, xcd = block & 7;
    const int at = xcd * q + min(xcd, r) + (block >> 3);
    const int per = group * tiles_n, g = at / per, first = g * group, size = min(tiles_m - first, group), rest = at - g * per;
    return {first + rest % size, rest / size};
}

// The same of a symmetric product: the tiles with n <= m, row by row of m.
__device__ __forceinline__ Tile triangle_of(int block, int tiles)
{
    const int total = tiles * (tiles + 1) / 2, q = total >> 3, r = total & 7, xcd = block & 7;
    const int at = xcd * q + min(xcd, r) + (block >> 3);
    int m = (int)((sqrtf(8.f * at + 1.f) - 1.f) * 0.5f);
    while (m * (m + 1) / 2 > at) --m;
    while ((m + 1) * (m + 2) / 2 <= at) ++m;
    return {m, at - m * (m + 1) / 2};
}

template <class T, int BM_, int BN_, int WM_, int WN_, int STAGES_, bool COLS_A_ = false, bool COLS_B_ = false, int KEPT_ = PX_KEPT_NONE>
struct TileShape {
    typedef T element;
    static constexpr int KEPT = KEPT_;                            // the form that A, its columns in memory, is kept in
    static constexpr bool COLS_A = COLS_A_, COLS_B = COLS_B_;     // the operand lies in memory as its columns
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int kThreads = WM * WN * 64, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    static constexpr int kStages = STAGES_, kStage = (BM + BN) * kRowBytes, kLds = kStages * kStage;
    static constexpr int kLoadsA = BM * kRowBytes / (kThreads * 16), kLoadsB = BN * kRowBytes / (kThreads * 16);
    static_assert(kLoadsA * kThreads * 16 == BM * kRowBytes && kLoadsB * kThreads * 16 == BN * kRowBytes, "whole loads");
};

// Which shape of tile a product is formed in, and in how many slices of k: by what it is estimated to take, in microseconds.  A compute
// unit works on per_cu tiles of a shape at once; a stage takes `alone` for one of them and `full` for per_cu (in fp32 alone32 and full32), and
// a round of tiles begins and ends in `ends`.  Fitted to products of 64 to 2048 x 384 to 65536 x 64 to 8192 and within some 20 % of them: bfloat16 2048 x 32768 x 1024 133, 170,
// 235, 407, 275 us in the first five shapes, 1500 x 50000 x 1000 180, 229, 328, 624, 352, 512 x 8192 x 512 21, 12.5, 11.5, 19.4, 15, 1024 x 1024 x 1024 31, 16, 12, 12, 9;
// fp32 512 x 8192 x 512 33 and 41 us in the second and third.
constexpr int kShapes = 6;
struct ShapeOf {
    int bm, bn, per_cu;
    double alone, full, alone32, full32, ends;
};
constexpr ShapeOf kShape[kShapes] = {
    {256, 256, 1, 1.53, 1.53, 0.00, 0.00, 8.7}, {128, 128, 2, 0.80, 0.93, 1.70, 2.62, 6.0}, {64, 64, 4, 0.45, 0.67, 0.45, 2.24, 4.5},
    {128, 16, 4, 0.45, 0.65, 0.45, 1.35, 5.5},  {64, 64, 2, 0.28, 0.60, 0.47, 1.17, 4.5},  {192, 192, 1, 0.92, 0.92, 0.00, 0.00, 7.0}};

inline double shape_cost(const ShapeOf &s, int64_t m, int64_t n, double k, int64_t count, bool f32, bool symmetric = false)
{
    const double tiles_m = (double)((m + s.bm - 1) / s.bm), tiles_n = (double)((n + s.bn - 1) / s.bn);
    const double tiles = (symmetric ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n) * count, each = ceil(tiles / 256);
    const double stages = ceil(k / (f32 ? 32 : 64)), rounds = floor(each / s.per_cu), rest = each - rounds * s.per_cu;
    auto round = [&](double at_once) {
        const double alone = f32 ? s.alone32 : s.alone, full = f32 ? s.full32 : s.full;
        const double stage = s.per_cu > 1 ? alone + (full - alone) * (at_once - 1) / (s.per_cu - 1) : full;
        return stages * stage + s.ends;
    };
    return rounds * round(s.per_cu) + (rest > 0 ? round(rest) : 0.0);
}

// `count` products [m, n] over k; the least estimate goes to *cost, if that is given.  The last shape is for orthogonalised updates alone.
inline int shape_for(int64_t m, int64_t n, double k, int64_t count, bool f32, double *cost = nullptr)
{
    int best = 0;
    double least = 1e300;
    for (int s = f32 ? 1 : 0; s < kShapes - 1; ++s) {          // (in fp32 the split's registers leave no room for tiles of 256)
        const double c = shape_cost(kShape[s], m, n, k, count, f32);
        if (c < least) least = c, best = s;
    }
    if (cost) *cost = least;
    return best;
}

// For orthogonalised updates, 16 bits.  A symmetric product [m, m] may take the tiles on one side of the diagonal alone (square ones), which
// pays where all tiles are more than the chip takes at once: turning a tile to store it on the other side takes 0.6 to 0.8 us.
inline StepShape step_shape_for(int64_t m, int64_t n, double k, int64_t count, bool symmetric)
{
    StepShape best = {0, false};
    double least = 1e300;
    for (int half = 0; half <= (symmetric ? 1 : 0); ++half)
        for (int s = 0; s < kShapes; ++s) {
            if (half && kShape[s].bm != kShape[s].bn) continue;
            const double c = shape_cost(kShape[s], m, n, k, count, false, half) + (half ? 0.8 : 0.0);
            if (c < least) least = c, best = {s, half != 0};
        }
    return best;
}

template <class T, bool COLS_A = false, bool COLS_B = false>
using Shape0 = TileShape<T, 256, 256, 2, 4, 2, COLS_A, COLS_B>;
template <class T, bool COLS_A = false, bool COLS_B = false>
using Shape1 = TileShape<T, 128, 128, 2, 2, 2, COLS_A, COLS_B>;
template <class T, bool COLS_A = false, bool COLS_B = false>
using Shape2 = TileShape<T, 64, 64, 2, 2, 2, COLS_A, COLS_B>;
template <class T, bool COLS_A = false, bool COLS_B = false>
using Shape3 = TileShape<T, 128, 16, 2, 1, 2, COLS_A, COLS_B>;
template <class T, bool COLS_A = false, bool COLS_B = false>
using Shape4 = TileShape<T, 64, 64, 2, 2, 5, COLS_A, COLS_B>;
template <class T, bool COLS_A = false, bool COLS_B = false>
using Shape5 = TileShape<T, 192, 192, 2, 4, 3, COLS_A, COLS_B>;

#ifdef __HIP_DEVICE_COMPILE__

__device__ __forceinline__ f32x4 multiply(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
// fp32: four products of k = 4; which four of a row's sixteen k each takes is the same for both operands.  (Where the split below does not hold.)
__device__ __forceinline__ f32x4 multiply(f32x4 a, f32x4 b, f32x4 c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// fp32 on the units of 16 bits, which multiply sixteen times as fast: x = p[0] + p[1] + p[2] in bfloat16, each the nearest to what the ones before leave, so that all 24 bits are
// there (of numbers from 2^-109 up).  For x from 1 to 2, p[1] is at most 2^-8 and p[2] 2^-17: of the nine products of two such sums the three of the lowest bits, at most 2^-24 of the whole
// together, half a step of fp32, and of either sign, are left out.  Six products of 16 bits in place of one, exact in the fp32 sums.  (p[0] cut off instead of rounded leaves p[1] twice and p[2]
// twice as large, and 2^-22 of a product: 1500 x 20000 x 1024 step 1.28 ms so, 1.30.)
struct Split {
    bf16x8 p[3];
};
__device__ __forceinline__ Split split(f32x4 low, f32x4 high)
{
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    typedef float f32x2_ __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    u32x4 p[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = i < 2 ? low[2 * i] : high[2 * i - 4], y = i < 2 ? low[2 * i + 1] : high[2 * i - 3];
        const unsigned first = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2_{x, y}, bf16x2));
        p[0][i] = first;
        const float rx = x - __uint_as_float(first << 16), ry = y - __uint_as_float(first & 0xffff0000u);
        const unsigned second = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2_{rx, ry}, bf16x2));
        p[1][i] = second;
        const float sx = rx - __uint_as_float(second << 16), sy = ry - __uint_as_float(second & 0xffff0000u);
        p[2][i] = __builtin_amdgcn_perm(__float_as_uint(sy), __float_as_uint(sx), 0x07060302u);
    }
    Split s;
#pragma unroll
    for (int k = 0; k < 3; ++k) s.p[k] = __builtin_bit_cast(bf16x8, p[k]);
    return s;
}

// Where the lane's values of acc[i][j] belong: rows m = first_m + 16 i + 0..3 and column n = first_n + 16 j of the product.
template <class S>
struct Place {
    int first_m, first_n;
    __device__ __forceinline__ Place(Tile t)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        first_m = t.m * S::BM + wave / S::WN * S::TM + (lane >> 4) * 4;
        first_n = t.n * S::BN + wave % S::WN * S::TN + (lane & 15);
    }
};

typedef __attribute__((address_space(3))) char lds_char;

// Eight bytes a lane out of LDS, sixteen lanes' worth turned: lane i of sixteen gets element i % 4 of lanes i / 4, 4 + i / 4, 8 + i / 4
// and 12 + i / 4.  (The pointer is restrict for what the compiler concludes from it: a read that it knows nothing of would wait for
// every load into LDS that is on its way, those of other stages among them.)
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ __forceinline__ s16x4 read_turned(lds_s16x4 *__restrict from) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(from); }

// One operand of a tile: B_ rows of it (BM or BN), of which the wavefront multiplies F x 16 from `mine` on.
template <class T, int B_, int F, int THREADS, bool COLS>
struct Side {
    typedef typename T::piece piece;
    static constexpr int kSize = sizeof(typename T::type), kDepth = kRowBytes / kSize;      // k of a stage
    static constexpr int kLoads = B_ * kRowBytes / (THREADS * 16), kReads = F * (COLS ? (kSize == 4 ? 4 : 2) : 1);
    static constexpr int kLine = COLS ? B_ * kSize : kRowBytes, kPieces = kLine / 16;       // a row in LDS
    const char *base;
    int64_t ld;
    int bytes, k, stages, part;         // (rows) of the buffer; k in bytes; stages, and the one that is not whole
    int width;                          // (columns) bytes of a row of k
    int at[kLoads], piece_at;
    // of the lane's pieces in LDS.  Rows, and columns of a power of two: the first one's, the others being a step or a changed bit away
    static constexpr bool kEach = COLS && (B_ & (B_ - 1)) != 0;
    int from[kEach ? F : 1];

    // the permutation of a row of k (of 24 pieces, within eight of them)
    static __device__ __forceinline__ int f(int row) { return (kSize == 4 ? (row >> 2 & 3) << 2 : (row & 3) << 1 | (row >> 3 & 1) << 3) & (kPieces - 1); }

    __device__ __forceinline__ Side(const char *p, int64_t ld_, int first, int rows, int k_, int mine)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        ld = ld_;
        stages = (k_ + kDepth - 1) / kDepth;
        const int left = min(rows - first, B_);
        if (COLS) {
            base = p + (int64_t)first * kSize;
            k = k_;
            width = (left * kSize + 15) & ~15;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int byte = (i * (THREADS / 64) + wave) * 1024 + lane * 16, row = byte / kLine;
                const int piece = (byte % kLine / 16) ^ f(row);
                at[i] = piece * 16 < width ? row * (int)ld + piece * 16 : (int)0x80000000;
            }
            const int g = lane >> 4, r = lane & 15;
            static_assert(kSize == 2 || !kEach, "whole powers of two in fp32");
#pragma unroll
            for (int i = 0; i < (kEach ? F : 1); ++i) {
                if (kSize == 4) from[i] = 4 * g * kLine + (((mine + r) / 4 ^ f(4 * g)) * 16) + (r & 3) * 4;
                else from[i] = (8 * g + (r >> 2)) * kLine + ((mine / 8 + 2 * i + ((r & 3) >> 1)) ^ f(8 * g + (r >> 2))) * 16 + (r & 1) * 8;
            }
        } else {
            base = p + first * ld;
            k = (k_ * kSize + 15) & ~15;
            bytes = (int)((left - 1) * ld) + k;
            part = k % kRowBytes ? stages - 1 : -1;
            piece_at = ((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) at[i] = min((i * (THREADS / 64) + wave) * 8 + (lane >> 3), left - 1) * (int)ld + piece_at;
            from[0] = (mine + (lane & 15)) * kRowBytes + ((lane >> 4) ^ (lane & 7)) * 16;
        }
    }

    // Stages past the end are asked for like any other, from a buffer of no bytes: zeros, and no traffic.  What lies beyond a row's
    // end, or beyond the last row of k, is beyond the buffer too.
    __device__ __forceinline__ void load(int stage, lds_char *to)
    {
        typedef __attribute__((address_space(3))) void lds_void;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const char *p = base;
        int size, k_at = 0;
        if (COLS) {
            const int rows = min(k - stage * kDepth, kDepth);
            p += (int64_t)min(stage, stages - 1) * kDepth * ld;
            size = rows > 0 ? (int)((rows - 1) * ld) + width : 0;
        } else {
            k_at = stage * kRowBytes;
            size = stage < stages ? bytes : 0;
            if (stage == part) {
                const int off = k_at + piece_at < k ? 0 : (int)0x80000000;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) at[i] |= off;
            }
        }
        const auto buffer = __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, size, 0x00027000);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (lds_void *)(to + (i * (THREADS / 64) + wave) * 1024), 16, at[i], k_at, 0, 0);
    }

    __device__ __forceinline__ void read(const lds_char *stage, int half, piece (&to)[F]) const
    {
#pragma unroll
        for (int i = 0; i < F; ++i) {
            if constexpr (!COLS) {
                typedef const __attribute__((address_space(3))) piece lds_piece;
                to[i] = *(lds_piece *)(stage + (from[0] ^ (half * 64)) + i * 16 * kRowBytes);
            } else if constexpr (kSize == 4) {
                typedef const __attribute__((address_space(3))) float lds_float;
#pragma unroll
                for (int q = 0; q < 4; ++q) to[i][q] = *(lds_float *)(stage + (from[0] ^ (i * 64)) + (half * 16 + q) * kLine);
            } else {
                const lds_char *first = stage + (kEach ? from[kEach ? i : 0] : from[0] ^ (i * 32)) + half * 32 * kLine;
                const s16x4 low = read_turned((lds_s16x4 *)first), high = read_turned((lds_s16x4 *)(first + 4 * kLine));
                to[i] = __builtin_bit_cast(piece, (s16x8)__builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        }
    }
};

// The columns of an operand that is kept in 8 bits: its codes come into registers, up to 16 neighbours of one k a load, a stage ahead of the one that they are written to LDS for as elements, where
// the other operand's loads would put theirs.  Each code is turned once a workgroup: 32 a thread and stage in tiles of 256 x 256 beside 64 products (2 operations a code of i8, half a one of e4m3, where
// the hardware scales and turns two at a time).
template <class T, int B_, int F, int THREADS, int FORM>
struct KeptSide {
    typedef Side<T, B_, F, THREADS, true> Columns;
    typedef typename T::piece piece;
    static constexpr int kSize = Columns::kSize, kDepth = Columns::kDepth, kLine = Columns::kLine, kReads = Columns::kReads;
    static constexpr int kCodes = B_ * kDepth / THREADS, kWide = kCodes < 16 ? kCodes : 16, kParts = kCodes / kWide, kAcross = B_ / kWide;
    static constexpr int kLoads = 2 * kParts;                     // codes, and their scale
    static_assert(kParts * kWide * THREADS == B_ * kDepth && kWide >= 8 && kAcross * kWide == B_, "whole loads");
    static_assert(kParts == 1 || THREADS / kAcross % 16 == 0, "parts' rows are permuted alike");
    static constexpr int kDown = THREADS / kAcross;               // rows between a thread's parts
    const char *base;
    const uint8_t *scale_base;
    int64_t ld;
    int k, stages, width;
    Columns columns;                    // (for its reads)
    int at, scale_at, to, turn;         // of the first part: in memory, in LDS; the first of its pieces (the others' last bits differ)
    struct Codes {
        uint32_t words[kParts][kWide / 4];
        uint8_t bytes[kParts];
    } codes;

    __device__ __forceinline__ KeptSide(const Operands &o, int first, int mine) : columns(o.a, o.lda, 0, 0, 0, mine)
    {
        ld = o.lda;
        k = o.k;
        stages = (k + kDepth - 1) / kDepth;
        base = o.a + first;
        scale_base = o.scales + first / kKeptGroup;
        width = min((int)ld - first, B_);
        const int row = threadIdx.x / kAcross, c = threadIdx.x % kAcross * kWide;
        at = c < width ? row * (int)ld + c : (int)0x80000000;
        scale_at = c < width ? row * (int)(ld / kKeptGroup) + c / kKeptGroup : (int)0x80000000;
        to = row * kLine;
        turn = (c * kSize / 16) ^ Columns::f(row);
        fetch(0);
    }

    // Parts `first` to `last` of a stage's codes into registers.
    __device__ __forceinline__ void fetch(int stage, int first = 0, int last = kParts)
    {
        // (of no rows, buffers of no bytes)
        const int rows = __builtin_amdgcn_readfirstlane(max(min(k - stage * kDepth, kDepth), 0)), ld_scales = (int)(ld / kKeptGroup);
        const int64_t row = (int64_t)min(stage, stages) * kDepth;
        const auto buffer = __builtin_amdgcn_make_buffer_rsrc((void *)(base + row * ld), 0, __builtin_amdgcn_readfirstlane(max(rows * (int)ld - ((int)ld - width), 0)), 0x00027000);
        const auto scales = __builtin_amdgcn_make_buffer_rsrc((void *)(scale_base + row * ld_scales), 0, __builtin_amdgcn_readfirstlane(max(rows * ld_scales - (ld_scales - width / kKeptGroup), 0)), 0x00027000);
#pragma unroll
        for (int i = first; i < last; ++i) {
            if constexpr (kWide == 16) {
                const auto v = __builtin_amdgcn_raw_buffer_load_b128(buffer, at + i * kDown * (int)ld, 0, 0);
#pragma unroll
                for (int q = 0; q < 4; ++q) codes.words[i][q] = v[q];
            } else {
                const auto v = __builtin_amdgcn_raw_buffer_load_b64(buffer, at + i * kDown * (int)ld, 0, 0);
                codes.words[i][0] = v[0];
                codes.words[i][1] = v[1];
            }
            codes.bytes[i] = __builtin_amdgcn_raw_buffer_load_b8(scales, scale_at + i * kDown * ld_scales, 0, 0);
        }
    }

    // Eight codes as elements of 16 bits, or four as those of 32.
    static __device__ __forceinline__ piece turned(const uint32_t *words, float scale)
    {
        if constexpr (kSize == 4) {
            const f32x8 v = decode8(FORM, u32x2{words[0], 0u}, scale);
            return f32x4{v[0], v[1], v[2], v[3]};
        } else if constexpr (FORM == PX_KEPT_I8) {
            typedef typename T::type vec __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(piece, __builtin_convertvector(decode8(FORM, u32x2{words[0], words[1]}, scale), vec));
        } else {
            uint32_t out[4];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                if constexpr (std::is_same<T, Bf16>::value) {
                    out[2 * q] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)words[q], scale, false));
                    out[2 * q + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)words[q], scale, true));
                } else {
                    out[2 * q] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)words[q], scale, false));
                    out[2 * q + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)words[q], scale, true));
                }
            }
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
            return __builtin_bit_cast(piece, u32x4{out[0], out[1], out[2], out[3]});
        }
    }

    // The first part alone.
    __device__ __forceinline__ Codes first() const
    {
        Codes c;
#pragma unroll
        for (int q = 0; q < kWide / 4; ++q) c.words[0][q] = codes.words[0][q];
        c.bytes[0] = codes.bytes[0];
        return c;
    }

    // Codes into LDS.
    __device__ __forceinline__ void put(const Codes &from, lds_char *into, int first = 0, int last = kParts) const
    {
        typedef __attribute__((address_space(3))) piece lds_piece;
        constexpr int kWords = kSize == 4 ? 1 : 2, kPieces = kWide / (4 * kWords);
#pragma unroll
        for (int i = first; i < last; ++i) {
            const bool none = FORM == PX_KEPT_E4M3 && from.bytes[i] == 255;
            const float scale = kept_scale(from.bytes[i]);
            uint32_t words[kWide / 4];
#pragma unroll
            for (int q = 0; q < kWide / 4; ++q) words[q] = none ? 0x7f7f7f7fu : from.words[i][q];          // (NaN)
#pragma unroll
            for (int q = 0; q < kPieces; ++q) *(lds_piece *)(into + to + i * kDown * kLine + (turn ^ q) * 16) = turned(words + q * kWords, scale);
        }
    }

    // What has been fetched, which is the stage's, into LDS; the next stage is fetched.
    __device__ __forceinline__ void load(int stage, lds_char *into)
    {
        put(codes, into);
        fetch(stage + 1);
    }

    __device__ __forceinline__ void read(const lds_char *stage, int half, piece (&into)[F]) const { columns.read(stage, half, into); }
};

template <class S, bool SPLIT>
__device__ __forceinline__ void form_tile(const Operands &o, Tile t, char *lds_, f32x4 (&acc)[S::FM][S::FN])
{
    typedef typename S::element T;
    typedef typename T::piece piece;
    lds_char *const lds = (lds_char *)lds_;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr bool kKept = S::KEPT != PX_KEPT_NONE;
    static_assert(!kKept || (S::COLS_A && S::kStages == 2), "kept operands are columns, a stage ahead in registers");
    typedef std::conditional_t<kKept, KeptSide<T, S::BM, S::FM, S::kThreads, kKept ? S::KEPT : PX_KEPT_I8>, Side<T, S::BM, S::FM, S::kThreads, S::COLS_A>> SideA;
    typedef Side<T, S::BN, S::FN, S::kThreads, S::COLS_B> SideB;
    SideA side_a = [&] {
        if constexpr (kKept) return SideA(o, t.m * S::BM, wave / S::WN * S::TM);
        else return SideA(o.a, o.lda, t.m * S::BM, o.m, o.k, wave / S::WN * S::TM);
    }();
    SideB side_b(o.b, o.ldb, t.n * S::BN, o.n, o.k, wave % S::WN * S::TN);
    const int stages = side_a.stages;
    constexpr int kBytesA = S::BM * kRowBytes;
    auto load = [&](int stage, int at) {
        lds_char *to = lds + at * S::kStage;
        side_a.load(stage, to);
        side_b.load(stage, to + kBytesA);
    };
    auto read = [&](int at, int half, piece (&a)[S::FM], piece (&b)[S::FN]) {
        const lds_char *from = lds + at * S::kStage;
        side_b.read(from + kBytesA, half, b);
        side_a.read(from, half, a);
    };
    auto multiply_all = [&](const piece (&a)[S::FM], const piece (&b)[S::FN]) {
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j) acc[i][j] = multiply(a[i], b[j], acc[i][j]);
    };
    constexpr int kLoads = SideA::kLoads + SideB::kLoads, kAhead = (S::kStages - 2) * kLoads;
    static_assert(kAhead < 64, "counted by the hardware");
    auto wait = [](auto ahead) {
        // all but `ahead` of this wavefront's loads have arrived and what it read is in registers; after the barrier, everybody's
        constexpr int n = decltype(ahead)::value;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);         // (nothing is moved across)
        __builtin_amdgcn_s_waitcnt((n & 15) | 0x70 | n >> 4 << 14);        // vmcnt(n) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };

#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (stages == 0) return;
    // Half a stage ahead: while one half is multiplied, the other is on its way from LDS to registers; the barrier stands between the
    // halves, when the whole stage has been read: the loads of the stage kStages later go where it was.
    constexpr int kReads = SideA::kReads + SideB::kReads, kProducts = S::FM * S::FN * (SideA::kSize == 4 ? 4 : 1);
    constexpr int kPerRead = kProducts / (kReads + 4) > 0 ? kProducts / (kReads + 4) : 1, kPerLoad = kPerRead;
    constexpr int kValu = 0x002, kMatrix = 0x008, kVector = 0x010, kLds = 0x100;         // the scheduler's groups of instructions
    piece a0[S::FM], b0[S::FN], a1[S::FM], b1[S::FN];
    typedef std::integral_constant<int, kAhead> some;
    typedef std::integral_constant<int, 0> all;
#pragma unroll
    for (int s = 0; s < S::kStages - 1; ++s) load(s, s);
    wait(some());
    // Codes of i8 in two parts (e4m3, of which less is to turn, gains nothing): one is turned in each half of a stage, so that the matrix units wait for neither.  A stage's first part goes into LDS in the half after which its place is free, the
    // second in the half before the stage is read, and each is fetched when its place in registers is free, a stage ahead.  (16384 x 4096 x 16384 from i8 1925 us, with both in one half 2035, in turn on one card.)
    constexpr bool kHalves = [] {
        if constexpr (kKept) return SideA::kParts == 2 && S::KEPT == PX_KEPT_I8 && !SPLIT;
        else return false;
    }();
    if constexpr (kHalves) {
        side_b.load(1, lds + S::kStage + kBytesA);
        side_a.put(side_a.codes, lds + S::kStage, 0, 1);
        side_a.fetch(2, 0, 1);
    } else {
        load(S::kStages - 1, S::kStages - 1);
    }
    read(0, 0, a0, b0);
    int at = 0;
    if constexpr (SPLIT) {
        for (int s = 0; s < stages; ++s) {
            read(at, 1, a1, b1);
            wait(some());
            load(s + S::kStages, at);
            at = at + 1 == S::kStages ? 0 : at + 1;
            Split b[S::FN], a = split(a0[0], a1[0]);
#pragma unroll
            for (int j = 0; j < S::FN; ++j) b[j] = split(b0[j], b1[j]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                // (the next rows' split between the products of these)
                const Split next = i + 1 < S::FM ? split(a0[i + 1 < S::FM ? i + 1 : 0], a1[i + 1 < S::FM ? i + 1 : 0]) : a;
                constexpr int kOf[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};        // the small ones first
#pragma unroll
                for (int k = 0; k < 6; ++k)
                    if (!kKept || kOf[k][0] == 0)           // (kept elements are bfloat16 numbers: their other parts are 0)
#pragma unroll
                    for (int j = 0; j < S::FN; ++j) acc[i][j] = multiply(a.p[kOf[k][0]], b[j].p[kOf[k][1]], acc[i][j]);
                a = next;
                constexpr int kSplit = 48, kEach = (kSplit + 6 * S::FN - 1) / (6 * S::FN);
#pragma unroll
                for (int k = 0; k < 6 * S::FN; ++k) {
                    __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 2);
                    __builtin_amdgcn_sched_group_barrier(kValu, kEach, 2);
                }
            }
            read(at, 0, a0, b0);
        }
        wait(all());
        return;
    }
    // (All but two: the second part's codes and scale are fetched in the half before the wait and go on. The first part's are fetched in the half after it, where the compiler may put them before or among the other operand's
    // loads, which the wait is for: they are waited for too, as nothing says that they are the last.)
    typedef std::integral_constant<int, kHalves ? 2 : kAhead> ready;
    for (int s = 0; s < stages; ++s) {
        read(at, 1, a1, b1);
        if constexpr (kHalves) {
            side_a.put(side_a.codes, lds + (at ^ 1) * S::kStage, 1, 2);
            side_a.fetch(s + 2, 1, 2);
        }
        multiply_all(a0, b0);
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            __builtin_amdgcn_sched_group_barrier(kLds, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kMatrix, kPerRead, 0);
            if constexpr (kHalves) __builtin_amdgcn_sched_group_barrier(kValu, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMatrix, kProducts, 0);
        wait(ready());
        if constexpr (kHalves) {
            // (LDS is read before it is written: the codes are turned among the products)
            lds_char *const to = lds + at * S::kStage;
            side_b.load(s + 2, to + kBytesA);
            const auto codes = side_a.first();
            side_a.fetch(s + 3, 0, 1);
            at ^= 1;
            read(at, 0, a0, b0);
            side_a.put(codes, to, 0, 1);
        } else if constexpr (kKept) {
            lds_char *const to = lds + at * S::kStage;
            side_b.load(s + S::kStages, to + kBytesA);
            const auto codes = side_a.codes;
            side_a.fetch(s + S::kStages + 1);
            at ^= 1;
            read(at, 0, a0, b0);
            side_a.put(codes, to);
        } else {
            load(s + S::kStages, at);
            at = at + 1 == S::kStages ? 0 : at + 1;
            read(at, 0, a0, b0);
        }
        multiply_all(a1, b1);
        // (what turns kept codes, between the products too)
        constexpr int kTurn = kHalves ? 2 : 3, kIssued = kHalves ? SideB::kLoads + 2 : kLoads;
#pragma unroll
        for (int i = 0; i < kIssued; ++i) {
            __builtin_amdgcn_sched_group_barrier(kVector, 1, 1);
            __builtin_amdgcn_sched_group_barrier(kMatrix, kPerLoad, 1);
            if constexpr (kKept) __builtin_amdgcn_sched_group_barrier(kValu, kTurn, 1);
        }
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            __builtin_amdgcn_sched_group_barrier(kLds, 1, 1);
            __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 1);
            if constexpr (kKept) __builtin_amdgcn_sched_group_barrier(kValu, kTurn, 1);
        }
        __builtin_amdgcn_sched_group_barrier(kMatrix, kProducts, 1);
    }
    // the loads of stages past the end write zeros: nobody else's data may be there before they have
    wait(all());
}

// In fp32 by the split, whose parts of an infinite element are inf - inf: a tile in which something is not finite is formed again
// without it, and is what the formula says.
template <class S>
__device__ __forceinline__ void tile_product(const Operands &o, Tile t, char *lds, f32x4 (&acc)[S::FM][S::FN])
{
    constexpr bool kSplit = std::is_same<typename S::element, F32>::value && S::FN >= 4;
    form_tile<S, kSplit>(o, t, lds, acc);
    if constexpr (kSplit) {
        float sum = 0.f;                   // (0 times each: 0, or NaN)
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum = fmaf(acc[i][j][r], 0.f, sum);
        volatile __attribute__((address_space(3))) int *const bad = (volatile __attribute__((address_space(3))) int *)(lds_char *)lds;
        if (threadIdx.x == 0) *bad = 0;
        __syncthreads();
        if (!(sum == 0.f)) *bad = 1;
        __syncthreads();
        const bool again = *bad != 0;
        __syncthreads();
        if (again) form_tile<S, false>(o, t, lds, acc);
    }
}

// Four values in the lane's own row n, as stored: contiguous in m.
template <class T>
__device__ __forceinline__ void store4(typename T::type *to, f32x4 v)
{
    typedef typename T::type vec __attribute__((ext_vector_type(4)));
    *(vec *)to = __builtin_convertvector(v, vec);
}

// Of 16 bits, two neighbouring tiles' values as eight contiguous in m: the sixteen lanes of rows 4 .. 7 (12 .. 15) of the first tile change places with
// those of rows 0 .. 3 (8 .. 11) of the second.  The lane's values are then of tile first + `tile`, rows `row` .. row + 7, and a row's 64 bytes go out in one store
// where two would write 32 each.
struct Pair {
    int tile, row;
    __device__ __forceinline__ Pair() : tile(threadIdx.x >> 4 & 1), row((threadIdx.x >> 5 & 1) * 8) {}
};
template <class T>
__device__ __forceinline__ typename T::piece paired(f32x4 first, f32x4 second)
{
    typedef typename T::type vec __attribute__((ext_vector_type(4)));
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_convertvector(first, vec)), b = __builtin_bit_cast(u32x2, __builtin_convertvector(second, vec));
    const auto low = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), high = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return __builtin_bit_cast(typename T::piece, u32x4{low[0], high[0], low[1], high[1]});
}

// The same before rounding.
__device__ __forceinline__ void paired32(f32x4 first, f32x4 second, float (&to)[8])
{
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(first[r]), __float_as_uint(second[r]), false, false);
        to[r] = __uint_as_float(both[0]);
        to[r + 4] = __uint_as_float(both[1]);
    }
}

// Neighbouring values into a row of which `left` elements remain, added to what it holds if `add`; whole: such groups are aligned.
template <class T, int COUNT>
__device__ __forceinline__ void put(typename T::type *to, const float (&v)[COUNT], int left, bool whole, bool add)
{
    typedef typename T::type type;
    typedef type vec __attribute__((ext_vector_type(COUNT)));
    if (whole && left >= COUNT) {
        vec old = {}, t;
        if (add) old = *(const vec *)to;
#pragma unroll
        for (int r = 0; r < COUNT; ++r) t[r] = (type)(add ? v[r] + (float)old[r] : v[r]);
        *(vec *)to = t;
    } else {
#pragma unroll
        for (int r = 0; r < COUNT; ++r)
            if (r < left) to[r] = (type)(add ? v[r] + (float)to[r] : v[r]);
    }
}

#endif

}  // namespace px
