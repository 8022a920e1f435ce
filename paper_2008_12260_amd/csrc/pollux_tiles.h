// Matrix products on the matrix units, shared by the loss and the orthogonalised update: one tile of
//   C[m, n] = sum_k A[m, k] B[n, k]
// per workgroup, both operands row-major with k contiguous, sums in fp32.
//
// Rows of both operands come into LDS 128 bytes of k at a time (64 elements of 16 bits, 32 of 32 bits), by loads that write
// LDS directly and are in flight while the stage before is multiplied: two stages, one barrier each.  A row's eight 16-byte
// pieces lie in LDS in the order piece ^ (row & 7): sixteen rows' pieces read by a wavefront then touch every bank once.
// The address a lane loads from is permuted instead of the one it writes to, which the hardware makes the lane's number.
// Each lane holds column n = lane & 15 of a 16 x 16 tile and four consecutive rows m: what runs over m (the vocabulary) is
// reduced mostly in registers, and four elements contiguous in m go out in one store.
// 8192 x 8192 x 4096 in bfloat16, tiles of 256 x 256: 1.27 PFLOP/s, where a large library product reaches 1.28 to 1.6.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

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

struct Operands {
    const char *a, *b;
    int64_t lda, ldb;       // bytes from row to row, multiples of 16, as are the pointers
    int rows_a, rows_b;
    int k_bytes;            // a multiple of 16; 0 gives a tile of zeros
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

template <class T, int BM_, int BN_, int WM_, int WN_>
struct TileShape {
    typedef T element;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int kThreads = WM * WN * 64, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    static constexpr int kStage = (BM + BN) * kRowBytes, kLds = 2 * kStage;
    static constexpr int kLoadsA = BM * kRowBytes / (kThreads * 16), kLoadsB = BN * kRowBytes / (kThreads * 16);
    static_assert(kLoadsA * kThreads * 16 == BM * kRowBytes && kLoadsB * kThreads * 16 == BN * kRowBytes, "whole loads");
};

constexpr int kShapes = 4;
struct ShapeOf {
    int bm, bn, per_cu;         // tile, workgroups a compute unit holds
    float rate;                 // of the matrix units' while it runs, relative
};
constexpr ShapeOf kShape[kShapes] = {{256, 256, 1, 1.0f}, {128, 128, 2, 0.75f}, {64, 64, 4, 0.45f}, {128, 16, 4, 0.15f}};

// The shape whose rounds over the compute units take least: ceil(tiles / (256 x per_cu)) rounds of per_cu tiles.
inline int shape_for(int64_t m, int64_t n, int64_t slices, bool f32)
{
    int best = 0;
    double least = 1e300;
    for (int s = 0; s < kShapes; ++s) {
        const ShapeOf &h = kShape[s];
        const double tiles = (double)((m + h.bm - 1) / h.bm) * ((n + h.bn - 1) / h.bn) * slices;
        const double cost = ceil(tiles / (256.0 * h.per_cu)) * h.per_cu * h.bm * h.bn / (f32 ? 1.0 : h.rate);
        if (cost < least) least = cost, best = s;
    }
    return best;
}

template <class T>
using Shape0 = TileShape<T, 256, 256, 2, 4>;
template <class T>
using Shape1 = TileShape<T, 128, 128, 2, 2>;
template <class T>
using Shape2 = TileShape<T, 64, 64, 2, 2>;
template <class T>
using Shape3 = TileShape<T, 128, 16, 2, 1>;

#ifdef __HIP_DEVICE_COMPILE__

__device__ __forceinline__ f32x4 multiply(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
// fp32: four products of k = 4; which four of a row's sixteen k each takes is the same for both operands
__device__ __forceinline__ f32x4 multiply(f32x4 a, f32x4 b, f32x4 c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
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

template <class S>
__device__ __forceinline__ void tile_product(const Operands &o, Tile t, char *lds, f32x4 (&acc)[S::FM][S::FN])
{
    typedef __attribute__((address_space(3))) void lds_void;
    typedef typename S::element::piece piece;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows_a = min(o.rows_a - t.m * S::BM, S::BM), rows_b = min(o.rows_b - t.n * S::BN, S::BN);
    // (rows - 1) * ld + k_bytes stays below 2^31: the entry points' limits see to it.  A load beyond the buffer gives zeros.
    const char *const base_a = o.a + (int64_t)t.m * S::BM * o.lda, *const base_b = o.b + (int64_t)t.n * S::BN * o.ldb;
    const int bytes_a = (int)((rows_a - 1) * o.lda) + o.k_bytes, bytes_b = (int)((rows_b - 1) * o.ldb) + o.k_bytes;
    const int piece_at = ((lane & 7) ^ (lane >> 3)) * 16;
    int at_a[S::kLoadsA], at_b[S::kLoadsB];
#pragma unroll
    for (int i = 0; i < S::kLoadsA; ++i) at_a[i] = min((i * (S::kThreads / 64) + wave) * 8 + (lane >> 3), rows_a - 1) * (int)o.lda + piece_at;
#pragma unroll
    for (int i = 0; i < S::kLoadsB; ++i) at_b[i] = min((i * (S::kThreads / 64) + wave) * 8 + (lane >> 3), rows_b - 1) * (int)o.ldb + piece_at;

    const int stages = (o.k_bytes + kRowBytes - 1) / kRowBytes, part = o.k_bytes % kRowBytes ? stages - 1 : -1;
    // Stages past the end are asked for like any other, from a buffer of no bytes: zeros, and no traffic.  Of a last stage that is
    // not whole, a row's pieces beyond its end are taken from beyond the buffer.
    auto load = [&](int stage) {
        const int k = stage * kRowBytes;
        char *to = lds + (stage & 1) * S::kStage + wave * 1024;
        if (stage == part) {
            const int off = k + piece_at < o.k_bytes ? 0 : (int)0x80000000;
#pragma unroll
            for (int i = 0; i < S::kLoadsA; ++i) at_a[i] |= off;
#pragma unroll
            for (int i = 0; i < S::kLoadsB; ++i) at_b[i] |= off;
        }
        const auto from_a = __builtin_amdgcn_make_buffer_rsrc((void *)base_a, 0, stage < stages ? bytes_a : 0, 0x00027000);
        const auto from_b = __builtin_amdgcn_make_buffer_rsrc((void *)base_b, 0, stage < stages ? bytes_b : 0, 0x00027000);
#pragma unroll
        for (int i = 0; i < S::kLoadsA; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from_a, (lds_void *)(to + i * S::kThreads * 16), 16, at_a[i], k, 0, 0);
#pragma unroll
        for (int i = 0; i < S::kLoadsB; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from_b, (lds_void *)(to + S::BM * kRowBytes + i * S::kThreads * 16), 16, at_b[i], k, 0, 0);
    };
    const int row_a = (wave / S::WN * S::TM + (lane & 15)) * kRowBytes, row_b = (S::BM + wave % S::WN * S::TN + (lane & 15)) * kRowBytes;
    const int piece_of = ((lane >> 4) ^ (lane & 7)) * 16;
    auto read = [&](int stage, int half, piece (&a)[S::FM], piece (&b)[S::FN]) {
        const char *from = lds + (stage & 1) * S::kStage + (piece_of ^ (half * 64));
#pragma unroll
        for (int j = 0; j < S::FN; ++j) b[j] = *(const piece *)(from + row_b + j * 16 * kRowBytes);
#pragma unroll
        for (int i = 0; i < S::FM; ++i) a[i] = *(const piece *)(from + row_a + i * 16 * kRowBytes);
    };
    auto multiply_all = [&](const piece (&a)[S::FM], const piece (&b)[S::FN]) {
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j) acc[i][j] = multiply(a[i], b[j], acc[i][j]);
    };
    auto wait_for_all = [] {
        // this wavefront's loads have arrived and what it read is in registers; after the barrier, everybody's
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);        // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (stages == 0) return;
    // Half a stage ahead: while one half is multiplied, the other is on its way from LDS to registers; the barrier stands between the
    // halves, when the whole stage has been read: the loads of the stage after next go where it was.
    constexpr int kReads = S::FM + S::FN, kLoads = S::kLoadsA + S::kLoadsB, kProducts = S::FM * S::FN * (sizeof(typename S::element::type) == 4 ? 4 : 1);
    constexpr int kPerRead = kProducts / (kReads + 4) > 0 ? kProducts / (kReads + 4) : 1, kPerLoad = kProducts / (kReads + 4) > 0 ? kProducts / (kReads + 4) : 1;
    constexpr int kMatrix = 0x008, kVector = 0x010, kLds = 0x100;         // the scheduler's groups of instructions
    piece a0[S::FM], b0[S::FN], a1[S::FM], b1[S::FN];
    load(0);
    wait_for_all();
    load(1);
    read(0, 0, a0, b0);
    for (int s = 0; s < stages; ++s) {
        read(s, 1, a1, b1);
        multiply_all(a0, b0);
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            __builtin_amdgcn_sched_group_barrier(kLds, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kMatrix, kPerRead, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMatrix, kProducts, 0);
        wait_for_all();
        load(s + 2);
        read(s + 1, 0, a0, b0);
        multiply_all(a1, b1);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            __builtin_amdgcn_sched_group_barrier(kVector, 1, 1);
            __builtin_amdgcn_sched_group_barrier(kMatrix, kPerLoad, 1);
        }
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            __builtin_amdgcn_sched_group_barrier(kLds, 1, 1);
            __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 1);
        }
        __builtin_amdgcn_sched_group_barrier(kMatrix, kProducts, 1);
    }
    // the loads of stages past the end write zeros: nobody else's data may be there before they have
    wait_for_all();
}

// Four values in the lane's own row n, as stored: contiguous in m.
template <class T>
__device__ __forceinline__ void store4(typename T::type *to, f32x4 v)
{
    typedef typename T::type vec __attribute__((ext_vector_type(4)));
    *(vec *)to = __builtin_convertvector(v, vec);
}

// The 4 x 4 block that four neighbouring lanes (columns n .. n + 3) hold of four rows m each, turned: lane q of the four gets
// row m + q of columns n .. n + 3.
__device__ __forceinline__ f32x4 turned(f32x4 v)
{
    const int q = threadIdx.x & 3;
    auto xor1 = [](float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xf, 0xf, true)); };     // quad_perm [1,0,3,2]
    auto xor2 = [](float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xf, 0xf, true)); };     // [2,3,0,1]
    // swap the off-diagonal elements of 2 x 2 blocks, then the off-diagonal blocks
    const bool odd = q & 1, high = q & 2;
    const float s01 = xor1(odd ? v[0] : v[1]), s23 = xor1(odd ? v[2] : v[3]);
    f32x4 w = {odd ? s01 : v[0], odd ? v[1] : s01, odd ? s23 : v[2], odd ? v[3] : s23};
    const float t0 = xor2(high ? w[0] : w[2]), t1 = xor2(high ? w[1] : w[3]);
    return f32x4{high ? t0 : w[0], high ? t1 : w[1], high ? w[2] : t0, high ? w[3] : t1};
}

#endif

}  // namespace px
