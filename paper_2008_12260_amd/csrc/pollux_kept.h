// Rows kept in 8 bits: 32 neighbours of a row share a scale, a power of two, so that scaling is exact and the only rounding is the
// code's own.  A code is a whole number of 7 bits and a sign (PX_KEPT_I8) or an e4m3 (PX_KEPT_E4M3); both are exact in bfloat16 and, but for its range, in fp16.
//
//   scale = the least 2^e with which the group's largest element has a code (at most 127, or 448);  code = round(v / scale), ties to even
//
// The scale's byte is e + 127; 255 stands for a group in which something is not finite: all of it is restored as NaN.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/pollux.h"
#include "pollux_rows.h"

namespace px {

constexpr int kKeptGroup = 32;
constexpr int64_t kept_width(int64_t d) { return (d + kKeptGroup - 1) / kKeptGroup * kKeptGroup; }      // bytes of a row's codes

#ifdef __HIP_DEVICE_COMPILE__

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// The value of a register in the neighbouring lanes l ^ 1 and l ^ 2.
template <int CTRL>
__device__ __forceinline__ uint32_t of_lane(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E;             // quad_perm [1,0,3,2] and [2,3,0,1]

__device__ __forceinline__ float kept_scale(uint32_t byte)
{
    // (2^-127 is below the normal numbers; a NaN for 255)
    return __uint_as_float(max(byte << 23, 0x00400000u) | (byte + 1 & 256u) << 14);
}

// The scale's byte from the bits of the group's largest size: one more than its exponent says where the fraction is from 127/128 on, or over 3/4 (round(127.5) is 128;
// 448 = 1.75 * 2^8).  Bits of infinities and NaNs are larger than all others.
__device__ __forceinline__ uint32_t kept_byte(int form, uint32_t size)
{
    const int e = (int)((size + (form == PX_KEPT_I8 ? 0x10000u : 0x1fffffu)) >> 23) - (form == PX_KEPT_I8 ? 6 : 8);
    return size >= 0x7f800000u ? 255u : (uint32_t)max(e, 0);
}

// Codes of eight neighbours, whose group's byte is given; what is not finite has codes of 0.
__device__ __forceinline__ u32x2 encode8(int form, f32x8 v, uint32_t byte)
{
    const float inverse = __uint_as_float((254u - min(byte, 253u)) << 23);
    u32x2 out;
    if (form == PX_KEPT_I8) {
        // (the sum's last bits are the rounded quotient)
        uint32_t t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = __float_as_uint(fmaf(v[i], inverse, 12582912.f));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t low = __builtin_amdgcn_perm(t[4 * k + 1], t[4 * k], 0x0c0c0400u), high = __builtin_amdgcn_perm(t[4 * k + 3], t[4 * k + 2], 0x04000c0cu);
            out[k] = low | high;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * k] * inverse, v[4 * k + 1] * inverse, 0, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * k + 2] * inverse, v[4 * k + 3] * inverse, w, true);
            out[k] = (uint32_t)w;
        }
    }
    if (byte == 255) out = u32x2{0u, 0u};
    return out;
}

__device__ __forceinline__ f32x8 decode8(int form, u32x2 codes, float scale)
{
    f32x8 v;
    if (form == PX_KEPT_I8) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = (float)((int)(codes[i >> 2] << (24 - 8 * (i & 3))) >> 24) * scale;
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const auto low = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[k], false), high = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[k], true);
            v[4 * k] = low[0] * scale;
            v[4 * k + 1] = low[1] * scale;
            v[4 * k + 2] = high[0] * scale;
            v[4 * k + 3] = high[1] * scale;
        }
    }
    return v;
}

// Bits of the largest size among four neighbouring lanes' eight values each: a group's.
__device__ __forceinline__ uint32_t group_size(f32x8 v)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    m = max(m, of_lane<kXor1>(m));
    return max(m, of_lane<kXor2>(m));
}

// The same of elements as they came from memory: of 16 bits two at a time, as whole numbers, whose order their sizes' is.
template <class V>
__device__ __forceinline__ uint32_t loaded_size(V v)
{
    if constexpr (sizeof(V) == 32) {
        return group_size(__builtin_convertvector(v, f32x8));
    } else {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        const u32x4 w = __builtin_bit_cast(u32x4, v) & 0x7fff7fffu;
        auto larger = [](uint32_t a, uint32_t b) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b))); };
        uint32_t m = larger(larger(w[0], w[1]), larger(w[2], w[3]));
        m = larger(m, of_lane<kXor1>(m));
        m = larger(m, of_lane<kXor2>(m));
        const uint16_t bits = (uint16_t)max(m & 0xffffu, m >> 16);
        if constexpr (std::is_same<V, typename Eight<__bf16>::type>::value) return (uint32_t)bits << 16;
        else return __float_as_uint((float)__builtin_bit_cast(_Float16, bits));
    }
}

// Four neighbouring lanes keep a group, eight values each: at `codes` the lane's eight, at `scale` the group's byte (by the first of them).
__device__ __forceinline__ void keep8_of(int form, f32x8 v, uint32_t size, uint8_t *codes, uint8_t *scale, bool there)
{
    const uint32_t byte = kept_byte(form, size);
    const u32x2 out = encode8(form, v, byte);
    if (!there) return;
    *(u32x2 *)codes = out;
    if ((threadIdx.x & 3) == 0) *scale = (uint8_t)byte;
}
__device__ __forceinline__ void keep8(int form, f32x8 v, uint8_t *codes, uint8_t *scale, bool there) { keep8_of(form, v, group_size(v), codes, scale, there); }
template <class V>
__device__ __forceinline__ void keep_loaded(int form, V v, uint8_t *codes, uint8_t *scale)
{
    keep8_of(form, __builtin_convertvector(v, f32x8), loaded_size(v), codes, scale, true);
}

#endif

}  // namespace px
