// Eight neighbouring elements of a row, loaded and stored as whole groups of 16 bytes (two in fp32) at any alignment of the element:
// rows may begin anywhere, and of odd lengths they do.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/pollux.h"

namespace px {

constexpr int kVec = 8;

template <class E>
struct Eight {
    typedef E type __attribute__((ext_vector_type(8)));
};

#ifdef __HIP_DEVICE_COMPILE__

typedef uint32_t words __attribute__((ext_vector_type(4)));
typedef words __attribute__((aligned(2), may_alias)) at_any;

// The first `left` of the eight are the row's; what is beyond is read as 0 and not written.
template <class E>
__device__ __forceinline__ typename Eight<E>::type load8(const E *from, int64_t left)
{
    typedef typename Eight<E>::type vec;
    vec v;
    if (left >= kVec) {
        if constexpr (sizeof(E) == 4) {
            const words a = *(const at_any *)from, b = *(const at_any *)(from + 4);
            v = __builtin_bit_cast(vec, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            v = __builtin_bit_cast(vec, *(const at_any *)from);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = i < left ? from[i] : (E)0.f;
    }
    return v;
}

template <class E>
__device__ __forceinline__ void store8(E *to, int64_t left, typename Eight<E>::type v)
{
    if (left >= kVec) {
        if constexpr (sizeof(E) == 4) {
            typedef E half __attribute__((ext_vector_type(4)));
            const half a = __builtin_shufflevector(v, v, 0, 1, 2, 3), b = __builtin_shufflevector(v, v, 4, 5, 6, 7);
            *(at_any *)to = __builtin_bit_cast(words, a);
            *(at_any *)(to + 4) = __builtin_bit_cast(words, b);
        } else {
            *(at_any *)to = __builtin_bit_cast(words, v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < left) to[i] = v[i];
    }
}

typedef float f32x8 __attribute__((ext_vector_type(8)));

template <class E>
__device__ __forceinline__ f32x8 load8f(const E *from, int64_t left)
{
    return __builtin_convertvector(load8(from, left), f32x8);
}
template <class E>
__device__ __forceinline__ void store8f(E *to, int64_t left, f32x8 v)
{
    store8(to, left, __builtin_convertvector(v, typename Eight<E>::type));
}

// Eight parameters of one of the three types, or `none` where there is no array.
__device__ __forceinline__ f32x8 parameters(const void *p, int type, int64_t at, int left, float none)
{
    f32x8 v;
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = none;
    if (!p) return v;
    if (type == PX_TYPE_F32) return load8f((const float *)p + at, left);
    if (type == PX_TYPE_BF16) return load8f((const __bf16 *)p + at, left);
    return load8f((const _Float16 *)p + at, left);
}

#endif

}  // namespace px
