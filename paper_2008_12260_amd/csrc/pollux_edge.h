// What the edge between two blocks and its gradients share: threads of a row, their sums, parameters, normalised rows.
//
// A row is a team's, eight neighbouring elements a thread (sixteen from 8192 on): 4 to 64 lanes of a wavefront up to 512 elements, whole wavefronts, which are then a
// workgroup, beyond.  Weights and gate stay in registers while the team goes through its rows, several at a time, so that a row costs one trip
// to memory and its sums' latency is shared.  Sums of a row: over lanes by moves between registers, over wavefronts through LDS, always in the same order.
#pragma once

#include "pollux_host.h"
#include "pollux_kept.h"
#include "pollux_rows.h"
#include "pollux_train.h"

namespace px {

struct EdgeKernelArgs {
    pollux_edge_dims d;
    EdgeArgs p;
    int team, chunk;
    bool ragged;                // threads of a row have more elements between them than it has
    float *parts, *ends;
};

#ifdef __HIP_DEVICE_COMPILE__

constexpr int kMostWaves = 16;

// v summed over the `team` lanes that a lane belongs to: 4 to 64.
__device__ __forceinline__ float over_lanes(float v, int team)
{
    auto moved = [&](auto ctrl) { return __uint_as_float(of_lane<decltype(ctrl)::value>(__float_as_uint(v))); };
    v += moved(std::integral_constant<int, kXor1>());
    v += moved(std::integral_constant<int, kXor2>());
    if (team >= 8) v += moved(std::integral_constant<int, 0x141>());          // mirrored in eight lanes: the other four
    if (team >= 16) v += moved(std::integral_constant<int, 0x140>());         // in sixteen: the other eight
    if (team >= 32) {
        const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    }
    if (team >= 64) {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    }
    return v;
}

// K sums over the team.  Of several wavefronts, `parity` says which half of the array in LDS is free: it was last read before a barrier that all have passed.
template <int K>
__device__ __forceinline__ void over_team(float (&v)[K], int team, float (*shared)[kMostWaves][8], int &parity)
{
    static_assert(K <= 8, "a row of the array");
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = over_lanes(v[k], min(team, 64));
    if (team <= 64) return;
    float(*const at)[8] = shared[parity];
    parity ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) at[threadIdx.x >> 6][k] = v[k];
    __syncthreads();
    const int waves = team >> 6;
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = at[0][k];
    for (int w = 1; w < waves; ++w)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += at[w][k];
}

// Eight parameters stored as one of the three types.
__device__ __forceinline__ void store_parameters(void *p, int type, int64_t at, int left, f32x8 v)
{
    if (type == PX_TYPE_F32) store8f((float *)p + at, left, v);
    else if (type == PX_TYPE_BF16) store8f((__bf16 *)p + at, left, v);
    else store8f((_Float16 *)p + at, left, v);
}

// Eight elements as they came from memory: of rows (T), or codes and their scale's byte.
template <class T>
struct Loaded {
    static constexpr int kWords = sizeof(T) * 2;
    uint32_t words[kWords];
    __device__ __forceinline__ void rows(const T *from, int left)
    {
        typedef uint32_t whole __attribute__((ext_vector_type(kWords)));
        const whole v = __builtin_bit_cast(whole, load8(from, left));
#pragma unroll
        for (int i = 0; i < kWords; ++i) words[i] = v[i];
    }
    __device__ __forceinline__ void kept(const uint8_t *values, const uint8_t *scales, int64_t at)
    {
        const u32x2 codes = *(const u32x2 *)(values + at);
        words[0] = codes[0];
        words[1] = codes[1];
        words[2] = scales[at / kKeptGroup];
    }
    __device__ __forceinline__ f32x8 of_rows() const
    {
        typedef uint32_t whole __attribute__((ext_vector_type(kWords)));
        whole v;
#pragma unroll
        for (int i = 0; i < kWords; ++i) v[i] = words[i];
        return __builtin_convertvector(__builtin_bit_cast(typename Eight<T>::type, v), f32x8);
    }
    // The normalised rows: kept, or formed again.
    __device__ __forceinline__ f32x8 normalised(int form, float2 stats) const
    {
        return form ? decode8(form, u32x2{words[0], words[1]}, kept_scale(words[2])) : (of_rows() - stats.x) * stats.y;
    }
};
__device__ __forceinline__ f32x8 fma8(f32x8 a, f32x8 b, f32x8 c)
{
#pragma unroll
    for (int i = 0; i < kVec; ++i) c[i] = fmaf(a[i], b[i], c[i]);
    return c;
}

// Sum of eight, and of their squares; what is beyond the row's end counts for nothing.
__device__ __forceinline__ float sum8(f32x8 v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
__device__ __forceinline__ float squares8(f32x8 v)
{
    float s = v[0] * v[0];
#pragma unroll
    for (int i = 1; i < kVec; ++i) s = fmaf(v[i], v[i], s);
    return s;
}
__device__ __forceinline__ f32x8 within(f32x8 v, int left)
{
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = i < left ? v[i] : 0.f;
    return v;
}

#endif

}  // namespace px
