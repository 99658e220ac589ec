// Device helpers of the acoustic-model operators: element types, reductions.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "am.h"

namespace wfd {

using f16 = _Float16;
using bf16 = __bf16;
struct f8 {          // OCP e4m3
    uint8_t bits;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(f16 x) { return static_cast<float>(x); }
__device__ __forceinline__ float to_f32(bf16 x) { return static_cast<float>(x); }
// Reductions over a wave, or over each 8, 16 or 32 lanes of it, without LDS: lanes meet
// by quad and row permutations, then rows of 16 and halves are swapped.  Every lane
// gets the result, always in the same order.
template <int kPattern>
__device__ __forceinline__ int dpp(int v)
{
    return __builtin_amdgcn_update_dpp(v, v, kPattern, 0xF, 0xF, true);
}

template <int kLanes = 64, typename Op>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, Op op)
{
    static_assert(kLanes == 8 || kLanes == 16 || kLanes == 32 || kLanes == 64, "");
    v = op(v, static_cast<uint32_t>(dpp<0xB1>(static_cast<int>(v))));    // lane ^ 1
    v = op(v, static_cast<uint32_t>(dpp<0x4E>(static_cast<int>(v))));    // lane ^ 2
    v = op(v, static_cast<uint32_t>(dpp<0x141>(static_cast<int>(v))));   // mirrored in 8
    if constexpr (kLanes == 8) return v;
    v = op(v, static_cast<uint32_t>(dpp<0x140>(static_cast<int>(v))));   // mirrored in 16
    if constexpr (kLanes == 16) return v;
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = op(r[0], r[1]);
    if constexpr (kLanes == 32) return v;
    const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return op(h[0], h[1]);
}

template <int kLanes = 64>
__device__ __forceinline__ float wave_sum(float v)
{
    return __uint_as_float(wave_reduce<kLanes>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}

__device__ __forceinline__ float wave_max(float v)
{
    return __uint_as_float(wave_reduce(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}

template <int kLanes = 64>
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v)
{
    return wave_reduce<kLanes>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

#define AM_LDS __attribute__((address_space(3)))
#define AM_GLOBAL __attribute__((address_space(1)))

// C consecutive elements of a row, at any address (wide accesses need no
// alignment on this hardware); n of them exist, the others read as `fill`.  The type
// says so by a typedef: in a `using` the compiler drops `aligned` without a word and
// takes the vector's own, and from that it may make a scalar load of an address that
// a wave's threads share, which drops the address's low bits.
template <typename T, int C, int kAlign>
struct ChunkOf {
    typedef T Type __attribute__((ext_vector_type(C), aligned(kAlign)));
    static_assert(alignof(Type) == kAlign, "");
};
template <typename T, int C, int kAlign = sizeof(T)>
using Chunk = typename ChunkOf<T, C, kAlign>::Type;

template <typename T, int C>
__device__ __forceinline__ Chunk<T, C> load_chunk(const T *p, int64_t n, T fill)
{
    if (n >= C) return *(const AM_GLOBAL Chunk<T, C> *)p;
    Chunk<T, C> v;
#pragma unroll
    for (int e = 0; e < C; e++) v[e] = e < n ? ((const AM_GLOBAL T *)p)[e] : fill;
    return v;
}

template <typename T, int C>
__device__ __forceinline__ void load_floats(const T *p, int64_t n, float (&x)[C], float fill = 0.0f)
{
    const Chunk<T, C> v = load_chunk<T, C>(p, n, static_cast<T>(fill));
#pragma unroll
    for (int e = 0; e < C; e++) x[e] = static_cast<float>(v[e]);
}

template <typename T, int C>
__device__ __forceinline__ void store_floats(T *p, int64_t n, const float (&x)[C])
{
    Chunk<T, C> v;
#pragma unroll
    for (int e = 0; e < C; e++) v[e] = static_cast<T>(x[e]);
    if (n >= C) {
        *(AM_GLOBAL Chunk<T, C> *)p = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < C; e++)
        if (e < n) ((AM_GLOBAL T *)p)[e] = v[e];
}

// To e4m3, to nearest, ties to even.  The conversion does not saturate: the
// values are at most 448 but for roundings (and 464 is the first that overflows).
template <int C>
__device__ __forceinline__ void store_floats(f8 *p, int64_t n, const float (&x)[C])
{
    using V = Chunk<uint32_t, C / 4, 1>;
    V v;
#pragma unroll
    for (int h = 0; h < C / 4; h++) {
        const int t = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h], x[4 * h + 1], 0, false);
        v[h] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h + 2], x[4 * h + 3], t, true));
    }
    if (n >= C) {
        *(AM_GLOBAL V *)p = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < C; e++)
        if (e < n) ((AM_GLOBAL uint8_t *)p)[e] = static_cast<uint8_t>(v[e >> 2] >> (e & 3) * 8);
}

// exp for softmax and activations: good to about |x| 2^-24 relative
__device__ __forceinline__ float am_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

}  // namespace wfd
