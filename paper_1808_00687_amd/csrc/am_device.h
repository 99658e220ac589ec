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
__device__ __forceinline__ float to_f32(f8 x) { return __builtin_amdgcn_cvt_f32_fp8(x.bits, 0); }

// float32 to T, to nearest, ties to even
template <typename T>
__device__ __forceinline__ T from_f32(float x)
{
    return static_cast<T>(x);
}

// the conversion does not saturate: a finite value past the range would be NaN
template <>
__device__ __forceinline__ f8 from_f32<f8>(float x)
{
    x = x > kE4m3Max ? kE4m3Max : x < -kE4m3Max ? -kE4m3Max : x;   // a NaN stays one
    return f8{static_cast<uint8_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xFF)};
}

__device__ __forceinline__ float wave_sum(float v)
{
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

__device__ __forceinline__ float wave_max(float v)
{
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v)
{
    for (int o = 32; o; o >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o)));
    return v;
}

}  // namespace wfd
