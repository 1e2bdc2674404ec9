// Eight consecutive values of a row in registers: 16-byte loads and stores, widening to fp32 and rounding back.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

namespace gelo {

__device__ __forceinline__ float widen_at(const __nv_bfloat16* e, int j) { return __bfloat162float(e[j]); }
__device__ __forceinline__ float widen_at(const __half* e, int j) { return __half2float(e[j]); }
__device__ __forceinline__ float widen_at(const float* e, int j) { return e[j]; }
__device__ __forceinline__ float widen_at(const uint8_t* e, int j) { return __half2float(__half(__nv_cvt_fp8_to_halfraw(e[j], __NV_E4M3))); }

__device__ __forceinline__ void round_to(float v, float* out) { *out = v; }
__device__ __forceinline__ void round_to(float v, __nv_bfloat16* out) { *out = __float2bfloat16_rn(v); }
__device__ __forceinline__ void round_to(float v, __half* out) { *out = __float2half_rn(v); }

// two values rounded to a 16-bit type, the first in the low half
template <typename T>
__device__ __forceinline__ uint32_t two_of(float a, float b);
template <>
__device__ __forceinline__ uint32_t two_of<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <>
__device__ __forceinline__ uint32_t two_of<__half>(float a, float b)
{
    const __half2 t = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}

template <typename T>
struct Eight {
    uint4 raw[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void store(T* p) const
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = raw[i];
    }
    __device__ __forceinline__ void widen(float (&v)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = widen_at(reinterpret_cast<const T*>(raw), j);
    }
    __device__ __forceinline__ void narrow(const float (&v)[8])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) reinterpret_cast<float*>(raw)[j] = v[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) reinterpret_cast<uint32_t*>(raw)[j] = two_of<T>(v[2 * j], v[2 * j + 1]);
        }
    }
};

// Eight E4M3 codes, nearest-even, saturating at +-448; a NaN stays one
__device__ __forceinline__ uint2 e4m3_codes(const float (&v)[8])
{
    uint32_t c[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; j += 2)
        c[j >> 2] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[j], v[j + 1]), __NV_SATFINITE, __NV_E4M3) << (8 * (j & 3));
    return make_uint2(c[0], c[1]);
}

}  // namespace gelo
