// Element types of the token-major operators (rows of activations with one token each): loads, stores and conversions
// of bf16, f16, f32 and e4m3 values. All arithmetic is done in fp32.
#ifndef UBP_TYPES_CUH_
#define UBP_TYPES_CUH_

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "ubp.h"

namespace ubp {

constexpr float E4M3_MAX = 448.f;
// Smallest scale a row of 8-bit values gets: the smallest normal fp32 number, so that a row of zeros has scale 2^-126 and
// codes 0 instead of a division by zero.
constexpr float ROW_SCALE_MIN = 1.17549435e-38f;

inline int dtype_size(int dt)
{
    switch (dt) {
        case UBP_F32: return 4;
        case UBP_F16: case UBP_BF16: return 2;
        case UBP_E4M3: return 1;
        default: return 0;
    }
}

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// two fp32 values -> two e4m3 codes (round to nearest even, values beyond +-448 become +-448, NaN stays NaN); `lo` in the
// low byte
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ __nv_fp8_storage_t from_f32<__nv_fp8_storage_t>(float v)
{
    return (__nv_fp8_storage_t)(e4m3x2(v, 0.f) & 0xffu);
}

// one 32-bit word of two 16-bit values -> fp32 pair
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&p);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&p);
}
// two e4m3 codes (low 16 bits of w) -> the same two values in f16 (exact: every e4m3 value is an f16 value)
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t w)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
    return r;
}

// eight consecutive elements <-> fp32, in 16-byte accesses (two of them for fp32; 8 bytes for e4m3)
template <typename T> __device__ __forceinline__ void load8(const T *p, float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2<T>(w[i]);
            v[2 * i] = f.x; v[2 * i + 1] = f.y;
        }
    }
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else if constexpr (sizeof(T) == 1) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(e4m3x2(v[0], v[1]) | (e4m3x2(v[2], v[3]) << 16),
                                                   e4m3x2(v[4], v[5]) | (e4m3x2(v[6], v[7]) << 16));
    } else {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
    }
}

// maximum that keeps a NaN (fmaxf drops it)
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

}  // namespace ubp
#endif
