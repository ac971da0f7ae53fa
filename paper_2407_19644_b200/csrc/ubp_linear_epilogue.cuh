// Epilogue of the token-major products: scales, bias, activation, gate, residual.
#ifndef UBP_LINEAR_EPILOGUE_CUH_
#define UBP_LINEAR_EPILOGUE_CUH_

#include "ubp_linear.h"
#include "ubp_types.cuh"

namespace ubp {

// v * sigmoid(u) = v / (1 + e^-u). __expf and the approximate division are within a few units of 2^-22 each, far below the
// 16-bit outputs' 2^-9 (bf16) / 2^-12 (f16) and inside the fp32 output's accumulation error. e^-u overflows to infinity for
// u < -88, where the quotient is -0 or 0, as the exact value rounds to (below 2^-120).
__device__ __forceinline__ float v_sigmoid(float v, float u) { return __fdividef(v, 1.f + __expf(fminf(-u, 80.f))); }

// (the choice outside the loop: with the switch inside an unrolled one, all five activations sit in the path N times over and
// the epilogue of the tensor-core kernel ran from instruction cache misses, 4 us for 32 x 32 outputs)
template <int N> __device__ __forceinline__ void apply_act(float (&v)[N], int act)
{
    switch (act) {
        case UBP_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = fmaxf(v[i], 0.f);
            break;
        case UBP_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = 0.5f * v[i] * (1.f + erff(v[i] * 0.70710678118654752f));
            break;
        case UBP_ACT_GELU_TANH:   // 0.5 v (1 + tanh(u)) = v sigmoid(2 u), u = sqrt(2 / pi) (v + 0.044715 v^3)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = v_sigmoid(v[i], 1.5957691216057308f * (v[i] + 0.044715f * v[i] * v[i] * v[i]));
            break;
        case UBP_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = v_sigmoid(v[i], v[i]);
            break;
        default: break;
    }
}
__device__ __forceinline__ float apply_act(float v, int act)
{
    float a[1] = {v};
    apply_act<1>(a, act);
    return a[0];
}

// one output element of type ydt at index i of a row-major array
__device__ __forceinline__ void store_elem(void *y, int64_t i, float v, int ydt)
{
    if (ydt == UBP_BF16) static_cast<__nv_bfloat16 *>(y)[i] = __float2bfloat16_rn(v);
    else if (ydt == UBP_F16) static_cast<__half *>(y)[i] = __float2half_rn(v);
    else static_cast<float *>(y)[i] = v;
}
__device__ __forceinline__ float load_elem(const void *p, int64_t i, int dt)
{
    if (dt == UBP_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
    if (dt == UBP_F16) return __half2float(static_cast<const __half *>(p)[i]);
    return static_cast<const float *>(p)[i];
}

}  // namespace ubp
#endif
