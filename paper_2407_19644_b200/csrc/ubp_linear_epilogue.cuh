// Epilogue of the token-major products: scales, bias, activation, gate, residual.
#ifndef UBP_LINEAR_EPILOGUE_CUH_
#define UBP_LINEAR_EPILOGUE_CUH_

#include "ubp_linear.h"
#include "ubp_types.cuh"

namespace ubp {

// v * sigmoid(u) = v / (1 + e^-u). __expf and the approximate division are within a few units of 2^-22 each, far below the
// 16-bit outputs' 2^-9 (bf16) / 2^-12 (f16) and inside the fp32 output's accumulation error. e^-u stops at e^88, above 2^126,
// where the division's quotient is defined as 0 for every finite v (the exact value is below 2^-120); unstopped it would be
// infinity, for which no quotient is defined.
__device__ __forceinline__ float v_sigmoid(float v, float u) { return __fdividef(v, 1.f + __expf(fminf(-u, 88.f))); }

// GELU with erf, 0.5 v (1 + erf(v / sqrt 2)) = max(v, 0) - 0.5 |v| erfc(|v| / sqrt 2). erfc(x) = t (a1 + t (a2 + ...)) e^(-x^2),
// t = 1 / (1 + p x): Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26, |error| <= 1.5 10^-7. Half the
// instructions of erff, which were what a tile's epilogue waited for (777 tokens on 1500 x 1003: 15.3 us a call, 14.95 this
// way). max(v, 0) is written as 0.5 v + 0.5 |v|, which keeps a NaN; from |v| = 20 on the second term is 0 (e^-200).
__device__ __forceinline__ float gelu_erf(float v)
{
    const float m = fminf(fabsf(v), 20.f), x = m * 0.70710678118654752f;
    const float t = __fdividef(1.f, fmaf(0.3275911f, x, 1.f));
    const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    return fmaf(-0.5f * m, poly * __expf(-x * x), fmaf(0.5f, v, 0.5f * fabsf(v)));
}

// (the choice outside the loop: with the switch inside an unrolled one, all five activations sit in the path N times over and
// the epilogue of the tensor-core kernel ran from instruction cache misses, 4 us for 32 x 32 outputs)
template <int N> __device__ __forceinline__ void apply_act(float (&v)[N], int act)
{
    switch (act) {
        case UBP_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];      // (fmaxf would turn a NaN into 0)
            break;
        case UBP_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = gelu_erf(v[i]);
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
