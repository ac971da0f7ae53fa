// Epilogue of the token-major products: scales, bias, activation, gate, residual.
#ifndef UBP_LINEAR_EPILOGUE_CUH_
#define UBP_LINEAR_EPILOGUE_CUH_

#include "ubp_linear.h"
#include "ubp_types.cuh"

namespace ubp {

// Two sets of activations: for 16-bit outputs approximations whose errors disappear in the output's rounding, and the FULL ones
// of fp32 outputs below them.
//
// v * sigmoid(u) = v / (1 + e^-u). __expf and the approximate division are within a few units of 2^-22 each, far below the
// 16-bit outputs' 2^-9 (bf16) / 2^-12 (f16). e^-u stops at e^88, above 2^126, where the division's quotient is defined as 0 for
// every finite v (the exact value is below 2^-120); unstopped it would be infinity, for which no quotient is defined.
__device__ __forceinline__ float v_sigmoid(float v, float u) { return __fdividef(v, 1.f + __expf(fminf(-u, 88.f))); }

// GELU with erf, 0.5 v (1 + erf(v / sqrt 2)) = v Phi(v), Phi the normal distribution function; with m = |v|: Phi(-m) =
// g(m) e^(-m^2 / 2), and g / t is a polynomial in t = 1 / (1 + p m), fitted here to the least relative error on [0, 15] (degree 6,
// p = 0.265: 6.5 10^-7). Phi(-15) is below 2^-149. Relative errors below 2^-17 down to the smallest results: 1 + erf and
// approximations of erfc with an absolute error lose the digits of the negative tail (1.5 10^-7 is a quarter of Phi(-5)).
__device__ __forceinline__ float phi_of(float v, float tail) { return v < 0.f ? tail : 1.f - tail; }
__device__ __forceinline__ float gelu_erf(float v)
{
    const float m = fminf(fabsf(v), 15.f), t = __fdividef(1.f, fmaf(0.265f, m, 1.f));
    float g = -0.0677110404f;
    g = fmaf(g, t, 0.195008963f);
    g = fmaf(g, t, -0.0659952313f);
    g = fmaf(g, t, 0.142232031f);
    g = fmaf(g, t, 0.0830461904f);
    g = fmaf(g, t, 0.107817546f);
    g = fmaf(g, t, 0.105601303f);
    return v * phi_of(v, g * t * __expf(-0.5f * m * m));
}

// FULL: relative errors of a few units of 2^-23 over the whole range (__expf loses a unit for every unit of its argument). The
// exponent is carried in two numbers: x log2(e) = th + tl, e^x = 2^th (1 + tl ln 2).
__device__ __forceinline__ float exp_two(float th, float tl) { return exp2f(th) * fmaf(tl, 0.69314718056f, 1.f); }
__device__ __forceinline__ float v_sigmoid_full(float v, float u)
{
    const float x = fmaxf(fminf(-u, 100.f), -100.f), th = x * 1.44269502f;                     // log2(e) = 1.44269502 + 1.9259630e-8
    return __fdividef(v, 1.f + exp_two(th, fmaf(x, 1.9259630e-8f, fmaf(x, 1.44269502f, -th))));
}
// v Phi(v) as above with degree 8 and p = 0.35 (3.2 10^-8), m^2 in two numbers. (normcdff is as good, but with it 777 tokens on
// 4096 x 2048 in bf16 took 31.4 us; this 21.8, the 16-bit form 21.0.)
__device__ __forceinline__ float gelu_full(float v)
{
    const float m = fminf(fabsf(v), 15.f), t = __fdividef(1.f, fmaf(0.35f, m, 1.f));
    float g = -0.0291627571f;
    g = fmaf(g, t, 0.14405556f);
    g = fmaf(g, t, -0.255891919f);
    g = fmaf(g, t, 0.159382522f);
    g = fmaf(g, t, -0.023257345f);
    g = fmaf(g, t, 0.105572328f);
    g = fmaf(g, t, 0.119816057f);
    g = fmaf(g, t, 0.139864266f);
    g = fmaf(g, t, 0.139621258f);
    const float h = m * m, l = fmaf(m, m, -h), th = h * -0.72134751f;                            // -log2(e) / 2 = -0.72134751 - 9.629815e-9
    const float tail = g * t * exp_two(th, fmaf(l, -0.72134751f, fmaf(h, -9.629815e-9f, fmaf(h, -0.72134751f, -th))));
    return v * phi_of(v, tail);
}

// (the choice outside the loop: with the switch inside an unrolled one, all five activations sit in the path N times over and
// the epilogue of the tensor-core kernel ran from instruction cache misses, 4 us for 32 x 32 outputs)
template <bool FULL, int N> __device__ __forceinline__ void apply_act(float (&v)[N], int act)
{
    switch (act) {
        case UBP_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];      // (fmaxf would turn a NaN into 0)
            break;
        case UBP_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = FULL ? gelu_full(v[i]) : gelu_erf(v[i]);
            break;
        case UBP_ACT_GELU_TANH:   // 0.5 v (1 + tanh(u)) = v sigmoid(2 u), u = sqrt(2 / pi) (v + 0.044715 v^3)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float u = 1.5957691216057308f * (v[i] + 0.044715f * v[i] * v[i] * v[i]);
                v[i] = FULL ? v_sigmoid_full(v[i], u) : v_sigmoid(v[i], u);
            }
            break;
        case UBP_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = FULL ? v_sigmoid_full(v[i], v[i]) : v_sigmoid(v[i], v[i]);
            break;
        default: break;
    }
}
__device__ __forceinline__ float apply_act(float v, int act, int ydt)
{
    float a[1] = {v};
    if (ydt == UBP_F32) apply_act<true>(a, act);
    else apply_act<false>(a, act);
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
