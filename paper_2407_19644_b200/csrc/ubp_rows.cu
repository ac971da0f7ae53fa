// Row operators in front of a block-pruned product: root mean square norm with the residual's addition, and rows to 8 bits
// with one scale a row.
//
//   h = x + r (r optional)                       rounded once where it is written back
//   y = (h * gamma) / sqrt(mean(h^2) + eps)      norm; without a norm y = x
//   s = max(max |y| / 448, 2^-126), q = e4m3(y / s)      8-bit output; else y in x's type
//
// One reduction serves both statistics: with t = h * gamma, y = t * rinv and rinv > 0, so max |y| = max |t| * rinv (rounding
// is monotonic, the maximum of the rounded products is the rounded product of the maximum). A row is therefore read once,
// kept in registers as fp32 over the reduction of (sum h^2, max |t|), and written once. Bound by HBM: (2 + 2 + 2 + 1) bytes
// an element for the 16-bit norm with an 8-bit output, 3 for the 16-bit rows.
// The statistics are fp32; x + r is not rounded before it is squared and multiplied.
//
// TPR threads work on a row, each on NV groups of eight elements (16-byte accesses) where every row starts on a 16-byte
// boundary, else on single elements. Rows that do not fit the registers of 512 threads are read twice (the second time
// from L2): nothing is written before the row's statistics are complete, and every element is read and written by one
// thread, so h may be written over x or r in every form.
#include <cuda_runtime.h>

#include <cstdint>

#include "ubp_internal.h"
#include "ubp_types.cuh"

namespace ubp {
namespace {

constexpr int ROWS_MAX_TPR = 512;   // threads of a row at most (128 registers each)

struct RowArgs {
    const void *x;
    const void *r;         // nullable
    const void *gamma;     // norm only
    void *h;               // nullable
    void *y;
    float *scales;         // 8-bit output only
    int64_t ldx, ldr, ldh, ldy;
    int64_t T;
    int C;
    float eps;
    int gamma_f32;
};

// (sum, max) over the TPR threads of a row; TPR is a power of two, rows of one block lie in consecutive threads. Every
// thread of the row gets the same two values: the partial results are combined in one fixed order.
template <bool NORM, bool Q>
__device__ __forceinline__ void row_reduce(float &sum, float &mx, int tpr, float2 *scratch)
{
    const int w = tpr < 32 ? tpr : 32;
    for (int o = w >> 1; o > 0; o >>= 1) {
        if (NORM) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (Q) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    }
    if (tpr > 32) {
        const int warp = threadIdx.x >> 5, nw = tpr >> 5, first = warp / nw * nw;
        if ((threadIdx.x & 31) == 0) scratch[warp] = make_float2(sum, mx);
        __syncthreads();
        float2 v = (int)(threadIdx.x & 31) < nw ? scratch[first + (threadIdx.x & 31)] : make_float2(0.f, 0.f);
        for (int o = 16; o > 0; o >>= 1) {
            if (NORM) v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
            if (Q) v.y = max_nan(v.y, __shfl_xor_sync(0xffffffffu, v.y, o));
        }
        sum = v.x; mx = v.y;
    }
}

template <typename T> __device__ __forceinline__ void gamma8(const RowArgs &a, int c, float (&g)[8])
{
    if (a.gamma_f32) load8<float>(static_cast<const float *>(a.gamma) + c, g);
    else load8<T>(static_cast<const T *>(a.gamma) + c, g);
}
template <typename T> __device__ __forceinline__ float gamma1(const RowArgs &a, int c)
{
    return a.gamma_f32 ? static_cast<const float *>(a.gamma)[c] : to_f32<T>(static_cast<const T *>(a.gamma)[c]);
}

// T: type of x, r, h; TO: output type; VEC: eight elements an access, else one; NV: accesses a thread keeps in registers,
// 0 = any length, read twice
template <typename T, typename TO, bool NORM, bool VEC, int NV>
__global__ void __launch_bounds__(ROWS_MAX_TPR) ubp_rows_kernel(const RowArgs a, const int tpr)
{
    constexpr bool Q = sizeof(TO) == 1;
    constexpr int E = VEC ? 8 : 1;
    __shared__ float2 scratch[ROWS_MAX_TPR / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int rows = blockDim.x / tpr, lane = threadIdx.x % tpr;
    const int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / tpr;
    const bool live = row < a.T;
    const T *x = static_cast<const T *>(a.x) + (live ? row : 0) * a.ldx;
    const T *r = a.r ? static_cast<const T *>(a.r) + (live ? row : 0) * a.ldr : nullptr;
    T *hrow = a.h ? static_cast<T *>(a.h) + (live ? row : 0) * a.ldh : nullptr;
    TO *y = static_cast<TO *>(a.y) + (live ? row : 0) * a.ldy;
    const int step = tpr * E;

    auto load = [&](int c, float (&v)[E]) {
        if constexpr (VEC) {
            load8<T>(x + c, v);
            if (r) {
                float w[8];
                load8<T>(r + c, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += w[e];
            }
        } else {
            v[0] = to_f32<T>(x[c]);
            if (r) v[0] += to_f32<T>(r[c]);
        }
    };
    auto gamma = [&](int c, float (&g)[E]) {
        if constexpr (VEC) gamma8<T>(a, c, g);
        else g[0] = gamma1<T>(a, c);
    };
    auto put_h = [&](int c, const float (&h)[E]) {
        if constexpr (VEC) {
            if (hrow) store8<T>(hrow + c, h);
        } else {
            if (hrow) hrow[c] = from_f32<T>(h[0]);
        }
    };
    auto put = [&](int c, const float (&t)[E], float rinv, float sinv) {
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            o[e] = NORM ? t[e] * rinv : t[e];
            if (Q) o[e] *= sinv;
        }
        if constexpr (VEC) store8<TO>(y + c, o);
        else y[c] = from_f32<TO>(o[0]);
    };

    float sum = 0.f, mx = 0.f;
    // h -> t = h * gamma (t = h without a norm), and both into the row's statistics
    auto stats = [&](int c, float (&v)[E]) {
        float g[E];
        if constexpr (NORM) gamma(c, g);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (NORM) { sum = fmaf(v[e], v[e], sum); v[e] *= g[e]; }
            if (Q) mx = max_nan(mx, fabsf(v[e]));
        }
    };
    constexpr int NK = NV > 0 ? NV : 1;
    float v[NK][E];
    if constexpr (NV > 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = k * step + lane * E;
            if (live && c < a.C) load(c, v[k]);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = k * step + lane * E;
            if (live && c < a.C) {
                if constexpr (NORM) put_h(c, v[k]);
                stats(c, v[k]);
            }
        }
    } else {
        if (live)
            for (int c = lane * E; c < a.C; c += step) { load(c, v[0]); stats(c, v[0]); }
    }
    row_reduce<NORM, Q>(sum, mx, tpr, scratch);
    const float rinv = NORM ? rsqrtf(sum / (float)a.C + a.eps) : 1.f;
    // A product with 1 / s instead of a division for each value (which made the kernel ALU-bound: 336 us instead of HBM's
    // 143 on 16384 x 8192): the quotient is off by at most 1.5 units of 2^-24, against half a code step of 2^-4. s is at
    // least 2^-126, so 1 / s is finite. rinv and 1 / s stay two products: theirs could overflow for a row of tiny values.
    float sinv = 1.f;
    if (Q) {
        const float s = max_nan(__fdiv_rn(NORM ? mx * rinv : mx, E4M3_MAX), ROW_SCALE_MIN);
        sinv = __fdiv_rn(1.f, s);
        if (live && lane == 0) a.scales[row] = s;
    }
    if constexpr (NV > 0) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = k * step + lane * E;
            if (live && c < a.C) put(c, v[k], rinv, sinv);
        }
    } else {
        if (live)
            for (int c = lane * E; c < a.C; c += step) {
                load(c, v[0]);
                if constexpr (NORM) put_h(c, v[0]);
                stats(c, v[0]);      // (the statistics are complete; this only applies gamma)
                put(c, v[0], rinv, sinv);
            }
    }
}

template <typename T, typename TO, bool NORM>
int launch_rows_t(const RowArgs &a, bool vec, cudaStream_t stream)
{
    // Threads per row: enough for at most four (vector) or eight (scalar) accesses a thread; blocks of at least 128 threads.
    const int e = vec ? 8 : 1;
    const int64_t groups = ((int64_t)a.C + e - 1) / e;
    int tpr = 32;
    while (tpr < ROWS_MAX_TPR && (int64_t)tpr * (vec ? 4 : 8) < groups) tpr *= 2;
    // few rows: the latency of one row is what counts, so spread it
    while (tpr < ROWS_MAX_TPR && a.T * tpr < 148 * 512 && tpr < groups) tpr *= 2;
    const int threads = tpr < 128 ? 128 : tpr, rows = threads / tpr;
    const int64_t blocks = (a.T + rows - 1) / rows;
    if (blocks > 0x7fffffff) return UBP_E_UNSUPPORTED;
    const int nv = (int)((groups + tpr - 1) / tpr);
    using Fn = void (*)(const RowArgs, const int);
    Fn fn;
    if (vec) {
        if (nv <= 1) fn = ubp_rows_kernel<T, TO, NORM, true, 1>;
        else if (nv <= 2) fn = ubp_rows_kernel<T, TO, NORM, true, 2>;
        else if (nv <= 4) fn = ubp_rows_kernel<T, TO, NORM, true, 4>;
        else fn = ubp_rows_kernel<T, TO, NORM, true, 0>;
    } else {
        if (nv <= 8) fn = ubp_rows_kernel<T, TO, NORM, false, 8>;
        else if (nv <= 16) fn = ubp_rows_kernel<T, TO, NORM, false, 16>;
        else fn = ubp_rows_kernel<T, TO, NORM, false, 0>;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t err = cudaLaunchKernelEx(&cfg, fn, a, tpr);
    if (err == cudaSuccess) err = cudaGetLastError();
    if (err != cudaSuccess) { set_last_cuda_error((int)err); return UBP_E_CUDA; }
    return UBP_OK;
}

template <bool NORM>
int launch_rows(const RowArgs &a, int dtype, int y_dtype, void *stream)
{
    const int b = dtype_size(dtype), bo = dtype_size(y_dtype);
    auto al = [](const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
    // eight elements an access: whole groups only, and every row of every operand on a boundary of its access
    const bool vec = a.C % 8 == 0 && al(a.x, 16) && a.ldx * b % 16 == 0 && (!a.r || (al(a.r, 16) && a.ldr * b % 16 == 0)) &&
                     (!a.h || (al(a.h, 16) && a.ldh * b % 16 == 0)) && al(a.y, bo == 1 ? 8 : 16) && a.ldy * bo % (bo == 1 ? 8 : 16) == 0 &&
                     (!NORM || al(a.gamma, 16));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (y_dtype == UBP_E4M3) {
        switch (dtype) {
            case UBP_BF16: return launch_rows_t<__nv_bfloat16, __nv_fp8_storage_t, NORM>(a, vec, st);
            case UBP_F16: return launch_rows_t<__half, __nv_fp8_storage_t, NORM>(a, vec, st);
            default: return launch_rows_t<float, __nv_fp8_storage_t, NORM>(a, vec, st);
        }
    }
    if constexpr (NORM) {
        switch (dtype) {
            case UBP_BF16: return launch_rows_t<__nv_bfloat16, __nv_bfloat16, true>(a, vec, st);
            case UBP_F16: return launch_rows_t<__half, __half, true>(a, vec, st);
            default: return launch_rows_t<float, float, true>(a, vec, st);
        }
    }
    return UBP_E_ARG;
}

bool aligned_to(const void *p, int n) { return n < 2 || (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(n - 1)) == 0; }

}  // namespace
}  // namespace ubp

extern "C" int ubp_rmsnorm(const void *x, int64_t ldx, const void *residual, int64_t ldr, const void *gamma, int gamma_dtype,
                           int dtype, int64_t T, int C, float eps, void *h, int64_t ldh, void *y, int64_t ldy, int y_dtype,
                           float *scales, void *stream)
{
    const int b = ubp::dtype_size(dtype), bo = ubp::dtype_size(y_dtype);
    if (!b || b == 1 || !bo || (y_dtype != dtype && y_dtype != UBP_E4M3)) return UBP_E_ARG;
    if (gamma_dtype != dtype && gamma_dtype != UBP_F32) return UBP_E_ARG;
    if (T < 0 || C < 1 || !(eps >= 0.f)) return UBP_E_ARG;
    if (T == 0) return UBP_OK;
    if (!x || !gamma || !y || (y_dtype == UBP_E4M3 && !scales)) return UBP_E_ARG;
    if ((T > 1 && (ldx < C || ldy < C || (residual && ldr < C) || (h && ldh < C)))) return UBP_E_ARG;
    if (!ubp::aligned_to(x, b) || !ubp::aligned_to(residual, b) || !ubp::aligned_to(h, b) || !ubp::aligned_to(y, bo) ||
        !ubp::aligned_to(gamma, ubp::dtype_size(gamma_dtype)) || !ubp::aligned_to(scales, 4)) return UBP_E_ARG;
    const ubp::RowArgs a{x, residual, gamma, h, y, scales, ldx, ldr, ldh, ldy, T, C, eps, gamma_dtype == UBP_F32};
    return ubp::launch_rows<true>(a, dtype, y_dtype, stream);
}

extern "C" int ubp_quant_rows(const void *x, int64_t ldx, int dtype, int64_t T, int C, void *q, int64_t ldq, float *scales,
                              void *stream)
{
    const int b = ubp::dtype_size(dtype);
    if (!b || b == 1 || T < 0 || C < 1) return UBP_E_ARG;
    if (T == 0) return UBP_OK;
    if (!x || !q || !scales || (T > 1 && (ldx < C || ldq < C))) return UBP_E_ARG;
    if (!ubp::aligned_to(x, b) || !ubp::aligned_to(scales, 4)) return UBP_E_ARG;
    const ubp::RowArgs a{x, nullptr, nullptr, nullptr, q, scales, ldx, 0, 0, ldq, T, C, 0.f, 0};
    return ubp::launch_rows<false>(a, dtype, UBP_E4M3, stream);
}
