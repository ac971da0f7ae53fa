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
// boundary, else on single elements. The grid stays on the SMs and walks the rows; a row's loads are issued before the
// statistics of the row before it are reduced, so that the reduction's two barrier-and-shuffle latencies and the stores pass
// under loads in flight (one row per block without that: 103 us instead of 61 for rows 8192 x 16384, HBM 45 % busy).
// Rows that do not fit the registers of a block are read twice (the second time from L2): there nothing is written before
// the row's statistics are complete. Every element is read and written by one thread, so h may be written over x or r in
// every form.
#include <cuda_runtime.h>

#include <cfloat>
#include <cstdint>

#include "ubp_internal.h"
#include "ubp_linear.h"
#include "ubp_types.cuh"

namespace ubp {
namespace {

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

// (sum, max) over the TPR threads of a row, in one fixed order, to every one of them. `scratch` alternates between two
// buffers from row to row: a warp that is one row ahead does not touch what the others still read.
template <bool NORM, bool Q, int TPR>
__device__ __forceinline__ void row_reduce(float &sum, float &mx, float2 *scratch)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (NORM) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (Q) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    }
    if constexpr (TPR > 32) {
        constexpr int NW = TPR / 32;
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = make_float2(sum, mx);
        __syncthreads();
        float2 v = scratch[threadIdx.x & (NW - 1)];
#pragma unroll
        for (int o = NW / 2; o > 0; o >>= 1) {
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

// E elements of x (or r) as they lie in memory
template <typename T, int E> struct Raw {
    static constexpr int N = E * (int)sizeof(T) / 16;
    uint4 w[N];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void get(float (&v)[E]) const
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[4 * i] = __uint_as_float(w[i].x); v[4 * i + 1] = __uint_as_float(w[i].y);
                v[4 * i + 2] = __uint_as_float(w[i].z); v[4 * i + 3] = __uint_as_float(w[i].w);
            }
        } else {
            const uint32_t u[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = unpack2<T>(u[i]);
                v[2 * i] = f.x; v[2 * i + 1] = f.y;
            }
        }
    }
};
template <typename T> struct Raw<T, 1> {
    T w;
    __device__ __forceinline__ void load(const T *p) { w = *p; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_f32<T>(w); }
};

__host__ __device__ constexpr int rows_block(int tpr) { return tpr < 128 ? 128 : tpr; }          // threads of a block
// Blocks an SM holds: 1024 threads of 64 registers, or 512 of 128 where a thread keeps more than 48 values of the row and
// the next one (nv accesses of e values; the next row's x and r as they lie in memory).
__host__ __device__ constexpr int rows_blocks_per_sm(int tpr, bool norm, int e, int nv, int size)
{
    return (nv * e + (nv * e * size + 3) / 4 * (norm ? 2 : 1) > 48 ? 512 : 1024) / rows_block(tpr);
}

// T: type of x, r, h; TO: output type; E: elements an access (8 or 1); TPR: threads a row; NV: accesses a thread keeps in
// registers, 0 = any length, read twice
template <typename T, typename TO, bool NORM, int E, int TPR, int NV>
__global__ void __launch_bounds__(rows_block(TPR), rows_blocks_per_sm(TPR, NORM, E, NV, (int)sizeof(T))) ubp_rows_kernel(const RowArgs a)
{
    constexpr bool Q = sizeof(TO) == 1;
    constexpr int STEP = TPR * E, ROWS = rows_block(TPR) / TPR;
    __shared__ float2 scratch[2][32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x % TPR, c0 = lane * E;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
    const T *x = static_cast<const T *>(a.x) + c0, *r = static_cast<const T *>(a.r) + c0;
    T *h = static_cast<T *>(a.h) + c0;
    TO *y = static_cast<TO *>(a.y) + c0;
    const bool has_r = NORM && a.r, has_h = NORM && a.h;

    float sum, mx;
    auto store_h = [&](int64_t at, const float (&v)[E]) {
        if constexpr (E == 8) store8<T>(h + at, v);
        else h[at] = from_f32<T>(v[0]);
    };
    // h -> t = h * gamma (t = h without a norm), and both into the row's statistics
    auto stats = [&](int c, float (&v)[E]) {
        float g[E];
        if constexpr (NORM) {
            if constexpr (E == 8) gamma8<T>(a, c, g);
            else g[0] = gamma1<T>(a, c);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (NORM) { sum = fmaf(v[e], v[e], sum); v[e] *= g[e]; }
            if (Q) mx = max_nan(mx, fabsf(v[e]));
        }
    };
    // The quotient y / s, two operations a value (a division for each made the kernel ALU-bound: 336 us instead of HBM's 143 on
    // 16384 x 8192). 1 / s in two fp32 numbers: r = 1 / s rounded down, r2 = (1 - r s) r, the difference exact in fp32. y r + y r2
    // with one rounding at the end is off by less than 2^-46 of the quotient before that rounding (2^-30 for scales beyond
    // 2^102, whose r2 is subnormal), so the codes are those of the divided values; y / s by r alone gave one f16 value in
    // 15 000 its neighbour's code. r2 >= 0 keeps the sign of a zero. An infinite scale has r = r2 = 0: finite values become 0,
    // infinities NaN. s is at least 2^-126, so 1 / s is finite. rinv and 1 / s stay two products: theirs could overflow for a
    // row of tiny values.
    float rinv, sinv, sinv2;
    auto finish = [&](bool live) {
        rinv = NORM ? rsqrtf(sum / (float)a.C + a.eps) : 1.f;
        if (Q) {
            const float s = max_nan(__fdiv_rn(NORM ? mx * rinv : mx, E4M3_MAX), ROW_SCALE_MIN);
            sinv = __frcp_rd(s);
            sinv2 = s <= FLT_MAX ? fmaf(-sinv, s, 1.f) * sinv : 0.f;
            if (live && lane == 0) a.scales[row] = s;
        }
    };
    // t -> the value that is stored
    auto out = [&](float t) {
        const float o = NORM ? t * rinv : t;
        return Q ? fmaf(o, sinv, o * sinv2) : o;
    };
    auto put = [&](int64_t at, const float (&v)[E]) {
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = out(v[e]);
        if constexpr (E == 8) store8<TO>(y + at, o);
        else y[at] = from_f32<TO>(o[0]);
    };

    // (rows of one block differ by less than ROWS, so all its threads make the same number of rounds)
    const int64_t rounds = ((int64_t)blockIdx.x * ROWS < a.T) ? (a.T - (int64_t)blockIdx.x * ROWS + stride - 1) / stride : 0;
    if constexpr (NV > 0 && E == 1) {
        // Single elements: whole loops under one condition each and no branch an element (with the conditions inside it was 61
        // instructions an element, which bound the kernel: norm 1531 x 2051 9.7 us, 7.6 so). Places past the row stay 0 and count for
        // nothing; gamma stays in registers from row to row.
        Raw<T, 1> nx[NV], nr[NORM ? NV : 1];
        float g[NORM ? NV : 1];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            nx[k].w = from_f32<T>(0.f);
            if constexpr (NORM) {
                nr[k].w = from_f32<T>(0.f);
                g[k] = c0 + k * STEP < a.C ? gamma1<T>(a, c0 + k * STEP) : 0.f;
            }
        }
        auto fetch = [&](int64_t t) {
            if (t >= a.T) return;
            const T *p = x + t * a.ldx;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (c0 + k * STEP < a.C) nx[k].load(p + k * STEP);
            if (has_r) {
                p = r + t * a.ldr;
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (c0 + k * STEP < a.C) nr[NORM ? k : 0].load(p + k * STEP);
            }
        };
        fetch(row);
        for (int64_t i = 0; i < rounds; ++i, row += stride) {
            const bool live = row < a.T;
            float v[NV];
            sum = 0.f; mx = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k) v[k] = to_f32<T>(nx[k].w);
            if (has_r) {
#pragma unroll
                for (int k = 0; k < NV; ++k) v[k] += to_f32<T>(nr[NORM ? k : 0].w);
            }
            if (has_h && live) {
                T *p = h + row * a.ldh;
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (c0 + k * STEP < a.C) p[k * STEP] = from_f32<T>(v[k]);
            }
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (NORM) { sum = fmaf(v[k], v[k], sum); v[k] *= g[NORM ? k : 0]; }
                if (Q) mx = max_nan(mx, fabsf(v[k]));
            }
            fetch(row + stride);
            row_reduce<NORM, Q, TPR>(sum, mx, scratch[i & 1]);
            finish(live);
            if (live) {
                TO *p = y + row * a.ldy;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    const float o = out(v[k]);
                    if (c0 + k * STEP < a.C) p[k * STEP] = from_f32<TO>(o);
                }
            }
        }
    } else if constexpr (NV > 0) {
        Raw<T, E> nx[NV], nr[NORM ? NV : 1];
        auto fetch = [&](int64_t t) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (t < a.T && c0 + k * STEP < a.C) {
                    nx[k].load(x + t * a.ldx + k * STEP);
                    if (NORM && has_r) nr[NORM ? k : 0].load(r + t * a.ldr + k * STEP);
                }
        };
        fetch(row);
        for (int64_t i = 0; i < rounds; ++i, row += stride) {
            const bool live = row < a.T;
            float v[NV][E];
            sum = 0.f; mx = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (live && c0 + k * STEP < a.C) {
                    nx[k].get(v[k]);
                    if constexpr (NORM) {
                        if (has_r) {
                            float w[E];
                            nr[k].get(w);
#pragma unroll
                            for (int e = 0; e < E; ++e) v[k][e] += w[e];
                        }
                        if (has_h) store_h(row * a.ldh + k * STEP, v[k]);
                    }
                    stats(c0 + k * STEP, v[k]);
                }
            fetch(row + stride);
            row_reduce<NORM, Q, TPR>(sum, mx, scratch[i & 1]);
            finish(live);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (live && c0 + k * STEP < a.C) put(row * a.ldy + k * STEP, v[k]);
        }
    } else {
        for (int64_t i = 0; i < rounds; ++i, row += stride) {      // (one row a block: every thread's row is live)
            sum = 0.f; mx = 0.f;
            auto load = [&](int64_t c, float (&v)[E]) {
                Raw<T, E> q;
                q.load(x + row * a.ldx + c);
                q.get(v);
                if (has_r) {
                    float w[E];
                    q.load(r + row * a.ldr + c);
                    q.get(w);
#pragma unroll
                    for (int e = 0; e < E; ++e) v[e] += w[e];
                }
            };
#pragma unroll 4
            for (int c = 0; c < a.C - c0; c += STEP) {
                float v[E];
                load(c, v);
                stats(c0 + c, v);
            }
            row_reduce<NORM, Q, TPR>(sum, mx, scratch[i & 1]);
            finish(true);
#pragma unroll 2
            for (int c = 0; c < a.C - c0; c += STEP) {
                float v[E];
                load(c, v);
                if (has_h) store_h(row * a.ldh + c, v);
                stats(c0 + c, v);      // (the statistics are complete; this only applies gamma)
                put(row * a.ldy + c, v);
            }
        }
    }
}

template <typename T, typename TO, bool NORM, int E, int TPR, int NV>
int launch_rows_k(const RowArgs &a, int sms, cudaStream_t stream)
{
    const int64_t rows = rows_block(TPR) / TPR, need = (a.T + rows - 1) / rows, fit = (int64_t)sms * rows_blocks_per_sm(TPR, NORM, E, NV, (int)sizeof(T));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(need < fit ? need : fit));
    cfg.blockDim = dim3((unsigned)rows_block(TPR));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t err = cudaLaunchKernelEx(&cfg, ubp_rows_kernel<T, TO, NORM, E, TPR, NV>, a);
    if (err == cudaSuccess) err = cudaGetLastError();
    if (err != cudaSuccess) { set_last_cuda_error((int)err); return UBP_E_CUDA; }
    return UBP_OK;
}

// Threads and accesses a row by its length: the fewest threads whose registers hold it, 32 (a warp a row, no barrier), 128 and
// more. On 16-byte accesses a row of 513 to 1024 or 2049 to 4096 elements takes four times the threads where the SMs hold every
// row at once anyway (f16, us, norm with 8-bit rows / 8-bit rows: 3 x 1024 1.77 / 1.39 on 128 threads, 2.56 / 1.54 on 32; 3000 x
// 1024 6.05 / 4.29 and 5.14 / 3.06; 3 x 4096 norm 2.21 on 512, 2.36 on 256; 16384 x 4096 80.2 / 58.6 and 79.9 / 35.0). Longer
// ones: 4096 x 8192 37.9 / 19.1 on 512 threads, 43.6 / 25.7 on 1024, 55.2 / 36.9 read twice; 2048 x 16384 38.8 / 16.8, read
// twice 49.6 / 24.3.
// Single elements cost their instructions, idle places too, and two to four rows an SM have to be under way: hence the close
// steps there. f16, 1531 rows, us as above:
//   255 elements     32 x 8 3.17 / 1.88, 128 x 8 4.34 / 3.28          1023   128 x 8 4.81 / 3.41, 256 x 8 6.30 / 3.60
//   2559             256 x 10 9.61 / 4.51, 512 x 8 11.3 / 6.22        3001   512 x 8 11.6 / 6.32, 512 x 10 12.8 / 6.77
//   4099             512 x 10 14.8 / 7.14, 512 x 16 24.9 / 8.73, 1024 x 8 21.5 / 11.4
//   6001             1024 x 8 22.4 / 12.2, 512 x 16 32.4 / 9.38       8191   1024 x 8 29.4 / 13.7, 512 x 16 40.8 / 11.8
//   9001             1024 x 10 34.0 / 14.4, 1024 x 16 55.5 / 16.9, read twice 45.9 / 30.8
//   12001            read twice 63.6 / 36.7, 1024 x 16 67.1 / 17.8    16001  read twice 88.8 / 46.5, 1024 x 16 82.7 / 24.9
// Sixteen places spill with the norm's two inputs and gamma beside them; without a norm they hold the row.
template <typename T, typename TO, bool NORM>
int launch_rows_t(const RowArgs &a, bool vec, cudaStream_t st)
{
    const int sms = device_sms();
    if (vec) {
        if (a.C <= 256) return launch_rows_k<T, TO, NORM, 8, 32, 1>(a, sms, st);
        if (a.C <= 512) return launch_rows_k<T, TO, NORM, 8, 32, 2>(a, sms, st);
        if (a.C <= 1024) {
            if (a.T <= (int64_t)sms * rows_blocks_per_sm(128, NORM, 8, 1, (int)sizeof(T))) return launch_rows_k<T, TO, NORM, 8, 128, 1>(a, sms, st);
            return launch_rows_k<T, TO, NORM, 8, 32, 4>(a, sms, st);
        }
        if (a.C <= 2048) return launch_rows_k<T, TO, NORM, 8, 128, 2>(a, sms, st);
        if (a.C <= 4096) {
            if (NORM && a.T <= (int64_t)sms * rows_blocks_per_sm(512, NORM, 8, 1, (int)sizeof(T))) return launch_rows_k<T, TO, NORM, 8, 512, 1>(a, sms, st);
            return launch_rows_k<T, TO, NORM, 8, 256, 2>(a, sms, st);
        }
        if (a.C <= 8192) return launch_rows_k<T, TO, NORM, 8, 512, 2>(a, sms, st);
        // (a norm of fp32 rows would need 32 + 64 registers for the row and the next one: read twice instead)
        if constexpr (!(NORM && sizeof(T) == 4))
            if (a.C <= 16384) return launch_rows_k<T, TO, NORM, 8, 512, 4>(a, sms, st);
        return launch_rows_k<T, TO, NORM, 8, 512, 0>(a, sms, st);
    }
    if (a.C <= 256) return launch_rows_k<T, TO, NORM, 1, 32, 8>(a, sms, st);
    if (a.C <= 1024) return launch_rows_k<T, TO, NORM, 1, 128, 8>(a, sms, st);
    if (a.C <= 2560) return launch_rows_k<T, TO, NORM, 1, 256, 10>(a, sms, st);
    if (a.C <= 4096) return launch_rows_k<T, TO, NORM, 1, 512, 8>(a, sms, st);
    if (a.C <= 5120) return launch_rows_k<T, TO, NORM, 1, 512, 10>(a, sms, st);
    if (a.C <= 8192) return launch_rows_k<T, TO, NORM, 1, NORM ? 1024 : 512, NORM ? 8 : 16>(a, sms, st);
    if (a.C <= 10240) return launch_rows_k<T, TO, NORM, 1, 1024, 10>(a, sms, st);
    if constexpr (!NORM)
        if (a.C <= 16384) return launch_rows_k<T, TO, NORM, 1, 1024, 16>(a, sms, st);
    return launch_rows_k<T, TO, NORM, 1, 512, 0>(a, sms, st);
}

template <bool NORM>
int launch_rows(const RowArgs &a, int dtype, int y_dtype, void *stream)
{
    const int b = dtype_size(dtype), bo = dtype_size(y_dtype);
    auto al = [](const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
    // eight elements an access: whole groups only, and every row of every operand on a boundary of its access (a single row has
    // no pitch)
    auto rows_on = [&](const void *p, int64_t ld, int size, int n) { return al(p, (uintptr_t)n) && (a.T <= 1 || ld * size % n == 0); };
    const int no = bo == 1 ? 8 : 16;
    const bool vec = a.C % 8 == 0 && rows_on(a.x, a.ldx, b, 16) && (!a.r || rows_on(a.r, a.ldr, b, 16)) &&
                     (!a.h || rows_on(a.h, a.ldh, b, 16)) && rows_on(a.y, a.ldy, bo, no) && (!NORM || al(a.gamma, 16));
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
    if (h && (h == y || (T > 1 && ((h == x && ldh != ldx) || (h == residual && ldh != ldr))))) return UBP_E_ARG;
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
