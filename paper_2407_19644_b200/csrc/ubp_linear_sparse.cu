// Token-major product with a block-pruned weight, few tokens: the kept blocks only.
//
//   z[t][o] = sum over entries (i, j, w[0..nbk)) with i <= o < i + nbk of w[o - i] x[t][j]
//
// The canonical format is grouped by the output row a block starts at, which makes the product a sparse matrix-vector
// product over START rows with nbk accumulators per token instead of one: p[i][b] = sum_j w_ij[b] x[j] needs one channel
// index per nbk weights and keeps everything in registers; the output row is the short sum z[o] = sum_b p[o - b][b].
//
// What bounds it: for a token or a few, the plan's bytes (kept weights + 2 bytes an entry), each read once and coalesced.
// A block of threads owns R consecutive output features (two row ranges of a gated layer) and recomputes the nbk - 1 start
// rows before its range, so that no partial sum leaves the block in that direction. S blocks of a cluster split the
// reduction at slab boundaries; their partial outputs meet in distributed shared memory. Sums run in a fixed order: results
// are bitwise reproducible.
// The activations of the cluster rank's channels lie in shared memory as [channel][token] (16-bit; 8-bit codes become f16,
// which holds every one of them), so an entry gathers all its tokens with one access. Eight lanes share a start row: enough
// to read whole 32-byte sectors, few enough that short rows fill their lanes and the lanes' sums join in three steps.
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "ubp_internal.h"
#include "ubp_linear.h"
#include "ubp_linear_epilogue.cuh"
#include "ubp_tc_common.cuh"

namespace ubp {
namespace {

constexpr int SP_THREADS = 512;
constexpr int SP_LANES = 8;           // lanes per start row
constexpr int SP_UNROLL = 4;          // entries a lane has in flight
constexpr int SP_MAX_ROWS = 128;      // output features per block
constexpr int SP_MAX_TOKENS = 8;      // tokens per block (more tokens: further blocks)
constexpr size_t SP_SMEM = 200 * 1024;

struct SpArgs {
    LinearArgs a;
    const float *wscale;              // 8-bit plans
    const uint32_t *off;
    const uint16_t *idx;
    const uint8_t *val;
    int nslab, S, R, ydt;
};

struct F8 {};                         // 8-bit weights (staged activations are f16)
template <typename W> struct XOf { using type = W; };
template <> struct XOf<F8> { using type = __half; };
template <typename W> constexpr int wsize = std::is_same<W, F8>::value ? 1 : 2;

// NBK weights of one entry -> fp32
template <typename W, int NBK> __device__ __forceinline__ void load_raw(const uint8_t *p, uint32_t (&r)[4])
{
    constexpr int bytes = NBK * wsize<W>;
    if constexpr (bytes == 16) {
        const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
        r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
    } else if constexpr (bytes == 8) {
        const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
        r[0] = v.x; r[1] = v.y;
    } else if constexpr (bytes == 4) {
        r[0] = __ldg(reinterpret_cast<const uint32_t *>(p));
    } else if constexpr (bytes == 2) {
        r[0] = __ldg(reinterpret_cast<const uint16_t *>(p));
    } else {
        r[0] = __ldg(p);
    }
}
template <typename W, int NBK> __device__ __forceinline__ void unpack_weights(const uint32_t (&r)[4], float (&w)[NBK])
{
    if constexpr (std::is_same<W, F8>::value) {
        if constexpr (NBK == 1) {
            w[0] = unpack2<__half>(e4m3x2_to_f16x2(r[0])).x;
        } else {
#pragma unroll
            for (int i = 0; i < NBK / 2; ++i) {
                const float2 f = unpack2<__half>(e4m3x2_to_f16x2(r[i >> 1] >> (16 * (i & 1))));
                w[2 * i] = f.x; w[2 * i + 1] = f.y;
            }
        }
    } else if constexpr (NBK == 1) {
        w[0] = unpack2<W>(r[0]).x;
    } else {
#pragma unroll
        for (int i = 0; i < NBK / 2; ++i) {
            const float2 f = unpack2<W>(r[i]);
            w[2 * i] = f.x; w[2 * i + 1] = f.y;
        }
    }
}

__device__ __forceinline__ float ld_cluster(const float *p, uint32_t rank)
{
    uint32_t a;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tc::smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

template <typename W, int NBK, int TT>
__global__ void __launch_bounds__(SP_THREADS) ubp_linear_sparse_kernel(const SpArgs p)
{
    using X = typename XOf<W>::type;
    constexpr int NACC = NBK * TT;
    const LinearArgs &a = p.a;
    extern __shared__ __align__(16) uint8_t smem[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const int S = p.S, rank = (int)blockIdx.x % S, f0 = (int)(blockIdx.x / S) * p.R;
    const int nf = a.F - f0 < p.R ? a.F - f0 : p.R;
    const int64_t t0 = (int64_t)blockIdx.y * TT;
    const int nt = a.T - t0 < TT ? (int)(a.T - t0) : TT;
    const int sl0 = (int)((int64_t)p.nslab * rank / S), sl1 = (int)((int64_t)p.nslab * (rank + 1) / S);
    const int c0 = sl0 * LIN_SLAB, c1 = sl1 * LIN_SLAB < a.C ? sl1 * LIN_SLAB : a.C;
    const int nseg = a.gated ? 2 : 1;
    // start rows of segment q: lo[q] .. q F + f0 + nf; local list: segment 0's, then segment 1's
    const int lo0 = f0 - (NBK - 1) > 0 ? f0 - (NBK - 1) : 0, n0 = f0 + nf - lo0;
    const int lo1 = a.F + f0 - (NBK - 1) > 0 ? a.F + f0 - (NBK - 1) : 0, n1 = nseg == 2 ? a.F + f0 + nf - lo1 : 0;
    const int nrow = n0 + n1;

    const int cw = (c1 - c0 + 1) & ~1;                      // staged channels (pairs)
    X *xs = reinterpret_cast<X *>(smem);                    // [cw][TT]
    // (the same layout in every block of the cluster, whatever its share of the channels: yp is read by offset)
    uint8_t *at = smem + (size_t)((p.nslab + S - 1) / S) * LIN_SLAB * TT * 2;
    float *part = reinterpret_cast<float *>(at);            // [nrow][NBK][TT]
    float *yp = part + (size_t)nseg * (p.R + NBK - 1) * NACC;   // [nseg][R][TT]

    asm volatile("griddepcontrol.wait;" ::: "memory");
    // ---- activations of channels c0 .. c1, two channels a thread
    {
        constexpr int xb = wsize<W>;
        const uint8_t *x = static_cast<const uint8_t *>(a.x) + (t0 * a.ldx + c0) * xb;
        const bool pair = (reinterpret_cast<uintptr_t>(x) % (2 * xb) == 0) && (a.ldx * xb) % (2 * xb) == 0;
        for (int c = 2 * (int)threadIdx.x; c < cw; c += 2 * SP_THREADS) {
            const bool two = c0 + c + 1 < c1;
            uint32_t w[TT];                                 // two channels of token t as two 16-bit values
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                w[t] = 0;
                if (t < nt) {
                    const uint8_t *s = x + ((int64_t)t * a.ldx + c) * xb;
                    if constexpr (xb == 2) {
                        if (pair && two) w[t] = *reinterpret_cast<const uint32_t *>(s);
                        else w[t] = *reinterpret_cast<const uint16_t *>(s) | (two ? (uint32_t)*reinterpret_cast<const uint16_t *>(s + 2) << 16 : 0u);
                    } else {
                        uint32_t c2;
                        if (pair && two) c2 = *reinterpret_cast<const uint16_t *>(s);
                        else c2 = s[0] | (two ? (uint32_t)s[1] << 8 : 0u);
                        w[t] = e4m3x2_to_f16x2(c2);
                    }
                }
            }
            uint32_t *d = reinterpret_cast<uint32_t *>(xs + (size_t)c * TT);
            if constexpr (TT == 1) {
                d[0] = w[0];
            } else {
                uint32_t o[TT];
#pragma unroll
                for (int t = 0; t < TT / 2; ++t) {
                    o[t] = __byte_perm(w[2 * t], w[2 * t + 1], 0x5410);
                    o[TT / 2 + t] = __byte_perm(w[2 * t], w[2 * t + 1], 0x7632);
                }
                if constexpr (TT == 2) {
                    *reinterpret_cast<uint2 *>(d) = make_uint2(o[0], o[1]);
                } else {
#pragma unroll
                    for (int t = 0; t < TT; t += 4) *reinterpret_cast<uint4 *>(d + t) = make_uint4(o[t], o[t + 1], o[t + 2], o[t + 3]);
                }
            }
        }
    }
    __syncthreads();

    // ---- partial sums of the start rows
    const int lane = threadIdx.x & (SP_LANES - 1), grp = (int)threadIdx.x / SP_LANES;
    for (int rb = (grp & ~3); rb < nrow; rb += SP_THREADS / SP_LANES) {      // a warp's four groups walk together
        const int r = rb + (grp & 3);
        float acc[NACC];
#pragma unroll
        for (int i = 0; i < NACC; ++i) acc[i] = 0.f;
        uint32_t e = 0, e1 = 0;
        if (r < nrow) {
            const int row = r < n0 ? lo0 + r : lo1 + (r - n0);
            e = __ldg(p.off + (size_t)row * p.nslab + sl0);
            e1 = __ldg(p.off + (size_t)row * p.nslab + sl1);
        }
        for (uint32_t k = e + lane; k < e1; k += SP_LANES * SP_UNROLL) {
            uint32_t raw[SP_UNROLL][4];
            int j[SP_UNROLL];
#pragma unroll
            for (int u = 0; u < SP_UNROLL; ++u) {
                const uint32_t ku = k + u * SP_LANES;
                raw[u][0] = raw[u][1] = raw[u][2] = raw[u][3] = 0;          // (beyond the row's end: weight 0, channel c0)
                j[u] = c0;
                if (ku < e1) {
                    load_raw<W, NBK>(p.val + (size_t)ku * (NBK * wsize<W>), raw[u]);
                    j[u] = __ldg(p.idx + ku);
                }
            }
#pragma unroll
            for (int u = 0; u < SP_UNROLL; ++u) {
                if (!UBP_CHK_SMEM(j[u] >= c0 && j[u] < c1, a.status)) continue;
                float w[NBK], x[TT];
                unpack_weights<W, NBK>(raw[u], w);
                const X *xp = xs + (size_t)(j[u] - c0) * TT;
                if constexpr (TT == 1) {
                    x[0] = to_f32<X>(*xp);
                } else {
                    uint32_t xw[TT / 2];
                    if constexpr (TT == 2) xw[0] = *reinterpret_cast<const uint32_t *>(xp);
                    else if constexpr (TT == 4) { const uint2 q = *reinterpret_cast<const uint2 *>(xp); xw[0] = q.x; xw[1] = q.y; }
                    else { const uint4 q = *reinterpret_cast<const uint4 *>(xp); xw[0] = q.x; xw[1] = q.y; xw[2] = q.z; xw[3] = q.w; }
#pragma unroll
                    for (int t = 0; t < TT / 2; ++t) { const float2 f = unpack2<X>(xw[t]); x[2 * t] = f.x; x[2 * t + 1] = f.y; }
                }
#pragma unroll
                for (int b = 0; b < NBK; ++b)
#pragma unroll
                    for (int t = 0; t < TT; ++t) acc[b * TT + t] = fmaf(w[b], x[t], acc[b * TT + t]);
            }
        }
        __syncwarp();
        // join the eight lanes: as long as a lane holds more than one sum, it keeps half of them and hands over the other
        int first = 0;
#pragma unroll
        for (int o = SP_LANES / 2, n = NACC; o > 0; o >>= 1) {
            if (n > 1) {
                n >>= 1;
                const bool up = (lane & o) != 0;
#pragma unroll
                for (int i = 0; i < NACC; ++i) {
                    if (i >= n) break;
                    const float send = up ? acc[i] : acc[i + n], keep = up ? acc[i + n] : acc[i];
                    acc[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                }
                if (up) first += n;
            } else {
                acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], o);
            }
        }
        constexpr int left = NACC >= SP_LANES ? NACC / SP_LANES : 1;
        if (r < nrow)
#pragma unroll
            for (int i = 0; i < left; ++i) part[(size_t)r * NACC + first + i] = acc[i];
    }
    __syncthreads();
    // ---- output rows of this block's channels
    for (int i = threadIdx.x; i < nseg * nf * TT; i += SP_THREADS) {
        const int t = i % TT, f = (i / TT) % nf, q = i / (TT * nf);
        const int lo = q ? lo1 : lo0, base = q ? n0 : 0, row = q * a.F + f0 + f;
        float s = 0.f;
#pragma unroll
        for (int b = 0; b < NBK; ++b)
            if (row - b >= lo) s += part[(size_t)(base + row - b - lo) * NACC + b * TT + t];
        yp[((size_t)q * p.R + f) * TT + t] = s;
    }
    if (S > 1) tc::cluster_sync();
    else __syncthreads();
    // ---- the cluster's partial outputs, epilogue: rank k finishes its share of the features
    const int fa = nf * rank / S, fb = nf * (rank + 1) / S, nshare = fb - fa;
    for (int i = threadIdx.x; i < nshare * nt; i += SP_THREADS) {
        const int f = fa + i % nshare, t = i / nshare;
        float z[2] = {0.f, 0.f};
        for (int q = 0; q < nseg; ++q) {
            const float *src = yp + ((size_t)q * p.R + f) * TT + t;
            float s = 0.f;
            if (S > 1) { for (int k = 0; k < S; ++k) s += ld_cluster(src, (uint32_t)k); }
            else s = *src;
            const int row = q * a.F + f0 + f;
            if (std::is_same<W, F8>::value) s *= a.xs[t0 + t] * p.wscale[row];
            if (a.bias) s += a.bias[row];
            z[q] = s;
        }
        float v = apply_act(z[0], a.act);
        if (nseg == 2) v *= z[1];
        if (a.res) v += load_elem(a.res, (t0 + t) * a.ldr + f0 + f, p.ydt);
        store_elem(a.y, (t0 + t) * a.ldy + f0 + f, v, p.ydt);
    }
    if (S > 1) tc::cluster_sync();                           // nobody leaves while its shared memory is being read
}

template <typename W, int NBK, int TT>
int launch_t(const SpArgs &p, int64_t chunks, size_t smem, cudaStream_t stream)
{
    const auto kern = ubp_linear_sparse_kernel<W, NBK, TT>;
    static bool done[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = -1;
    if (dev < 0 || dev >= 64 || !done[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SP_SMEM);
        if (e != cudaSuccess) { set_last_cuda_error((int)e); return UBP_E_CUDA; }
        if (dev >= 0 && dev < 64) done[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.a.F + p.R - 1) / p.R * p.S), (unsigned)chunks);
    cfg.blockDim = dim3(SP_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.S;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { set_last_cuda_error((int)e); return UBP_E_CUDA; }
    return UBP_OK;
}

template <typename W, int NBK>
int launch_nbk(const SpArgs &p, int TT, int64_t chunks, size_t smem, cudaStream_t st)
{
    switch (TT) {
        case 1: return launch_t<W, NBK, 1>(p, chunks, smem, st);
        case 2: return launch_t<W, NBK, 2>(p, chunks, smem, st);
        case 4: return launch_t<W, NBK, 4>(p, chunks, smem, st);
        default: return launch_t<W, NBK, 8>(p, chunks, smem, st);
    }
}
template <typename W>
int launch_w(const SpArgs &p, int nbk, int TT, int64_t chunks, size_t smem, cudaStream_t st)
{
    switch (nbk) {
        case 1: return launch_nbk<W, 1>(p, TT, chunks, smem, st);
        case 2: return launch_nbk<W, 2>(p, TT, chunks, smem, st);
        case 4: return launch_nbk<W, 4>(p, TT, chunks, smem, st);
        default: return launch_nbk<W, 8>(p, TT, chunks, smem, st);
    }
}

}  // namespace

int launch_linear_sparse(const ubp_linear_plan *pl, const LinearArgs &a, int y_dtype, void *stream)
{
    SpArgs p;
    p.a = a;
    p.wscale = reinterpret_cast<const float *>(pl->dev + pl->img.scale_off);
    p.off = reinterpret_cast<const uint32_t *>(pl->dev + pl->img.off_off);
    p.idx = reinterpret_cast<const uint16_t *>(pl->dev + pl->img.idx_off);
    p.val = pl->dev + pl->img.val_off;
    p.nslab = pl->img.nslab;
    p.ydt = y_dtype;
    const int nbk = pl->img.nbk, nseg = a.gated ? 2 : 1;
    // tokens per block: the power of two that takes the launch's tokens in as few blocks as eight would
    const int64_t chunks = (a.T + SP_MAX_TOKENS - 1) / SP_MAX_TOKENS, per = (a.T + chunks - 1) / chunks;
    int TT = 1;
    while (TT < per) TT *= 2;
    const int64_t nchunk = (a.T + TT - 1) / TT;
    if (nchunk > 65535) return UBP_E_UNSUPPORTED;
    int sms = 148, dev = 0;
    if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    // split of the reduction: up to four, and as far as the staged channels have to fit shared memory
    int S = 1;
    while (S < 4 && S * 2 <= p.nslab) S *= 2;
    // features per block: two blocks an SM over the whole grid
    int64_t R = ((int64_t)a.F * S * nchunk + 2 * sms - 1) / (2 * sms);
    R = R < 8 ? 8 : R > SP_MAX_ROWS ? SP_MAX_ROWS : R;
    if (R > a.F) R = a.F;
    size_t smem;
    for (;;) {
        const size_t cw = (size_t)((p.nslab + S - 1) / S) * LIN_SLAB;
        smem = cw * TT * 2 + (size_t)nseg * ((size_t)(R + nbk - 1) * nbk + R) * TT * 4;
        if (smem <= SP_SMEM) break;
        if (S < 8 && S * 2 <= p.nslab) S *= 2;
        else if (R > 8) R /= 2;
        else return UBP_E_UNSUPPORTED;
    }
    p.S = S;
    p.R = (int)R;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (pl->dtype) {
        case UBP_BF16: return launch_w<__nv_bfloat16>(p, nbk, TT, nchunk, smem, st);
        case UBP_F16: return launch_w<__half>(p, nbk, TT, nchunk, smem, st);
        default: return launch_w<F8>(p, nbk, TT, nchunk, smem, st);
    }
}

}  // namespace ubp
