// Token-major product with a block-pruned weight, few tokens: the kept blocks only.
//
//   z[t][o] = sum over entries (i, j, w[0..nbk)) with i <= o < i + nbk of w[o - i] x[t][j]
//
// The canonical format is grouped by the output row a block starts at, which makes the product a sparse matrix-vector
// product over START rows with nbk accumulators per token instead of one: p[i][b] = sum_j w_ij[b] x[j] needs one channel
// index per nbk weights and keeps everything in registers; the output row is the short sum z[o] = sum_b p[o - b][b].
//
// What bounds it: for a token or a few, the plan's bytes (kept weights + 2 bytes an entry). A block of threads owns R
// consecutive output features (two row ranges of a gated layer) and recomputes the nbk - 1 start rows before its range, so
// that no partial sum leaves the block. Its entries are one contiguous run per slab and range, which bulk copies stream
// through a ring in shared memory: up to 190 KB an SM in flight, started before the kernel waits for the one before it (the
// weights are constants of the layer). The first form -- lanes load their entries from global memory, four blocks of a
// cluster to a reduction -- was bound by the latency of its offset -> entry -> next row chains: 6.9 us for a token on
// 4096 x 4096 at 80 % and 20.4 us on 16384 x 4096 gated in 8 bits, DRAM 10 % busy.
// The activations of a group of slabs lie in shared memory as [channel][token] (16-bit; 8-bit codes become f16, which holds
// every one of them), so an entry gathers all its tokens with one access. Sixteen lanes share a start row. Sums run in a
// fixed order (a row that spans two stages of the ring is continued after the block's barrier): results are bitwise
// reproducible.
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
constexpr int SP_LANES = 16;          // lanes per start row
constexpr int SP_UNROLL = 4;          // entries a lane has in flight
constexpr int SP_MAX_TOKENS = 8;      // tokens per block (more tokens: further blocks)
constexpr uint32_t SP_STAGE = 48 * 1024;
constexpr int SP_MAX_STAGES = 4;
constexpr size_t SP_X = 64 * 1024;    // staged activations at most (at least one slab: 64 KB of eight tokens)
constexpr size_t SP_SMEM = 224 * 1024;

struct SpArgs {
    LinearArgs a;
    const float *wscale;              // 8-bit plans
    const uint32_t *off;
    const uint16_t *idx;
    const uint8_t *val;
    int nslab, R, ydt;
    int nstage;                       // stages of the ring
    uint32_t cap;                     // entries a stage holds (multiple of 16)
    int xslabs;                       // slabs staged together
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
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
    } else if constexpr (bytes == 8) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        r[0] = v.x; r[1] = v.y;
    } else if constexpr (bytes == 4) {
        r[0] = *reinterpret_cast<const uint32_t *>(p);
    } else if constexpr (bytes == 2) {
        r[0] = *reinterpret_cast<const uint16_t *>(p);
    } else {
        r[0] = *p;
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

template <typename W, int NBK, int TT>
__global__ void __launch_bounds__(SP_THREADS, 1) ubp_linear_sparse_kernel(const SpArgs p)
{
    using X = typename XOf<W>::type;
    constexpr int NACC = NBK * TT, VB = NBK * wsize<W>;          // accumulators of a start row; bytes of an entry's weights
    const LinearArgs &a = p.a;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bar_full[SP_MAX_STAGES];
    __shared__ int abort_flag;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const int f0 = (int)blockIdx.x * p.R, nf = a.F - f0 < p.R ? a.F - f0 : p.R;
    const int64_t t0 = (int64_t)blockIdx.y * TT;
    const int nt = a.T - t0 < TT ? (int)(a.T - t0) : TT;
    const int nseg = a.gated ? 2 : 1;
    // start rows of row range q: lo .. q F + f0 + nf
    const int lo0 = f0 - (NBK - 1) > 0 ? f0 - (NBK - 1) : 0, n0 = f0 + nf - lo0;
    const int lo1 = a.F + f0 - (NBK - 1) > 0 ? a.F + f0 - (NBK - 1) : 0, n1 = nseg == 2 ? a.F + f0 + nf - lo1 : 0;
    const int nrow = n0 + n1, pitch = p.R + NBK;                 // offsets kept of a run: up to R + NBK - 1 rows and the end
    const int nrun = p.nslab * nseg;                             // runs of entries: (slab, range), range fastest

    // shared memory: ring [stage][weights | channels], activations [channel][TT], partial sums [row][NBK][TT], offsets
    const uint32_t vbytes = p.cap * VB, stage_bytes = vbytes + p.cap * 2;
    X *xs = reinterpret_cast<X *>(smem + (size_t)p.nstage * stage_bytes);
    const int xw = p.xslabs * LIN_SLAB;
    float *part = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(xs) + (size_t)xw * TT * 2);
    uint32_t *off = reinterpret_cast<uint32_t *>(part + (size_t)nseg * (p.R + NBK - 1) * NACC);

    for (int i = threadIdx.x; i < nrun * pitch; i += SP_THREADS) {
        const int run = i / pitch, r = i - run * pitch, q = nseg == 2 ? run & 1 : 0, n = q ? n1 : n0;
        const int64_t at = (int64_t)(nseg == 2 ? run >> 1 : run) * a.M + (q ? lo1 : lo0) + (r < n ? r : n);
        off[i] = __ldg(p.off + at);
    }
    for (int i = threadIdx.x; i < nrow * NACC; i += SP_THREADS) part[i] = 0.f;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int s = 0; s < p.nstage; ++s) tc::mbar_init(tc::smem_u32(&bar_full[s]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    // Walks the runs in pieces of at most `cap` entries whose ends are multiples of 16 entries (16-byte aligned copies): a
    // piece may begin or end with entries of other rows, which nobody reads.
    struct Cursor { int run; uint32_t pos; };
    auto run_begin = [&](int run) { return off[run * pitch] & ~15u; };
    auto run_end = [&](int run) { return off[run * pitch + ((nseg == 2 && (run & 1)) ? n1 : n0)]; };
    auto piece = [&](Cursor &c, uint32_t &b, uint32_t &e) {
        while (c.run < nrun && (c.pos >= run_end(c.run))) { if (++c.run < nrun) c.pos = run_begin(c.run); }
        if (c.run >= nrun) return false;
        b = c.pos;
        e = (run_end(c.run) + 15u) & ~15u;
        if (e - b > p.cap) e = b + p.cap;
        c.pos = e;
        return true;
    };
    auto issue = [&](int st, uint32_t b, uint32_t e) {
        const uint32_t bar = tc::smem_u32(&bar_full[st]), n = e - b, dst = tc::smem_u32(smem) + (uint32_t)st * stage_bytes;
        tc::mbar_expect_tx(bar, n * (VB + 2));
        tc::bulk_load(dst, p.val + (size_t)b * VB, n * VB, bar);
        tc::bulk_load(dst + vbytes, p.idx + b, n * 2, bar);
    };
    Cursor ahead{0, run_begin(0)}, here{0, run_begin(0)};
    if (threadIdx.x == 0) {
        uint32_t b, e;
        for (int s = 0; s < p.nstage && piece(ahead, b, e); ++s) issue(s, b, e);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");

    const int lane = threadIdx.x & (SP_LANES - 1), grp = (int)threadIdx.x / SP_LANES;
    int st = 0, xg = -1;
    uint32_t ph = 0, pb, pe;
    bool ok = true;
    while (piece(here, pb, pe)) {
        const int run = here.run, slab = nseg == 2 ? run >> 1 : run, q = nseg == 2 ? run & 1 : 0;
        if (slab / p.xslabs != xg) {
            // ---- activations of the next group of slabs, two channels a thread
            xg = slab / p.xslabs;
            const int c0 = xg * xw, c1 = a.C - c0 < xw ? a.C : c0 + xw;
            constexpr int xb = wsize<W>;
            const uint8_t *x = static_cast<const uint8_t *>(a.x) + (t0 * a.ldx + c0) * xb;
            const bool pair = (reinterpret_cast<uintptr_t>(x) % (2 * xb) == 0) && (a.ldx * xb) % (2 * xb) == 0;
#pragma unroll 2
            for (int c = 2 * (int)threadIdx.x; c < c1 - c0; c += 2 * SP_THREADS) {
                const bool two = c0 + c + 1 < c1;
                uint32_t w[TT];                                  // two channels of token t as two 16-bit values
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    w[t] = 0;
                    if (t < nt) {
                        const uint8_t *s = x + ((int64_t)t * a.ldx + c) * xb;
                        if constexpr (xb == 2) {
                            if (pair && two) w[t] = *reinterpret_cast<const uint32_t *>(s);
                            else w[t] = *reinterpret_cast<const uint16_t *>(s) | (two ? (uint32_t)*reinterpret_cast<const uint16_t *>(s + 2) << 16 : 0u);
                        } else {
                            if (pair && two) w[t] = *reinterpret_cast<const uint16_t *>(s);
                            else w[t] = s[0] | (two ? (uint32_t)s[1] << 8 : 0u);
                        }
                    }
                }
                if constexpr (xb == 1) {
#pragma unroll
                    for (int t = 0; t < TT; ++t) w[t] = e4m3x2_to_f16x2(w[t]);
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
            __syncthreads();
        }
        if (ok) ok = tc::mbar_wait(tc::smem_u32(&bar_full[st]), ph, &abort_flag);
        if (ok) {
            // ---- the rows with entries in this piece
            const uint32_t *ro = off + run * pitch;
            const int n = q ? n1 : n0, base = q ? n0 : 0;
            const uint8_t *val = smem + (size_t)st * stage_bytes;
            const uint16_t *idx = reinterpret_cast<const uint16_t *>(val + vbytes);
            const X *xslab = xs + (size_t)(slab - xg * p.xslabs) * LIN_SLAB * TT;
            [[maybe_unused]] const int width = a.C - slab * LIN_SLAB < LIN_SLAB ? a.C - slab * LIN_SLAB : LIN_SLAB;
            int first = 0;                                       // first row that ends behind the piece's begin
            for (int hi = n; first < hi;) {
                const int mid = (first + hi) >> 1;
                if (ro[mid + 1] > pb) hi = mid;
                else first = mid + 1;
            }
            for (int rb = first + (grp & ~1); rb < n && ro[rb] < pe; rb += SP_THREADS / SP_LANES) {   // a warp's two groups walk together
                const int r = rb + (grp & 1);
                uint32_t e = 0, e1 = 0;
                if (r < n) {
                    e = ro[r] > pb ? ro[r] - pb : 0u;
                    e1 = (ro[r + 1] < pe ? ro[r + 1] : pe);
                    e1 = e1 > pb ? e1 - pb : 0u;
                }
                float acc[NACC];
#pragma unroll
                for (int i = 0; i < NACC; ++i) acc[i] = 0.f;
                for (uint32_t k = e + lane; k < e1; k += SP_LANES * SP_UNROLL) {
                    uint32_t raw[SP_UNROLL][4];
                    int j[SP_UNROLL];
#pragma unroll
                    for (int u = 0; u < SP_UNROLL; ++u) {
                        const uint32_t ku = k + u * SP_LANES;
                        raw[u][0] = raw[u][1] = raw[u][2] = raw[u][3] = 0;      // (beyond the row's end: weight 0)
                        j[u] = -1;
                        if (ku < e1) {
                            load_raw<W, NBK>(val + (size_t)ku * VB, raw[u]);
                            j[u] = idx[ku];
                        }
                    }
#pragma unroll
                    for (int u = 0; u < SP_UNROLL; ++u) {
                        if (j[u] < 0 || !UBP_CHK_SMEM(j[u] < width, a.status)) continue;
                        float w[NBK], x[TT];
                        unpack_weights<W, NBK>(raw[u], w);
                        const X *xp = xslab + (size_t)j[u] * TT;
                        if constexpr (TT == 1) {
                            x[0] = to_f32<X>(*xp);
                        } else {
                            uint32_t xw2[TT / 2];
                            if constexpr (TT == 2) xw2[0] = *reinterpret_cast<const uint32_t *>(xp);
                            else if constexpr (TT == 4) { const uint2 v = *reinterpret_cast<const uint2 *>(xp); xw2[0] = v.x; xw2[1] = v.y; }
                            else { const uint4 v = *reinterpret_cast<const uint4 *>(xp); xw2[0] = v.x; xw2[1] = v.y; xw2[2] = v.z; xw2[3] = v.w; }
#pragma unroll
                            for (int t = 0; t < TT / 2; ++t) { const float2 f = unpack2<X>(xw2[t]); x[2 * t] = f.x; x[2 * t + 1] = f.y; }
                        }
#pragma unroll
                        for (int b = 0; b < NBK; ++b)
#pragma unroll
                            for (int t = 0; t < TT; ++t) acc[b * TT + t] = fmaf(w[b], x[t], acc[b * TT + t]);
                    }
                }
                __syncwarp();
                // join the lanes: as long as a lane holds more than one sum, it keeps half of them and hands over the other
                int at = 0;
#pragma unroll
                for (int o = SP_LANES / 2, m = NACC; o > 0; o >>= 1) {
                    if (m > 1) {
                        m >>= 1;
                        const bool up = (lane & o) != 0;
#pragma unroll
                        for (int i = 0; i < NACC; ++i) {
                            if (i >= m) break;
                            const float send = up ? acc[i] : acc[i + m], keep = up ? acc[i + m] : acc[i];
                            acc[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                        }
                        if (up) at += m;
                    } else {
                        acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], o);
                    }
                }
                constexpr int left = NACC >= SP_LANES ? NACC / SP_LANES : 1;
                // (with fewer sums than lanes several lanes hold the same one: the first of them adds it)
                constexpr int same = NACC >= SP_LANES ? 1 : SP_LANES / NACC;
                if (r < n && (lane & (same - 1)) == 0)
#pragma unroll
                    for (int i = 0; i < left; ++i) part[(size_t)(base + r) * NACC + at + i] += acc[i];
            }
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t b, e;
            if (piece(ahead, b, e)) issue(st, b, e);
        }
        if (++st == p.nstage) { st = 0; ph ^= 1u; }
    }
    if (!ok && threadIdx.x == 0) atomicExch(a.status, 1);
    // ---- output rows and epilogue: neighbouring threads hold neighbouring features
    for (int i = threadIdx.x; i < nf * nt; i += SP_THREADS) {
        const int f = i % nf, t = i / nf;
        float z[2] = {0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (q == nseg) break;
            const int lo = q ? lo1 : lo0, base = q ? n0 : 0, row = q * a.F + f0 + f;
            float s = 0.f;
#pragma unroll
            for (int b = 0; b < NBK; ++b)
                if (row - b >= lo) s += part[(size_t)(base + row - b - lo) * NACC + b * TT + t];
            if (std::is_same<W, F8>::value) s *= a.xs[t0 + t] * p.wscale[row];
            if (a.bias) s += a.bias[row];
            z[q] = s;
        }
        float v = apply_act(z[0], a.act);
        if (nseg == 2) v *= z[1];
        if (a.res) v += load_elem(a.res, (t0 + t) * a.ldr + f0 + f, p.ydt);
        store_elem(a.y, (t0 + t) * a.ldy + f0 + f, v, p.ydt);
    }
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
    cfg.gridDim = dim3((unsigned)((p.a.F + p.R - 1) / p.R), (unsigned)chunks);
    cfg.blockDim = dim3(SP_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
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
    // Features per block: one block an SM over the whole grid, at least 8 (each block recomputes nbk - 1 start rows). Shared
    // memory: the activations of as many slabs as fit 64 KB, the partial sums and offsets, and the rest for the ring.
    const int vb = nbk * (pl->dtype == UBP_E4M3 ? 1 : 2);
    p.cap = SP_STAGE / (uint32_t)(vb + 2) & ~63u;                // (a stage and its parts stay 128-byte aligned)
    p.xslabs = (int)(SP_X / ((size_t)LIN_SLAB * TT * 2));
    if (p.xslabs > p.nslab) p.xslabs = p.nslab;
    int64_t R = ((int64_t)a.F * nchunk + sms - 1) / sms;
    R = R < 8 ? 8 : R > a.F ? a.F : R;
    size_t smem;
    for (;; R = (R + 1) / 2) {
        const size_t fixed = (size_t)p.xslabs * LIN_SLAB * TT * 2 + (size_t)nseg * (R + nbk - 1) * nbk * TT * 4 +
                             (size_t)p.nslab * nseg * (R + nbk) * 4;
        const size_t stage = (size_t)p.cap * (vb + 2);
        p.nstage = fixed < SP_SMEM ? (int)((SP_SMEM - fixed) / stage) : 0;
        if (p.nstage > SP_MAX_STAGES) p.nstage = SP_MAX_STAGES;
        smem = fixed + (size_t)p.nstage * stage;
        if (p.nstage >= 2) break;
        if (R <= 1) return UBP_E_UNSUPPORTED;
    }
    p.R = (int)R;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (pl->dtype) {
        case UBP_BF16: return launch_w<__nv_bfloat16>(p, nbk, TT, nchunk, smem, st);
        case UBP_F16: return launch_w<__half>(p, nbk, TT, nchunk, smem, st);
        default: return launch_w<F8>(p, nbk, TT, nchunk, smem, st);
    }
}

}  // namespace ubp
