// Token-major product with a block-pruned weight, few tokens: the kept blocks only.
//
//   z[t][o] = sum over entries (i, j, w[0..nbk)) with i <= o < i + nbk of w[o - i] x[t][j]
//
// The canonical format is grouped by the output row a block starts at, which makes the product a sparse matrix-vector
// product over START rows with nbk accumulators per token instead of one: p[i][b] = sum_j w_ij[b] x[j] needs one channel
// index per nbk weights and keeps everything in registers; the output row is the short sum z[o] = sum_b p[o - b][b].
//
// What bounds it: for a token or a few, the plan's bytes (kept weights + 2 bytes an entry) as long as few instructions go with
// them. A block of threads owns a run of output features (two row ranges of a gated layer) and recomputes the start rows
// before its range that reach into it, so that no partial sum leaves the block. A warp takes a bundle of start rows at a time
// (8, 16 or 32 lanes a row): the plan deals the rows' chunks to the lanes in the order they are read, so a step is one
// coalesced 512-byte load of weights, one of channels, and no test; the lanes' sums join once a bundle. The weights are
// constants of the layer, so the first steps are loaded before the kernel waits for the one before it, and the next steps'
// loads are always under way. Forms that were measured before this one, us for a token on 4096 x 4096 at 80 % bf16 /
// 16384 x 4096 gated e4m3 (this: 3.65 / 6.5): a group of lanes per row in the canonical order, four blocks of a cluster to a
// reduction, 6.9 / 20.4 (chains of dependent loads); a ring of bulk copies in shared memory, 6.7 / 14.0 (a stage holds too few
// rows for the warps, and its barriers add up); equal shares of the canonical stream to groups of lanes, 5.6 / 12.6 (170
// instructions a chunk, most of them for finding rows).
// The activations lie in shared memory as [channel][token] (16-bit; 8-bit codes become f16, which holds every one of them),
// so an entry gathers all its tokens with one access. Every sum has a fixed order: results are bitwise reproducible.
//
// Infinities and NaN in x reach the outputs that keep their channel and no other. The plan fills rows up with entries of weight
// zero at a channel of its own choice, whose product with an infinity would be NaN: a warp whose sums are not finite does the
// bundle once more without them (two or three instructions a bundle for every other call).
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <type_traits>

#include "ubp_internal.h"
#include "ubp_linear.h"
#include "ubp_linear_epilogue.cuh"
#include "ubp_tc_common.cuh"

namespace ubp {
namespace {

constexpr int SP_THREADS = 512;       // and twice that for large layers, see launch_linear_sparse
constexpr int SP_MAX_TOKENS = 8;      // tokens per block (more tokens: further blocks)
constexpr size_t SP_X = 128 * 1024;   // staged activations at most (fewer tokens per block where a row is long)
constexpr size_t SP_SMEM = 224 * 1024;
constexpr int SP_TWO_C = 48 * 1024;   // channels of a token that leave room for a second block on the SM

struct SpArgs {
    LinearArgs a;
    const float *wscale;              // 8-bit plans
    const uint32_t *off;
    const uint16_t *idx;
    const uint8_t *val;
    const uint32_t *cnt;              // entries of a start row
    uint32_t steps;                   // of the whole plan
    int lanes;                        // lanes per start row
    int grid, ydt;
    bool wide;                        // twice the threads
};

struct F8 {};                         // 8-bit weights (staged activations are f16)
template <typename W> struct XOf { using type = W; };
template <> struct XOf<F8> { using type = __half; };
template <typename W> constexpr int wsize = std::is_same<W, F8>::value ? 1 : 2;

// EPC 16-bit channel numbers of a chunk, two a word (aligned to their size up to 16 bytes)
template <int EPC> __device__ __forceinline__ void load_channels(const uint16_t *p, uint32_t (&j)[EPC > 1 ? EPC / 2 : 1])
{
    if constexpr (EPC == 1) {
        j[0] = __ldg(p);
    } else if constexpr (EPC == 2) {
        j[0] = __ldg(reinterpret_cast<const uint32_t *>(p));
    } else if constexpr (EPC == 4) {
        const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
        j[0] = v.x; j[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < EPC / 8; ++i) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p) + i);
            j[4 * i] = v.x; j[4 * i + 1] = v.y; j[4 * i + 2] = v.z; j[4 * i + 3] = v.w;
        }
    }
}
// a * b + c of two 16-bit values and an fp32 sum (the product is not rounded)
template <typename X> __device__ __forceinline__ float fma_mixed(uint16_t a, uint16_t b, float c)
{
    float d;
    if constexpr (std::is_same<X, __half>::value) asm("fma.rn.f32.f16 %0, %1, %2, %3;" : "=f"(d) : "h"(a), "h"(b), "f"(c));
    else asm("fma.rn.f32.bf16 %0, %1, %2, %3;" : "=f"(d) : "h"(a), "h"(b), "f"(c));
    return d;
}
// weight i of a chunk as 16 bits (8-bit codes: f16, which holds every one of them)
template <typename W> struct Chunk16 {
    uint32_t w[8 / wsize<W>];
    __device__ __forceinline__ explicit Chunk16(const uint4 &c)
    {
        const uint32_t r[4] = {c.x, c.y, c.z, c.w};
        if constexpr (std::is_same<W, F8>::value) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = e4m3x2_to_f16x2(r[i >> 1] >> (16 * (i & 1)));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = r[i];
        }
    }
    __device__ __forceinline__ uint16_t at(int i) const { return (uint16_t)(w[i / 2] >> (16 * (i & 1))); }
};

// Steps a lane has in flight beside the ones it works on, and blocks of a kernel an SM should have room for: a step is four
// registers of weights and epc / 2 of channels, twice; two blocks (one of the kernel before) have 64 registers a thread.
__host__ __device__ constexpr int sp_unroll(int nacc, int epc) { return (nacc <= 8 && epc <= 2) || (nacc <= 4 && epc <= 4) ? 4 : 2; }
__host__ __device__ constexpr int sp_blocks(int nacc, int epc) { return nacc <= 8 && epc <= 8 ? 2 : 1; }
// a block of twice the threads has 64 registers a thread too: no more sums than fit
__host__ __device__ constexpr bool sp_wide(int nacc) { return nacc <= 32; }

// The tokens of channel j, two a word
template <typename X, int TT> __device__ __forceinline__ void load_tokens(const X *xs, uint32_t j, uint32_t (&xw)[TT > 1 ? TT / 2 : 1])
{
    const X *xp = xs + j * TT;
    if constexpr (TT == 1) xw[0] = *reinterpret_cast<const uint16_t *>(xp);
    else if constexpr (TT == 2) xw[0] = *reinterpret_cast<const uint32_t *>(xp);
    else if constexpr (TT == 4) { const uint2 v = *reinterpret_cast<const uint2 *>(xp); xw[0] = v.x; xw[1] = v.y; }
    else { const uint4 v = *reinterpret_cast<const uint4 *>(xp); xw[0] = v.x; xw[1] = v.y; xw[2] = v.z; xw[3] = v.w; }
}

// The sums of one bundle's rows without the fillers: `steps` steps from val and idx on, n entries of this lane's row. Same order
// of additions as in the kernel, so a row without infinities gets the value it has without them. Out of line, to keep its
// registers out of the main loop.
template <typename W, int NBK, int TT>
__device__ __noinline__ void sums_without_fillers(const typename XOf<W>::type *xs, const uint8_t *val, const uint16_t *idx, uint32_t steps, uint32_t n,
                                                  int lanes, int C, float *sums, int *status)
{
    using X = typename XOf<W>::type;
    constexpr int NACC = NBK * TT, EPC = 16 / (NBK * wsize<W>);
    const uint32_t lane = threadIdx.x & 31, own = lane & (uint32_t)(lanes - 1);
    float acc[NACC];
#pragma unroll
    for (float &v : acc) v = 0.f;
#pragma unroll 1
    for (uint32_t s = 0; s < steps; ++s) {
        const uint32_t first = (s * (uint32_t)lanes + own) * EPC;
        if (first >= n) continue;
        const Chunk16<W> w(__ldg(reinterpret_cast<const uint4 *>(val) + (size_t)s * 32 + lane));
        uint32_t j[EPC > 1 ? EPC / 2 : 1];
        load_channels<EPC>(idx + ((size_t)s * 32 + lane) * EPC, j);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
            const uint32_t c = EPC == 1 ? j[0] : (e & 1) ? j[e / 2] >> 16 : j[e / 2] & 0xffffu;
            if (first + e >= n || !UBP_CHK_SMEM((int)c < C, status)) continue;
            uint32_t xw[TT > 1 ? TT / 2 : 1];
            load_tokens<X, TT>(xs, c, xw);
#pragma unroll
            for (int i = 0; i < NACC; ++i)
                acc[i] = fma_mixed<X>(w.at(e * NBK + i / TT), (uint16_t)(xw[i % TT / 2] >> (16 * (i % TT & 1))), acc[i]);
        }
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < NACC; ++i) {
        for (int o = 1; o < lanes; o <<= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
        if (own == 0) sums[i] = acc[i];
    }
}

template <typename W, int NBK, int TT, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS > SP_THREADS ? 1 : sp_blocks(NBK * TT, 16 / (NBK * wsize<W>)))
ubp_linear_sparse_kernel(const SpArgs p)
{
    using X = typename XOf<W>::type;
    constexpr int NACC = NBK * TT, EPC = 16 / (NBK * wsize<W>);     // accumulators of a start row; entries of a chunk
    constexpr int U = sp_unroll(NACC, EPC);
    const LinearArgs &a = p.a;
    extern __shared__ __align__(16) uint8_t smem[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const int rb = 32 / p.lanes;                                    // start rows of a bundle
    const int fb = (a.F + rb - 1) / rb;                             // features in groups of rb: this block's share of them
    const int f0 = (int)((int64_t)fb * blockIdx.x / gridDim.x) * rb, fe = (int)((int64_t)fb * (blockIdx.x + 1) / gridDim.x) * rb;
    const int nf = (fe < a.F ? fe : a.F) - f0;
    const int64_t t0 = (int64_t)blockIdx.y * TT;
    const int nt = a.T - t0 < TT ? (int)(a.T - t0) : TT;
    const int nseg = a.gated ? 2 : 1;
    // bundles of row range q: those with start rows in q F + f0 - (NBK - 1) .. q F + f0 + nf
    const int lo0 = (f0 - (NBK - 1) > 0 ? f0 - (NBK - 1) : 0) / rb, n0 = (f0 + nf + rb - 1) / rb - lo0;
    const int lo1 = (a.F + f0 - (NBK - 1) > 0 ? a.F + f0 - (NBK - 1) : 0) / rb, n1 = nseg == 2 ? (a.F + f0 + nf + rb - 1) / rb - lo1 : 0;
    const int ntask = nf > 0 ? n0 + n1 : 0;

    // shared memory: activations [channel][TT], sums of start rows [range][row][NBK][TT]
    X *xs = reinterpret_cast<X *>(smem);
    float *part = reinterpret_cast<float *>(smem + (((size_t)a.C * TT * 2 + 31) & ~(size_t)15));

    const int lane = threadIdx.x & 31, warp = (int)threadIdx.x >> 5;
    struct Batch { uint4 val[U]; uint32_t j[U][EPC > 1 ? EPC / 2 : 1]; };
    const uint4 *val = reinterpret_cast<const uint4 *>(p.val) + lane;
    const uint16_t *idx = p.idx + lane * EPC;
    auto load = [&](uint32_t s, uint32_t s1, Batch &b) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + u < s1) {
                b.val[u] = __ldg(val + (size_t)(s + u) * 32);
                load_channels<EPC>(idx + (size_t)(s + u) * (32 * EPC), b.j[u]);
            }
    };
    auto bundle_of = [&](int task) { return task < n0 ? lo0 + task : lo1 + (task - n0); };
    int task = warp;
    uint32_t s = 0, s1 = 0;
    Batch cur;
    auto steps_of = [&](int task, uint32_t &s, uint32_t &s1) {
        const uint32_t first = __ldg(p.off + bundle_of(task)), end = __ldg(p.off + bundle_of(task) + 1);
        if (!UBP_CHK_SMEM(first <= end && end <= p.steps, a.status)) return;
        s = first; s1 = end;
    };
    if (task < ntask) steps_of(task, s, s1);
    load(s, s1, cur);

    asm volatile("griddepcontrol.wait;" ::: "memory");
    // ---- activations
    {
        constexpr int xb = wsize<W>;
        const uint8_t *x = static_cast<const uint8_t *>(a.x) + t0 * a.ldx * xb;
        if (TT == 1 && reinterpret_cast<uintptr_t>(x) % (8 * xb) == 0) {
            // one token: eight channels a thread
            for (int c = 8 * (int)threadIdx.x; c < a.C; c += 8 * THREADS) {
                if (c + 8 <= a.C) {
                    if constexpr (xb == 2) {
                        *reinterpret_cast<uint4 *>(xs + c) = *reinterpret_cast<const uint4 *>(x + (size_t)c * 2);
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2 *>(x + c);
                        *reinterpret_cast<uint4 *>(xs + c) = make_uint4(e4m3x2_to_f16x2(v.x), e4m3x2_to_f16x2(v.x >> 16), e4m3x2_to_f16x2(v.y), e4m3x2_to_f16x2(v.y >> 16));
                    }
                } else {
                    for (int e = c; e < a.C; ++e) {
                        if constexpr (xb == 2) reinterpret_cast<uint16_t *>(xs)[e] = reinterpret_cast<const uint16_t *>(x)[e];
                        else reinterpret_cast<uint16_t *>(xs)[e] = (uint16_t)e4m3x2_to_f16x2(x[e]);
                    }
                }
            }
        } else {
            // two channels a thread
            const bool pair = (reinterpret_cast<uintptr_t>(x) % (2 * xb) == 0) && (a.ldx * xb) % (2 * xb) == 0;
#pragma unroll 4
            for (int c = 2 * (int)threadIdx.x; c < a.C; c += 2 * THREADS) {
                const bool two = c + 1 < a.C;
                uint32_t v[TT];                                     // two channels of token t as two 16-bit values
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    v[t] = 0;
                    if (t < nt) {
                        const uint8_t *s = x + ((int64_t)t * a.ldx + c) * xb;
                        if constexpr (xb == 2) {
                            if (pair && two) v[t] = *reinterpret_cast<const uint32_t *>(s);
                            else v[t] = *reinterpret_cast<const uint16_t *>(s) | (two ? (uint32_t)*reinterpret_cast<const uint16_t *>(s + 2) << 16 : 0u);
                        } else {
                            if (pair && two) v[t] = *reinterpret_cast<const uint16_t *>(s);
                            else v[t] = s[0] | (two ? (uint32_t)s[1] << 8 : 0u);
                        }
                    }
                }
                if constexpr (xb == 1) {
#pragma unroll
                    for (int t = 0; t < TT; ++t) v[t] = e4m3x2_to_f16x2(v[t]);
                }
                uint32_t *d = reinterpret_cast<uint32_t *>(xs + (size_t)c * TT);      // (one channel past C is inside the padding)
                if constexpr (TT == 1) {
                    d[0] = v[0];
                } else {
                    uint32_t o[TT];
#pragma unroll
                    for (int t = 0; t < TT / 2; ++t) {
                        o[t] = __byte_perm(v[2 * t], v[2 * t + 1], 0x5410);
                        o[TT / 2 + t] = __byte_perm(v[2 * t], v[2 * t + 1], 0x7632);
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (h == 0 || two) {
                            uint32_t *dh = d + h * (TT / 2);
                            const uint32_t *oh = o + h * (TT / 2);
                            if constexpr (TT == 2) dh[0] = oh[0];
                            else if constexpr (TT == 4) *reinterpret_cast<uint2 *>(dh) = make_uint2(oh[0], oh[1]);
                            else *reinterpret_cast<uint4 *>(dh) = make_uint4(oh[0], oh[1], oh[2], oh[3]);
                        }
                }
            }
        }
    }
    __syncthreads();

    // ---- this warp's bundles
    float acc[NACC];                                                // [row of the block][token]
#pragma unroll
    for (float &v : acc) v = 0.f;
    while (task < ntask) {
        uint32_t ns = s + U, ns1 = s1;
        int ntask_ = task;
        if (ns >= s1) {
            ntask_ += (THREADS / 32);
            ns = ns1 = 0;
            if (ntask_ < ntask) steps_of(ntask_, ns, ns1);
        }
        Batch next;
        load(ns, ns1, next);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s + u >= s1) break;
            const Chunk16<W> w(cur.val[u]);
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
                const uint32_t j = EPC == 1 ? cur.j[u][0] : (e & 1) ? cur.j[u][e / 2] >> 16 : cur.j[u][e / 2] & 0xffffu;
                if (!UBP_CHK_SMEM((int)j < a.C, a.status)) continue;
                uint32_t xw[TT > 1 ? TT / 2 : 1];
                load_tokens<X, TT>(xs, j, xw);
#pragma unroll
                for (int b = 0; b < NBK; ++b)
#pragma unroll
                    for (int t = 0; t < TT; ++t)
                        acc[b * TT + t] = fma_mixed<X>(w.at(e * NBK + b), (uint16_t)(xw[t / 2] >> (16 * (t & 1))), acc[b * TT + t]);
            }
        }
        if (ntask_ != task) {
            // the bundle's last batch: join the lanes of each row. In the first three steps a lane keeps half of its sums and
            // hands over the other half as long as it has more than one.
            int at = 0;
#pragma unroll
            for (int o = 1, m = NACC; o < 8; o <<= 1) {
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
            constexpr int left = NACC >= 8 ? NACC / 8 : 1;
            for (int o = 8; o < p.lanes; o <<= 1)
#pragma unroll
                for (int i = 0; i < left; ++i) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
            // one lane per sum writes it (with fewer sums than lanes several lanes hold the same one)
            const int own = lane & (p.lanes - 1);
            float *dst = part + ((size_t)task * rb + lane / p.lanes) * NACC + at;
            if (own < (NACC >= 8 ? 8 : NACC) &&
                UBP_CHK_SMEM((uint64_t)(reinterpret_cast<uint8_t *>(dst + left) - smem) <= tc::dbg_dynamic_smem(), a.status)) {
#pragma unroll
                for (int i = 0; i < left; ++i) dst[i] = acc[i];
            }
            float none = 0.f;                                       // (not zero: an infinity or NaN among the sums)
#pragma unroll
            for (int i = 0; i < left; ++i) none = fmaf(acc[i], 0.f, none);
            if (__any_sync(0xffffffffu, !(none == 0.f))) {
                const int row = bundle_of(task) * rb + lane / p.lanes;
                uint32_t first = 0, end = 0;
                steps_of(task, first, end);
                sums_without_fillers<W, NBK, TT>(xs, p.val + (size_t)first * 512, p.idx + (size_t)first * (32 * EPC), end - first,
                                                 row < a.M ? __ldg(p.cnt + row) : 0u, p.lanes, a.C,
                                                 part + ((size_t)task * rb + lane / p.lanes) * NACC, a.status);
            }
#pragma unroll
            for (float &v : acc) v = 0.f;
        }
        task = ntask_; s = ns; s1 = ns1;
        cur = next;
    }
    __syncthreads();
    // ---- output rows and epilogue: neighbouring threads hold neighbouring features
    for (int i = threadIdx.x; i < nf * nt; i += THREADS) {
        const int t = TT == 1 ? 0 : i / nf, f = i - t * nf;
        float z[2] = {0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (q == nseg) break;
            const int row = q * a.F + f0 + f;
            if (!UBP_CHK_GMEM(row < a.M && f0 + f < a.F && t0 + t < a.T, a.status)) break;
            const float *src = part + ((size_t)(q ? n0 : 0) * rb + row - (q ? lo1 : lo0) * rb) * NACC + t;
            const float ws = std::is_same<W, F8>::value ? a.xs[t0 + t] * p.wscale[row] : 1.f, b0 = a.bias ? a.bias[row] : 0.f;
            float sum = 0.f;
#pragma unroll
            for (int b = 0; b < NBK; ++b)
                if (row - b >= 0) sum += src[-b * (NACC - TT)];       // start row row - b, its weight b: (-b rows + b) * TT
            z[q] = sum * ws + b0;
        }
        float v = apply_act(z[0], a.act, p.ydt);
        if (nseg == 2) v *= z[1];
        if (a.res) v += load_elem(a.res, (t0 + t) * a.ldr + f0 + f, p.ydt);
        store_elem(a.y, (t0 + t) * a.ldy + f0 + f, v, p.ydt);
    }
}

template <typename W, int NBK, int TT, int THREADS>
int launch_n(const SpArgs &p, int64_t chunks, size_t smem, cudaStream_t stream)
{
    const auto kern = ubp_linear_sparse_kernel<W, NBK, TT, THREADS>;
    static std::atomic<bool> done[64] = {};          // (calls come from any thread)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = -1;
    if (dev < 0 || dev >= 64 || !done[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SP_SMEM);
        if (e != cudaSuccess) { set_last_cuda_error((int)e); return UBP_E_CUDA; }
        if (dev >= 0 && dev < 64) done[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.grid, (unsigned)chunks);
    cfg.blockDim = dim3(THREADS);
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

template <typename W, int NBK, int TT>
int launch_t(const SpArgs &p, int64_t chunks, size_t smem, cudaStream_t stream)
{
    if constexpr (sp_wide(NBK * TT))
        if (p.wide) return launch_n<W, NBK, TT, 2 * SP_THREADS>(p, chunks, smem, stream);
    return launch_n<W, NBK, TT, SP_THREADS>(p, chunks, smem, stream);
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

// The power of two that takes the tokens in as few blocks as eight would, and whose activations fit (a token of the longest
// row, 65536 channels, is 128 KB).
void linear_sparse_tokens(const ubp_linear_plan *p, int64_t T, int *tokens, int64_t *groups)
{
    const int64_t chunks = (T + SP_MAX_TOKENS - 1) / SP_MAX_TOKENS, per = chunks ? (T + chunks - 1) / chunks : 1;
    int t = 1;
    while (t < per) t *= 2;
    while (t > 1 && (size_t)p->C * t * 2 > SP_X) t /= 2;
    *tokens = t;
    *groups = (T + t - 1) / t;
}

int launch_linear_sparse(const ubp_linear_plan *pl, const LinearArgs &a, int y_dtype, int sms, void *stream)
{
    SpArgs p;
    p.a = a;
    p.wscale = reinterpret_cast<const float *>(pl->dev + pl->img.scale_off);
    p.off = reinterpret_cast<const uint32_t *>(pl->dev + pl->img.off_off);
    p.idx = reinterpret_cast<const uint16_t *>(pl->dev + pl->img.idx_off);
    p.val = pl->dev + pl->img.val_off;
    p.steps = (uint32_t)pl->img.steps;
    p.cnt = reinterpret_cast<const uint32_t *>(pl->dev + pl->img.cnt_off);
    p.ydt = y_dtype;
    const int nbk = pl->img.nbk, nseg = a.gated ? 2 : 1;
    int TT;
    int64_t nchunk;
    linear_sparse_tokens(pl, a.T, &TT, &nchunk);
    if (nchunk > 65535) return UBP_E_UNSUPPORTED;
    // Blocks per chunk of tokens: together one for every SM, and not one less while there are rows for it: an SM without a
    // block has room for two of the next launch (whose blocks come early, see above), and those two take twice the time of
    // the others. Large layers: as many rows as shared memory leaves room for.
    const int rb = 32 / pl->img.lanes;
    const int64_t fb = ((int64_t)a.F + rb - 1) / rb;
    // A layer whose loads take long gains more from twice the loads under way on an SM than from the next launch's early start,
    // from some 18 MB of kept weights on: two blocks an SM for a token and blocks of up to four rows, whose neighbours'
    // recomputed start rows are few (bf16, blocks of 4: 25 MB 6.1 us, 6.8 with one, 6.6 with one of twice the threads; 15 MB
    // 5.7, 5.1, 5.3), else a block of twice the threads (f16, blocks of 8, 45 MB: a token 11.0 us, 13.3 with 512 threads, 12.4
    // with two blocks; two tokens 14.3, 19.9, 27; 4 tokens on the 25 MB 8.7, 10.5, 13.4).
    const size_t kept = (size_t)pl->img.entries * (nbk * dtype_size(pl->dtype) + 2);
    const bool large = kept >= ((size_t)18 << 20), two = large && TT == 1 && nbk <= 4 && nchunk == 1 && pl->C <= SP_TWO_C;
    p.wide = large && !two;
    int64_t grid = ((two ? 2 : 1) * sms + nchunk - 1) / nchunk;
    size_t smem;
    for (;; grid *= 2) {
        if (grid > fb) grid = fb;
        const int64_t span = (fb + grid - 1) / grid + (nbk - 1 + rb - 1) / rb + 1;      // bundles of a range at most
        smem = (((size_t)a.C * TT * 2 + 31) & ~(size_t)15) + (size_t)nseg * span * rb * nbk * TT * 4;
        if (smem <= SP_SMEM) break;
        if (grid == fb) return UBP_E_UNSUPPORTED;
    }
    p.lanes = pl->img.lanes;
    p.grid = (int)grid;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (pl->dtype) {
        case UBP_BF16: return launch_w<__nv_bfloat16>(p, nbk, TT, nchunk, smem, st);
        case UBP_F16: return launch_w<__half>(p, nbk, TT, nchunk, smem, st);
        default: return launch_w<F8>(p, nbk, TT, nchunk, smem, st);
    }
}

}  // namespace ubp
