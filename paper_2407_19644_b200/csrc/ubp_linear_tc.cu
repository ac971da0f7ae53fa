// Token-major product with a block-pruned weight on the tensor cores: the densified weight, bf16 / f16 / e4m3 operands as
// they are, fp32 accumulators in tensor memory. Both operands are K-major in the 128-byte swizzle: 64 (16-bit) or 128
// (8-bit) values of a row = one 128-byte line = a "chunk", four MMAs of 32 bytes each. TMA brings the lines, out-of-range
// rows and channels as zeros.
//
// ubp_linear_few_kernel -- up to some hundred tokens, and more of them where the pair kernel's large tiles would leave SMs
//   idle (777 tokens x 1500 x 1003: 120 blocks, 12.3 us; 48 pairs 14.8): bound by reading the dense weight, so every SM has to
//   stream.
//   The weight is the A operand (128 rows of it per block: with tokens as A the tensor core would read 128 mostly empty
//   rows per MMA for a handful of weight rows), the tokens are B (N = tokens rounded up to 16). S blocks of a cluster split
//   the reduction; partial sums meet in distributed shared memory, and rank k finishes its share of the tokens.
// ubp_linear_many_kernel -- many tokens: bound by the tensor cores. A CTA pair owns 256 tokens x 256 features (cta_group::2,
//   each CTA stages its 128 tokens and half of the features), persistent, two accumulators so that the epilogue of one tile
//   runs under the main loop of the next. Tokens are the accumulator's lanes: a thread holds one token's features, so a
//   gated layer's gate and up columns (interleaved in groups of 16 by the plan) meet in one thread; the finished values
//   turn through 4 KB of shared memory per warp so that stores and residual loads are whole 64-byte runs.
//
// Rows of x past the last token are zeros or another token's data; each touches its own output row only. The reduction's
// padding is zero on the weight side AND on the x side (TMA fills channels past C with zeros), so nothing outside x is read.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <mutex>
#include <type_traits>

#include "ubp_internal.h"
#include "ubp_linear.h"
#include "ubp_linear_epilogue.cuh"
#include "ubp_tc_common.cuh"

namespace ubp {
namespace {

using namespace tc;

constexpr uint32_t LT_SWZ_128B = 2;
constexpr int LT_LINE = 128;                    // bytes of a row in one chunk
constexpr int LT_EPI_WARPS = 8;                 // warps 2..9
// Copies are issued by two threads, lane 0 of warp 0 (weights, and the announcement of a stage's bytes) and of the last warp
// (activations): an issue holds its thread for more than a hundred cycles, and with one thread that is what a chunk waits for.
constexpr int LT_X_WARP = 2 + LT_EPI_WARPS;
constexpr int LT_THREADS = (3 + LT_EPI_WARPS) * 32;
constexpr int LT_MAX_STAGES = 12;

struct TcLinArgs {
    LinearArgs a;
    const float *wscale;
    int ydt;
    int nk;              // chunks of the reduction
    int rows;            // dense rows that hold the layer (M, or 2 x F rounded up to 16)
    int vec4;            // rows of y and of the residual are aligned to four elements
    int unaligned_bias;  // 1: bias is not 16-byte aligned
    int group;           // pair kernel: token tiles that walk the features together
};

__device__ __forceinline__ uint64_t kmajor_desc(uint32_t saddr) { return make_desc(saddr, 16, 1024, LT_SWZ_128B); }

// instruction descriptor: D = f32; A, B both K-major and of one type: 16 bits (0 = f16, 1 = bf16), or e4m3 (code 0 too)
__device__ __forceinline__ uint32_t lin_idesc(int m, int n, int fmt)
{
    return (1u << 4) | ((uint32_t)fmt << 7) | ((uint32_t)fmt << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// One chunk: four MMAs over 4 x 32 bytes of the 128-byte lines; the whole warp calls, one elected lane issues.
#define UBP_LIN_MMA4(GROUP, KIND)                                                                                    \
    asm volatile(                                                                                                    \
        "{\n\t.reg .pred pe, pa, pt;\n\t.reg .b64 a, b;\n\t"                                                         \
        "elect.sync _|pe, 0xffffffff;\n\t"                                                                           \
        "setp.ne.b32 pa, %4, 0;\n\tsetp.eq.b32 pt, 0, 0;\n\t"                                                        \
        "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, pa;\n\t"                              \
        "add.s64 a, %1, 2;\n\tadd.s64 b, %2, 2;\n\t"                                                                 \
        "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], a, b, %3, pt;\n\t"                                \
        "add.s64 a, %1, 4;\n\tadd.s64 b, %2, 4;\n\t"                                                                 \
        "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], a, b, %3, pt;\n\t"                                \
        "add.s64 a, %1, 6;\n\tadd.s64 b, %2, 6;\n\t"                                                                 \
        "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], a, b, %3, pt;\n\t}"                               \
        ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory")

template <bool F8> __device__ __forceinline__ void mma4_cta1(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (F8) UBP_LIN_MMA4("1", "f8f6f4");
    else UBP_LIN_MMA4("1", "f16");
}
template <bool F8> __device__ __forceinline__ void mma4_cta2(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (F8) UBP_LIN_MMA4("2", "f8f6f4");
    else UBP_LIN_MMA4("2", "f16");
}
__device__ __forceinline__ void commit_one(uint32_t bar)     // whole warp calls, one elected lane issues
{
    asm volatile("{\n\t.reg .pred pe;\n\telect.sync _|pe, 0xffffffff;\n\t"
                 "@pe tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
// 16 bytes at this place in the shared memory of another block of the cluster
__device__ __forceinline__ float4 ld_rank4(const float *p, uint32_t rank)
{
    uint32_t a;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void add4(float (&z)[4], const float4 &v) { z[0] += v.x; z[1] += v.y; z[2] += v.z; z[3] += v.w; }
// four elements of a row, of which the first n exist; whole accesses where the row is aligned to them
template <typename T> __device__ __forceinline__ void load4(const T *p, int n, bool vec, float (&v)[4])
{
    if (vec) {
        if constexpr (sizeof(T) == 4) {
            const float4 q = *reinterpret_cast<const float4 *>(p);
            v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
        } else {
            const uint2 q = *reinterpret_cast<const uint2 *>(p);
            const float2 a = unpack2<T>(q.x), b = unpack2<T>(q.y);
            v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = j < n ? to_f32<T>(p[j]) : 0.f;
    }
}
template <typename T> __device__ __forceinline__ void store4(T *p, int n, bool vec, const float (&v)[4])
{
    if (vec) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
        else *reinterpret_cast<uint2 *>(p) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = from_f32<T>(v[j]);
    }
}

// A block whose waits ran out leaves nothing under way that could still write to the shared or tensor memory it gives up: the
// threads that issued copies wait for the last ones of every stage, and the warp that issued MMAs for those, a millisecond at
// most (a stage whose other half was never issued does not complete).
constexpr uint64_t LT_DRAIN_NS = 1000000;
__device__ __forceinline__ void drain_copies(const uint64_t *bar_full, int stages, int issued)
{
    int gave_up = 0;
    for (int f = issued > stages ? issued - stages : 0; f < issued; ++f)
        mbar_wait(smem_u32(&bar_full[f % stages]), (uint32_t)(f / stages) & 1u, &gave_up, LT_DRAIN_NS);
}

// ------------------------------------------------------------------ few tokens
constexpr uint32_t FEW_A = 128 * LT_LINE;       // weight lines of one chunk: 16 KB
// One block an SM (TC_PAIR_MIN_SMEM). Half the shared memory, so that the next launch's blocks could set up and start their
// weight copies beside these, was slower: 24 tokens on 4096 x 8192 f16 17.0 us against 15.4, the ring is then too short.
constexpr uint32_t FEW_BUDGET = 200 * 1024;
__host__ __device__ constexpr int few_kch(int nt) { return nt <= 128 ? 2 : 1; }       // chunks per stage
__host__ __device__ constexpr uint32_t few_stage(int nt) { return (uint32_t)few_kch(nt) * (FEW_A + (uint32_t)nt * LT_LINE); }
__host__ __device__ constexpr int few_stages(int nt)
{
    const int s = (int)(FEW_BUDGET / few_stage(nt));
    return s > LT_MAX_STAGES ? LT_MAX_STAGES : s;
}

// Epilogue of a few-token tile: every thread holds four features (32 threads a token, 16 of a gated layer); the epilogue
// warps load their scales and biases while the main loop runs.
struct FewCols {
    float w0[4], w1[4], b0[4], b1[4];
    int f, n, dl;                                               // first feature, features that exist, first dense row in the tile
};
template <bool F8>
__device__ __forceinline__ FewCols few_cols(const TcLinArgs &p, int rt, int tid)
{
    const LinearArgs &a = p.a;
    const int per = a.gated ? 16 : 32, o = (tid & (per - 1)) * 4;
    FewCols c;
    c.f = rt * (per * 4) + o;
    c.dl = a.gated ? (o >> 4) * 32 + (o & 15) : o;
    c.n = a.F - c.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = j < c.n ? c.f + j : a.F - 1, u = a.gated ? a.F + r : r;
        c.w0[j] = F8 ? __ldg(p.wscale + r) : 1.f;
        c.w1[j] = F8 ? __ldg(p.wscale + u) : 1.f;
        c.b0[j] = a.bias ? __ldg(a.bias + r) : 0.f;
        c.b1[j] = a.bias ? __ldg(a.bias + u) : 0.f;
    }
    return c;
}
// Tokens ta .. tb of the tile: the cluster's partial sums red[token][128], in the ranks' order, to y.
template <bool F8, typename T>
__device__ __forceinline__ void few_epilogue(const TcLinArgs &p, const FewCols &c, const float *red, int tid, int64_t t0, int ta, int tb, int S)
{
    const LinearArgs &a = p.a;
    if (c.n <= 0) return;
    const bool vec = p.vec4 && c.n >= 4;
    const int per = a.gated ? 16 : 32, step = LT_THREADS / per;
#pragma unroll 2
    for (int t = ta + tid / per; t < tb; t += step) {
        float z[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f}, r[4] = {0.f, 0.f, 0.f, 0.f};
        if (!UBP_CHK_GMEM(t0 + t < a.T && c.f < a.F && c.f + (vec ? 4 : 1) <= a.F, a.status)) continue;
        if (!UBP_CHK_SMEM((uint32_t)(t * 128 + c.dl + (a.gated ? 20 : 4)) * 4u <= tc::dbg_dynamic_smem(), a.status)) continue;
        const float *src = red + t * 128 + c.dl;
        if (a.res) load4(static_cast<const T *>(a.res) + (t0 + t) * a.ldr + c.f, c.n, vec, r);
        const float xs = F8 ? a.xs[t0 + t] : 1.f;
        if (S > 1) {
            for (int k = 0; k < S; ++k) {
                add4(z, ld_rank4(src, (uint32_t)k));
                if (a.gated) add4(u, ld_rank4(src + 16, (uint32_t)k));
            }
        } else {
            add4(z, *reinterpret_cast<const float4 *>(src));
            if (a.gated) add4(u, *reinterpret_cast<const float4 *>(src + 16));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            z[j] = (F8 ? z[j] * (xs * c.w0[j]) : z[j]) + c.b0[j];
            u[j] = (F8 ? u[j] * (xs * c.w1[j]) : u[j]) + c.b1[j];
        }
        apply_act<sizeof(T) == 4>(z, a.act);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = (a.gated ? z[j] * u[j] : z[j]) + r[j];
        store4(static_cast<T *>(a.y) + (t0 + t) * a.ldy + c.f, c.n, vec, z);
    }
}

// grid: (row tile, token tile, rank) with the rank fastest; clusters of S blocks. NT: tokens per tile (multiple of 16).
// T: type of y (an instance each: with three epilogues in one kernel 777 tokens on 1500 x 1003 took 12.4 us, 12.3 so).
template <bool F8, typename T>
__global__ void __launch_bounds__(LT_THREADS, 1)
ubp_linear_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const TcLinArgs p,
                      const int fmt, const int NT, const int ntt, const int S)
{
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    __shared__ __align__(8) uint64_t bar_full[LT_MAX_STAGES], bar_empty[LT_MAX_STAGES], bar_acc, bar_drain;
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const LinearArgs &a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)blockIdx.x % S, tile = (int)(blockIdx.x / S), rt = tile / ntt, tt = tile % ntt;
    const int64_t t0 = (int64_t)tt * NT;
    const int nt = a.T - t0 < NT ? (int)(a.T - t0) : NT;
    const int k0 = (int)((int64_t)p.nk * rank / S), k1 = (int)((int64_t)p.nk * (rank + 1) / S);
    const int KCH = few_kch(NT), stages = few_stages(NT);
    const uint32_t stage_bytes = few_stage(NT), boff = (uint32_t)KCH * FEW_A;
    const int nst = (k1 - k0 + KCH - 1) / KCH;
    const int line = F8 ? 128 : 64;                            // values per chunk
    uint32_t cols = 32;
    while (cols < (uint32_t)NT) cols <<= 1;

    auto issue_w = [&](int f) {
        const int st = f % stages;
        const uint32_t bar = smem_u32(&bar_full[st]);
        mbar_expect_tx(bar, stage_bytes);
        tma_load_3d(smem_u32(smem + (size_t)st * stage_bytes), &tmW, 0, rt * 128, k0 + f * KCH, bar);
    };
    // the ring's first weight lines are constants of the layer: under way before anything else
    // (the activations' bytes may land before a stage's bytes are announced: its phase cannot end before)
    const int pre = nst < stages ? nst : stages;
    if (threadIdx.x == 0) {
        prefetch_tensormap(&tmX);
        abort_flag = 0;
        for (int s = 0; s < stages; ++s) { mbar_init(smem_u32(&bar_full[s]), 1); mbar_init(smem_u32(&bar_empty[s]), 1); }
        mbar_init(smem_u32(&bar_acc), 1);
        mbar_init(smem_u32(&bar_drain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        for (int f = 0; f < pre; ++f) issue_w(f);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    // the next kernel of the stream may start once this one holds its tensor memory
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = tmem_base_slot;
    bool ok = true;
    int issued = 0;                                             // stages that this thread has issued copies for

    if (warp == 0 || warp == LT_X_WARP) {
        if (lane == 0) {
            auto issue_x = [&](int i) {
                const int st = i % stages;
                const uint32_t bar = smem_u32(&bar_full[st]);
                for (int u = 0; u < KCH; ++u)
                    tma_load_2d(smem_u32(smem + (size_t)st * stage_bytes + boff + (uint32_t)(u * NT * LT_LINE)), &tmX,
                                (k0 + i * KCH + u) * line, (int)t0, bar);
            };
            const bool w = warp == 0;
            asm volatile("griddepcontrol.wait;" ::: "memory");
            for (issued = w ? pre : 0; issued < nst; ++issued) {
                if (issued >= stages) ok = mbar_wait(smem_u32(&bar_empty[issued % stages]), (uint32_t)(issued / stages - 1) & 1u, &abort_flag);
                if (!ok) break;
                if (w) issue_w(issued);
                else issue_x(issued);
            }
        }
    } else if (warp == 1) {
        const uint32_t idesc = lin_idesc(128, NT, fmt);
        for (int i = 0; i < nst && ok; ++i) {
            const int st = i % stages;
            ok = mbar_wait(smem_u32(&bar_full[st]), (uint32_t)(i / stages) & 1u, &abort_flag);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t base = smem_u32(smem) + (uint32_t)st * stage_bytes;
            for (int u = 0; u < KCH; ++u)
                if (k0 + i * KCH + u < k1)
                    mma4_cta1<F8>(tmem, kmajor_desc(base + (uint32_t)u * FEW_A), kmajor_desc(base + boff + (uint32_t)(u * NT * LT_LINE)),
                                  idesc, (i > 0 || u > 0) ? 1u : 0u);
            __syncwarp();
            commit_one(smem_u32(&bar_empty[st]));
        }
        if (ok) commit_one(smem_u32(&bar_acc));
    }
    if (!(lane == 0 && (warp == 0 || warp == LT_X_WARP))) asm volatile("griddepcontrol.wait;" ::: "memory");
    float *red = reinterpret_cast<float *>(smem);              // [NT][128] partial sums, over the (finished) ring
    const int tid = (int)threadIdx.x;
    const FewCols fc = few_cols<F8>(p, rt, tid);
    if (warp >= 2 && warp < LT_X_WARP) {
        ok = mbar_wait_relaxed(smem_u32(&bar_acc), 0, &abort_flag);
        if (ok) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int q = warp & 3;
            for (int c = (warp - 2) >> 2; c < NT / 16; c += LT_EPI_WARPS / 4) {
                uint32_t r[16];
                tmem_ld16(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(c * 16), r);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                for (int i = 0; i < 16; ++i) red[(size_t)(c * 16 + i) * 128 + q * 32 + lane] = k1 > k0 ? __uint_as_float(r[i]) : 0.f;
            }
        }
    }
    if (!ok && lane == 0) atomicExch(a.status, 1);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (S > 1) cluster_sync();
    else __syncthreads();
    // ---- epilogue of this rank's share of the tokens
    {
        const int ta = (int)((int64_t)nt * rank / S), tb = (int)((int64_t)nt * (rank + 1) / S);
        few_epilogue<F8, T>(p, fc, red, tid, t0, ta, tb, S);
    }
    if (*(volatile int *)&abort_flag) {
        if (issued) drain_copies(bar_full, stages, issued);
        if (warp == 1) {
            int gave_up = 0;
            commit_one(smem_u32(&bar_drain));
            mbar_wait(smem_u32(&bar_drain), 0, &gave_up, LT_DRAIN_NS);
        }
        __syncwarp();
    }
    if (S > 1) cluster_sync();                                  // nobody leaves while its partial sums are being read
    else __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
    }
}

// ------------------------------------------------------------------ many tokens
constexpr int MANY_STAGES = 6;
constexpr uint32_t MANY_TURN = 32 * 32 * 4;      // staging of one epilogue warp
// Token tiles that walk the features together: as many as keep 32 MB of activations in L2, eight at least. Sustained, 8 / 16 /
// 32 / 64 tiles: 8192 tokens x 16384 x 4096 e4m3 (1 MB a tile) 439 / 432 / 428 / 428 us; 16384 x 8192 x 2048 bf16 (1 MB) 417 /
// 411 / 410 / 445; 8192 x 4096 x 4096 bf16 (2 MB) 207 / 207 / 223 / 223; 8192 x 4096 x 8192 bf16 (4 MB) 423 / 431.
constexpr int64_t MANY_GROUP_BYTES = 32 << 20;
constexpr int MANY_GROUP_LEAST = 8;
__host__ __device__ constexpr uint32_t many_stage(int nt) { return 128 * LT_LINE + (uint32_t)(nt / 2) * LT_LINE; }

// One warp's 32 tokens x 32 values -> y, with the residual. E elements an access (8, 4, 2 or 1: what the rows of y and of the
// residual are aligned to and the layer's features are a multiple of); 32 / E lanes hold a token's 32 values.
template <typename T, int E>
__device__ __forceinline__ void store_turned_e(const uint8_t *turn, const T *res, int64_t ldr, T *y, int64_t ldy, int nt, int nf, int lane,
                                               int *status)
{
    constexpr int LPR = 32 / E, UN = E >= 4 ? E / 2 : E == 2 ? 4 : 8;      // lanes a token; steps under way (E steps of E tokens)
    const int c = (lane % LPR) * E;
    if (c >= nf) return;
#pragma unroll 1
    for (int i0 = 0; i0 < 32 / E; i0 += UN) {
        float w[UN][E];
        if (res) {
#pragma unroll
            for (int i = 0; i < UN; ++i) {
                const int t = (i0 + i) * E + lane / LPR;
                if (t < nt) {
                    const T *p = res + t * ldr + c;
                    if constexpr (E == 8) load8(p, w[i]);
                    else if constexpr (E == 4) load4(p, 4, true, w[i]);
                    else if constexpr (E == 2 && sizeof(T) == 2) { const float2 v = unpack2<T>(*reinterpret_cast<const uint32_t *>(p)); w[i][0] = v.x; w[i][1] = v.y; }
                    else if constexpr (E == 2) { const float2 v = *reinterpret_cast<const float2 *>(p); w[i][0] = v.x; w[i][1] = v.y; }
                    else w[i][0] = to_f32<T>(*p);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int r = (i0 + i) * E + lane / LPR;
            if (r >= nt || !UBP_CHK_GMEM(r < 32 && c + E <= nf, status)) continue;
            float o[E];
            const uint8_t *row = turn + r * 128;
            if constexpr (E >= 4) {
#pragma unroll
                for (int h = 0; h < E / 4; ++h) {
                    const float4 v = *reinterpret_cast<const float4 *>(row + (((c / 4 + h) ^ (r & 7)) << 4));
                    o[4 * h] = v.x; o[4 * h + 1] = v.y; o[4 * h + 2] = v.z; o[4 * h + 3] = v.w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = *reinterpret_cast<const float *>(row + (((c >> 2) ^ (r & 7)) << 4) + ((c & 3) + e) * 4);
            }
            if (res) {
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] += w[i][e];
            }
            T *p = y + r * ldy + c;
            if constexpr (E == 8) store8(p, o);
            else if constexpr (E == 4) store4(p, 4, true, o);
            else if constexpr (E == 2 && sizeof(T) == 2) *reinterpret_cast<uint32_t *>(p) = pack2<T>(o[0], o[1]);
            else if constexpr (E == 2) *reinterpret_cast<float2 *>(p) = make_float2(o[0], o[1]);
            else *p = from_f32<T>(o[0]);
        }
    }
}
// trow, f0: the warp's first token and the chunk's first feature
template <typename T, bool VEC8>
__device__ __forceinline__ void store_turned(const uint8_t *turn, const LinearArgs &a, int64_t trow, int f0, int lane, int vec)
{
    const int nt = a.T - trow < 32 ? (int)(a.T - trow) : 32, nf = a.F - f0 < 32 ? a.F - f0 : 32;
    if (nt <= 0 || nf <= 0) return;
    const T *res = a.res ? static_cast<const T *>(a.res) + trow * a.ldr + f0 : nullptr;
    T *y = static_cast<T *>(a.y) + trow * a.ldy + f0;
    if constexpr (VEC8) {
        store_turned_e<T, 8>(turn, res, a.ldr, y, a.ldy, nt, nf, lane, a.status);
    } else {
        if (vec == 4) store_turned_e<T, 4>(turn, res, a.ldr, y, a.ldy, nt, nf, lane, a.status);
        else if (vec == 2) store_turned_e<T, 2>(turn, res, a.ldr, y, a.ldy, nt, nf, lane, a.status);
        else store_turned_e<T, 1>(turn, res, a.ldr, y, a.ldy, nt, nf, lane, a.status);
    }
}

// NT: features (dense rows) per tile, 128 or 256. vec: elements an access to y and the residual may take;
// VEC8: that is 8 (an instance of its own: the registers of the narrow forms cost the wide one 5 % in spills).
// F32: fp32 output (its activations beside the 16-bit ones in one instance cost those 2 to 5 %).
template <bool F8, int NT, bool VEC8, bool F32>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LT_THREADS, 1)
ubp_linear_many_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const TcLinArgs p,
                       const int fmt, const int ntm, const int ntn, const int vec)
{
    constexpr int S = MANY_STAGES;
    constexpr uint32_t STAGE = many_stage(NT), AB = 128 * LT_LINE;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    // identical layout in both CTAs: multicast commits and remote arrives address barriers by offset
    __shared__ __align__(8) uint64_t bar_full[S], bar_peer[S], bar_empty[S], bar_acc_full[2], bar_acc_empty[2], bar_drain;
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const LinearArgs &a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int npairs = (int)(gridDim.x >> 1), pair = (int)(blockIdx.x >> 1), ntiles = ntm * ntn;
    const int nmy = pair < ntiles ? (ntiles - pair + npairs - 1) / npairs : 0;
    const int line = F8 ? 128 : 64;
    auto tile_at = [&](int i, int &m, int &n) {
        const int t = pair + i * npairs, per = p.group * ntn, g = t / per, r = t - g * per;
        const int gm = ntm - g * p.group < p.group ? ntm - g * p.group : p.group;
        n = r / gm;
        m = g * p.group + (r - n * gm);
    };

    if (threadIdx.x == 0) {
        prefetch_tensormap(&tmW);
        prefetch_tensormap(&tmX);
        abort_flag = 0;
        for (int s = 0; s < S; ++s) {
            mbar_init(smem_u32(&bar_full[s]), 1);
            mbar_init(smem_u32(&bar_peer[s]), 1);              // leader: the other CTA's lines have landed
            mbar_init(smem_u32(&bar_empty[s]), 1);
        }
        mbar_init(smem_u32(&bar_drain), 1);
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&bar_acc_full[b]), 1);
            mbar_init(smem_u32(&bar_acc_empty[b]), 2 * LT_EPI_WARPS);    // leader only
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = tmem_base_slot;
    bool ok = true;
    int issued = 0;                                             // stages that this thread has issued copies for

    if (warp == 0 || warp == LT_X_WARP) {
        if (lane == 0) {
            auto issue_w = [&](int st, int n, int k) {
                const uint32_t bar = smem_u32(&bar_full[st]);
                mbar_expect_tx(bar, STAGE);
                tma_load_3d(smem_u32(smem + (size_t)st * STAGE + AB), &tmW, 0, n * NT + (int)rank * (NT / 2), k, bar);
            };
            auto issue_x = [&](int st, int m, int k) {
                tma_load_2d(smem_u32(smem + (size_t)st * STAGE), &tmX, k * line, m * 256 + (int)rank * 128, smem_u32(&bar_full[st]));
            };
            int m = 0, n = 0;
            const bool w = warp == 0;
            const int pre = w && nmy > 0 ? (p.nk < S ? p.nk : S) : 0;  // first tile: the ring's weight lines before the wait
            if (nmy > 0) tile_at(0, m, n);
            for (int k = 0; k < pre; ++k) issue_w(k, n, k);
            asm volatile("griddepcontrol.wait;" ::: "memory");
            int st = 0, round = 0;
            for (int i = 0; i < nmy && ok; ++i) {
                tile_at(i, m, n);
                for (int k = 0; k < p.nk; ++k, ++issued) {
                    if (issued >= pre) {
                        if (round > 0) {
                            ok = mbar_wait(smem_u32(&bar_empty[st]), (uint32_t)(round - 1) & 1u, &abort_flag);
                            if (!ok) break;
                        }
                        if (w) issue_w(st, n, k);
                        else issue_x(st, m, k);
                    }
                    if (++st == S) { st = 0; ++round; }
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t idesc = lin_idesc(256, NT, fmt);
            int st = 0;
            uint32_t ph = 0;
            for (int i = 0; i < nmy && ok; ++i) {
                const int b = i & 1;
                const uint32_t acc = tmem + (uint32_t)b * 256u;
                if (i >= 2) {
                    ok = mbar_wait(smem_u32(&bar_acc_empty[b]), (uint32_t)((i >> 1) - 1) & 1u, &abort_flag);
                    if (!ok) break;
                }
                for (int k = 0; k < p.nk; ++k) {
                    ok = mbar_wait(smem_u32(&bar_full[st]), ph, &abort_flag) && mbar_wait(smem_u32(&bar_peer[st]), ph, &abort_flag);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t base = smem_u32(smem) + (uint32_t)st * STAGE;
                    mma4_cta2<F8>(acc, kmajor_desc(base), kmajor_desc(base + AB), idesc, k > 0 ? 1u : 0u);
                    __syncwarp();
                    mma2_commit_both(smem_u32(&bar_empty[st]));
                    if (++st == S) { st = 0; ph ^= 1u; }
                }
                if (!ok) break;
                mma2_commit_both(smem_u32(&bar_acc_full[b]));
            }
        } else if (lane == 0) {
            // the other CTA: tell the leader that this CTA's lines of a stage have landed (its own tensor core reads them)
            int st = 0;
            uint32_t ph = 0;
            for (int f = 0; f < nmy * p.nk && ok; ++f) {
                ok = mbar_wait(smem_u32(&bar_full[st]), ph, &abort_flag);
                if (!ok) break;
                mbar_arrive_remote(smem_u32(&bar_peer[st]), 0);
                if (++st == S) { st = 0; ph ^= 1u; }
            }
        }
    } else {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        const int q = warp & 3, half = (warp - 2) >> 2;
        uint8_t *turn = smem + (size_t)S * STAGE + (size_t)(warp - 2) * MANY_TURN;     // [32 tokens][32 values] fp32, swizzled
        const int nchunk = a.gated ? NT / 64 : NT / 32;          // chunks of 32 output features
        for (int i = 0; i < nmy && ok; ++i) {
            const int b = i & 1;
            int m, n;
            tile_at(i, m, n);
            const int64_t trow = (int64_t)m * 256 + (int)rank * 128 + q * 32;        // first token of this warp
            const int64_t tl = trow + lane;
            const float xs = F8 ? (tl < a.T ? a.xs[tl] : 0.f) : 1.f;
            ok = mbar_wait_relaxed(smem_u32(&bar_acc_full[b]), (uint32_t)(i >> 1) & 1u, &abort_flag);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + (uint32_t)b * 256u + ((uint32_t)(q * 32) << 16);
            bool released = false;
            // 16 accumulator columns -> scaled and biased; `row` = weight row of the first
            auto scaled16 = [&](const uint32_t (&r)[16], int row, float (&z)[16]) {
#pragma unroll
                for (int j = 0; j < 16; ++j) z[j] = __uint_as_float(r[j]);
                if (row + 16 <= a.M && ((row | p.unaligned_bias) & 3) == 0) {
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        if (F8) {
                            const float4 s4 = __ldg(reinterpret_cast<const float4 *>(p.wscale + row + j));
                            z[j] *= xs * s4.x; z[j + 1] *= xs * s4.y; z[j + 2] *= xs * s4.z; z[j + 3] *= xs * s4.w;
                        }
                        if (a.bias) {
                            const float4 b4 = __ldg(reinterpret_cast<const float4 *>(a.bias + row + j));
                            z[j] += b4.x; z[j + 1] += b4.y; z[j + 2] += b4.z; z[j + 3] += b4.w;
                        }
                    }
                } else if (F8 || a.bias) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int o = row + j < a.M ? row + j : a.M - 1;                 // (rows past the layer are not stored)
                        if (F8) z[j] *= xs * __ldg(p.wscale + o);
                        if (a.bias) z[j] += __ldg(a.bias + o);
                    }
                }
            };
#pragma unroll 1
            for (int c = half; c < nchunk; c += 2) {
                const int f0 = (a.gated ? n * (NT / 2) : n * NT) + c * 32;           // first output feature of the chunk
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    float z[16];
                    uint32_t r[16];
                    if (a.gated) {
                        float u[16];
                        uint32_t r2[16];
                        tmem_ld16(acc + (uint32_t)(c * 64 + h * 32), r);
                        tmem_ld16(acc + (uint32_t)(c * 64 + h * 32 + 16), r2);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                        scaled16(r, f0 + h * 16, z);
                        scaled16(r2, a.F + f0 + h * 16, u);
                        apply_act<F32>(z, a.act);
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[j] *= u[j];
                    } else {
                        tmem_ld16(acc + (uint32_t)(c * 32 + h * 16), r);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                        scaled16(r, f0 + h * 16, z);
                        apply_act<F32>(z, a.act);
                    }
                    // turn: lane = token row writes its 16 values, 16-byte pieces XORed with the row
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<float4 *>(turn + lane * 128 + (((4 * h + j) ^ (lane & 7)) << 4)) = make_float4(z[4 * j], z[4 * j + 1], z[4 * j + 2], z[4 * j + 3]);
                }
                if (c + 2 >= nchunk) {                           // last read of this accumulator by this warp
                    released = true;
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    if (lane == 0) {
                        if (rank == 0) mbar_arrive(smem_u32(&bar_acc_empty[b]));
                        else mbar_arrive_remote(smem_u32(&bar_acc_empty[b]), 0);
                    }
                }
                __syncwarp();
                if constexpr (F32) store_turned<float, VEC8>(turn, a, trow, f0, lane, vec);
                else if (p.ydt == UBP_BF16) store_turned<__nv_bfloat16, VEC8>(turn, a, trow, f0, lane, vec);
                else store_turned<__half, VEC8>(turn, a, trow, f0, lane, vec);
                __syncwarp();
            }
            if (!released && lane == 0) {
                if (rank == 0) mbar_arrive(smem_u32(&bar_acc_empty[b]));
                else mbar_arrive_remote(smem_u32(&bar_acc_empty[b]), 0);
            }
        }
    }
    if (!ok && lane == 0) atomicExch(a.status, 1);
    // neither CTA frees tensor memory or leaves while the other could still be the target of the pair's MMAs or commits
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (*(volatile int *)&abort_flag) {
        if (issued) drain_copies(bar_full, S, issued);
        if (warp == 1 && rank == 0) {
            int gave_up = 0;
            mma2_commit_both(smem_u32(&bar_drain));
            mbar_wait(smem_u32(&bar_drain), 0, &gave_up, LT_DRAIN_NS);
        }
        __syncwarp();
    }
    cluster_sync();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// Rows of x that a tensor copy cannot take (not 16-byte aligned) -> [T][Kp] rows, zeros past C.
template <typename T>
__global__ void __launch_bounds__(256) ubp_linear_pad_kernel(const T *__restrict__ x, int64_t ldx, int64_t T_, int C, T *__restrict__ out, int Kp,
                                                              int *status)
{
    constexpr int E = 16 / (int)sizeof(T);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int groups = Kp / E;
    const int64_t n = T_ * groups;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t t = i / groups;
        const int c = (int)(i - t * groups) * E;
        if (!UBP_CHK_GMEM(t < T_ && c + E <= Kp, status)) continue;
        alignas(16) T v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = c + e < C ? x[t * ldx + c + e] : T(0);
        *reinterpret_cast<uint4 *>(out + t * Kp + c) = *reinterpret_cast<const uint4 *>(v);
    }
}

// ------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encoder()
{
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

int encode(CUtensorMap *tm, const void *base, int dtype, uint32_t rank, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box)
{
    const EncodeTiledFn enc = encoder();
    if (!enc) return UBP_E_CUDA;
    const cuuint32_t one[3] = {1, 1, 1};
    const CUtensorMapDataType t = dtype == UBP_E4M3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : dtype == UBP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const CUresult r = enc(tm, t, rank, const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) { set_last_cuda_error((int)cudaErrorInvalidValue); return UBP_E_CUDA; }
    return UBP_OK;
}
// weight: (values of a line, rows, lines) so that one copy brings several chunks
int encode_w(CUtensorMap *tm, const ubp_linear_plan *pl, int rows, int chunks)
{
    const int b = pl->dtype == UBP_E4M3 ? 1 : 2;
    const cuuint64_t dims[3] = {(cuuint64_t)(LT_LINE / b), (cuuint64_t)pl->img.Mp, (cuuint64_t)(pl->img.Kp * b / LT_LINE)};
    const cuuint64_t strides[2] = {(cuuint64_t)pl->img.Kp * b, LT_LINE};
    const cuuint32_t box[3] = {(cuuint32_t)(LT_LINE / b), (cuuint32_t)rows, (cuuint32_t)chunks};
    return encode(tm, pl->dev + pl->img.dense_off, pl->dtype, 3, dims, strides, box);
}
int encode_x(CUtensorMap *tm, const void *x, int dtype, int64_t ldx, int64_t T, int C, int rows)
{
    const int b = dtype == UBP_E4M3 ? 1 : 2;
    const cuuint64_t dims[2] = {(cuuint64_t)C, (cuuint64_t)T};
    // (a single row's stride is never used but has to be a valid one)
    const cuuint64_t strides[1] = {T > 1 ? (cuuint64_t)ldx * b : ((cuuint64_t)C * b + 15) & ~(cuuint64_t)15};
    const cuuint32_t box[2] = {(cuuint32_t)(LT_LINE / b), (cuuint32_t)rows};
    return encode(tm, x, dtype, 2, dims, strides, box);
}

int fail(cudaError_t e) { set_last_cuda_error((int)e); return UBP_E_CUDA; }

// dynamic shared memory once per device and kernel (calls come from any thread); one block per SM (see TC_PAIR_MIN_SMEM)
template <typename K> int allow_smem(K kern, std::atomic<bool> (&done)[64], size_t least)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = -1;
    if (dev >= 0 && dev < 64 && done[dev]) return UBP_OK;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024);
    if (e != cudaSuccess) return fail(e);
    int per_sm = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, LT_THREADS, least);
    if (e != cudaSuccess) return fail(e);
    if (per_sm != 1) return UBP_E_UNSUPPORTED;
    if (dev >= 0 && dev < 64) done[dev] = true;
    return UBP_OK;
}

template <bool F8, typename T>
int launch_few(const CUtensorMap &tmW, const CUtensorMap &tmX, const TcLinArgs &p, int fmt, int NT, int ntt, int S, cudaStream_t st)
{
    static std::atomic<bool> done[64] = {};
    const auto kern = ubp_linear_few_kernel<F8, T>;
    if (int rc = allow_smem(kern, done, TC_PAIR_MIN_SMEM)) return rc;
    size_t smem = (size_t)few_stages(NT) * few_stage(NT) + 1024;
    if (smem < TC_PAIR_MIN_SMEM) smem = TC_PAIR_MIN_SMEM;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.rows + 127) / 128 * ntt * S));
    cfg.blockDim = dim3(LT_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)S;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, tmW, tmX, p, fmt, NT, ntt, S);
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? UBP_OK : fail(e);
}

template <bool F8, int NT, bool VEC8, bool F32>
int launch_many(const CUtensorMap &tmW, const CUtensorMap &tmX, const TcLinArgs &p, int fmt, int sms, int vec, cudaStream_t st)
{
    static std::atomic<bool> done[64] = {};
    const auto kern = ubp_linear_many_kernel<F8, NT, VEC8, F32>;
    const size_t smem = (size_t)MANY_STAGES * many_stage(NT) + LT_EPI_WARPS * MANY_TURN + 1024;
    static_assert(MANY_STAGES * many_stage(128) + LT_EPI_WARPS * MANY_TURN + 1024 >= TC_PAIR_MIN_SMEM, "one block per SM");
    if (int rc = allow_smem(kern, done, smem)) return rc;
    const int64_t ntm = (p.a.T + 255) / 256, ntn = (p.rows + NT - 1) / NT;
    if (ntm * ntn > 0x7fffffff) return UBP_E_UNSUPPORTED;
    const int64_t pairs = ntm * ntn < sms / 2 ? ntm * ntn : sms / 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * pairs));
    cfg.blockDim = dim3(LT_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, tmW, tmX, p, fmt, (int)ntm, (int)ntn, vec);
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? UBP_OK : fail(e);
}

}  // namespace

bool linear_x_direct(const ubp_linear_plan *pl, const void *x, int64_t ldx, int64_t T)
{
    const int b = pl->dtype == UBP_E4M3 ? 1 : 2;
    return (reinterpret_cast<uintptr_t>(x) & 15) == 0 && (T <= 1 || ldx * b % 16 == 0);
}

int launch_linear_tc(const ubp_linear_plan *pl, const LinearArgs &args, int y_dtype, const LinearChoice &ch, void *workspace, int sms, void *stream)
{
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool f8 = pl->dtype == UBP_E4M3;
    const int b = f8 ? 1 : 2, fmt = pl->dtype == UBP_BF16 ? 1 : 0;
    TcLinArgs p;
    p.a = args;
    p.wscale = reinterpret_cast<const float *>(pl->dev + pl->img.scale_off);
    p.ydt = y_dtype;
    p.nk = pl->img.Kp * b / LT_LINE;
    p.unaligned_bias = (reinterpret_cast<uintptr_t>(args.bias) & 15) != 0;
    const int64_t group = MANY_GROUP_BYTES / ((int64_t)256 * pl->img.Kp * b);
    p.group = (int)(group > MANY_GROUP_LEAST ? group : MANY_GROUP_LEAST);
    p.rows = pl->gated ? (pl->F + 15) / 16 * 32 : pl->M;
    if (args.T > 0x7fffffff) return UBP_E_UNSUPPORTED;
    const uintptr_t ob = (uintptr_t)(y_dtype == UBP_F32 ? 4 : 2);
    auto rows_on = [&](const void *q, int64_t ld, uintptr_t n) { return (reinterpret_cast<uintptr_t>(q) & (n - 1)) == 0 && (args.T <= 1 || ((uint64_t)ld * ob) % n == 0); };
    p.vec4 = rows_on(args.y, args.ldy, 4 * ob) && (!args.res || rows_on(args.res, args.ldr, 4 * ob));
    const void *x = args.x;
    int64_t ldx = args.ldx;
    int C = pl->C;
    if (!linear_x_direct(pl, x, ldx, args.T)) {
        const int64_t n = args.T * (pl->img.Kp * b / 16);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((n + 255) / 256 < 8 * sms ? (n + 255) / 256 : 8 * sms));
        cfg.blockDim = dim3(256);
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        cudaError_t e = f8 ? cudaLaunchKernelEx(&cfg, ubp_linear_pad_kernel<uint8_t>, static_cast<const uint8_t *>(x), ldx, args.T, C, static_cast<uint8_t *>(workspace), pl->img.Kp, args.status)
                           : cudaLaunchKernelEx(&cfg, ubp_linear_pad_kernel<uint16_t>, static_cast<const uint16_t *>(x), ldx, args.T, C, static_cast<uint16_t *>(workspace), pl->img.Kp, args.status);
        if (e == cudaSuccess) e = cudaGetLastError();
        if (e != cudaSuccess) return fail(e);
        x = workspace; ldx = pl->img.Kp; C = pl->img.Kp;
    }
    CUtensorMap tmW, tmX;
    if (ch.kernel == LIN_FEW) {
        if (int rc = encode_w(&tmW, pl, 128, few_kch(ch.cols))) return rc;
        if (int rc = encode_x(&tmX, x, pl->dtype, ldx, args.T, C, ch.cols)) return rc;
        const int ntt = (int)((args.T + ch.cols - 1) / ch.cols);
        auto few = [&](auto f8_) {
            constexpr bool f = decltype(f8_)::value;
            switch (y_dtype) {
                case UBP_BF16: return launch_few<f, __nv_bfloat16>(tmW, tmX, p, fmt, ch.cols, ntt, ch.split, st);
                case UBP_F16: return launch_few<f, __half>(tmW, tmX, p, fmt, ch.cols, ntt, ch.split, st);
                default: return launch_few<f, float>(tmW, tmX, p, fmt, ch.cols, ntt, ch.split, st);
            }
        };
        return f8 ? few(std::true_type{}) : few(std::false_type{});
    }
    if (int rc = encode_w(&tmW, pl, ch.cols / 2, 1)) return rc;
    if (int rc = encode_x(&tmX, x, pl->dtype, ldx, args.T, C, 128)) return rc;
    int vec = 8;
    while (vec > 1 && !(pl->F % vec == 0 && rows_on(args.y, args.ldy, vec * ob < 16 ? vec * ob : 16) &&
                        (!args.res || rows_on(args.res, args.ldr, vec * ob < 16 ? vec * ob : 16)))) vec /= 2;
    auto by_out = [&](auto f8_, auto nt_, auto v_) {
        constexpr bool f = decltype(f8_)::value, v = decltype(v_)::value;
        constexpr int n = decltype(nt_)::value;
        return y_dtype == UBP_F32 ? launch_many<f, n, v, true>(tmW, tmX, p, fmt, sms, vec, st) : launch_many<f, n, v, false>(tmW, tmX, p, fmt, sms, vec, st);
    };
    auto by_vec = [&](auto f8_, auto nt_) { return vec == 8 ? by_out(f8_, nt_, std::true_type{}) : by_out(f8_, nt_, std::false_type{}); };
    auto by_tile = [&](auto f8_) { return ch.cols == 128 ? by_vec(f8_, std::integral_constant<int, 128>{}) : by_vec(f8_, std::integral_constant<int, 256>{}); };
    return f8 ? by_tile(std::true_type{}) : by_tile(std::false_type{});
}

}  // namespace ubp
