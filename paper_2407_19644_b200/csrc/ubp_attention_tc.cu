// Attention of many query rows over a paged cache on the tensor cores: prompts, their continuations, and a prefix that a batch
// shares.
//
//   S = Q K^T (128 rows x 128 keys, fp32 in tensor memory), P = 2^(S scale log2e - m) in 16 bits, O = O + P V (fp32 in tensor memory)
//
// A block owns 256 rows (tokens times heads of a group) in two tiles of 128 that share the staged keys and values: while one
// tile's scores go through the softmax, the tensor cores work on the other's products. Four warps a tile hold its softmax, a thread
// a row: scores come from tensor memory, weights go back over them and are the second product's A operand from there; nothing passes
// through shared memory. (Two threads a row, eight warps a tile: 5 % slower, the halves wait for one another in every step.)
// One warp issues the products, three the copies: a page of the cache is a TMA box (64 values x tokens), in the 128-byte swizzle, so
// that K is the K-major and V the MN-major operand as they lie in the cache.
// Measured on a prompt of 8192 (3100 to 3600 cycles a step; the products are 2048 of them): a tile's softmax takes 2000 -- 370 to
// bring the scores, 290 for the maximum, 1360 for the weights, with the special function unit busy for 1024 for each of the two
// tiles -- and then its next scores are 1100 away: the end of its product with V, and its product with K, behind the other tile's.
// In long runs the card reports its power limit. Tried: scores in two halves of 64 keys that are ready ahead (a product of 64
// columns takes 48 cycles, not 32: 9 to 20 % slower); the maximum beside weights by the old reference, repeated if that will not
// do (no difference); a part of the exponentials as polynomials (no difference, more of them slower).
// O is rescaled only when a score lies far enough above the row's reference (AttnRef: weights stay below 2^8, 2^12 in f16, sums far from
// overflow); the sum over the weights takes them before they are rounded to 16 bits.
// Steps are dealt to the blocks as in ubp_attention.h: one block an SM, the same number of key tiles for each.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <mutex>
#include <type_traits>

#include "ubp_attention_copy.cuh"
#include "ubp_attention_steps.cuh"
#include "ubp_f32x2.cuh"

namespace ubp {

namespace {

using namespace tc;

constexpr int AT_BN = 128, AT_TILE = 128, AT_THREADS = 384;
// Warps of the first warpgroup copy keys, issue products, copy values and queries; the others do the softmax. Registers a thread: 168 at the
// launch (384 threads), then 80 for the first warpgroup and 208 for the two others.
constexpr int AT_K_WARP = 0, AT_MMA_WARP = 1, AT_V_WARP = 2, AT_Q_WARP = 3, AT_SOFT_WARP = 4;
constexpr uint32_t AT_PANEL = 128 * 128;                       // 128 rows of 64 values
constexpr uint32_t AT_SWZ = 2;                                 // 128-byte swizzle
constexpr uint32_t AT_TURN = 32 * 128;                         // a softmax warp's: 128 bytes of each of its rows
__host__ __device__ constexpr int at_stages(int dp) { return dp == 128 ? 2 : 4; }
__host__ __device__ constexpr uint32_t at_part(int dp) { return (uint32_t)(dp / 64) * AT_PANEL; }
__host__ __device__ constexpr uint32_t at_smem(int dp) { return (2 + 2 * (uint32_t)at_stages(dp)) * at_part(dp) + 8 * AT_TURN + 1024; }
static_assert(at_smem(64) >= TC_PAIR_MIN_SMEM && at_smem(128) <= 226 * 1024, "one block an SM: a block holds all tensor memory");
static_assert(sizeof(AttnPlace<AT_THREADS>) <= 8 * AT_TURN, "lies there until the steps are dealt");

// N steps of 16 along the reduction: D (tensor memory) (+)= A B, A from shared memory, or the 16-bit values of tensor memory from
// column `a` on. The whole warp calls with equal arguments, one elected lane issues: from a branch of a single lane the operands
// had to be made uniform one by one, 120 cycles a product instead of the 64 that it takes. Few products wait in the tensor cores'
// queue, so what the issuing warp does between them is time lost: see `uniform`. (Two issuing warps, one a tile: their products
// interleave, both tiles wait for both: 12 to 25 % slower.)
#define AT_MMA_BEGIN "{\n\t.reg .pred pe, pa, pt;\n\t.reg .b64 x, y;\n\t.reg .b32 z;\n\telect.sync _|pe, 0xffffffff;\n\tsetp.ne.b32 pa, %4, 0;\n\tsetp.eq.b32 pt, 0, 0;\n\t"
#define AT_MMA_SS(X, Y, P) "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], " X ", " Y ", %3, " P ";\n\t"
#define AT_MMA_TS(X, Y, P) "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [" X "], " Y ", %3, " P ";\n\t"
__device__ __forceinline__ void mma_ss1(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(AT_MMA_BEGIN AT_MMA_SS("%1", "%2", "pa") "}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ss4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)     // 32 bytes a step
{
    asm volatile(AT_MMA_BEGIN AT_MMA_SS("%1", "%2", "pa")
                 "add.s64 x, %1, 2;\n\tadd.s64 y, %2, 2;\n\t" AT_MMA_SS("x", "y", "pt")
                 "add.s64 x, %1, 4;\n\tadd.s64 y, %2, 4;\n\t" AT_MMA_SS("x", "y", "pt")
                 "add.s64 x, %1, 6;\n\tadd.s64 y, %2, 6;\n\t" AT_MMA_SS("x", "y", "pt") "}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts4(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)     // 8 columns, 16 rows of 128 bytes a step
{
    asm volatile(AT_MMA_BEGIN AT_MMA_TS("%1", "%2", "pa")
                 "add.s32 z, %1, 8;\n\tadd.s64 y, %2, 128;\n\t" AT_MMA_TS("z", "y", "pt")
                 "add.s32 z, %1, 16;\n\tadd.s64 y, %2, 256;\n\t" AT_MMA_TS("z", "y", "pt")
                 "add.s32 z, %1, 24;\n\tadd.s64 y, %2, 384;\n\t" AT_MMA_TS("z", "y", "pt") "}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void commit_one(uint32_t bar)     // whole warp calls, one elected lane issues
{
    asm volatile("{\n\t.reg .pred pe;\n\telect.sync _|pe, 0xffffffff;\n\t"
                 "@pe tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// bits 0 .. n - 1
__device__ __forceinline__ uint32_t bits_below(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

// instruction descriptor: D = f32, A and B of one 16-bit type (0 = f16, 1 = bf16), A K-major, M = 128
__device__ __forceinline__ uint32_t at_idesc(int n, int fmt, int b_mn)
{
    return (1u << 4) | ((uint32_t)fmt << 7) | ((uint32_t)fmt << 10) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

struct AtBars {
    uint64_t q_full[2], q_empty[2], s_full[2], p_half[2], p_full[2], o_full[2];
    uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4], patch, drain;
};

// A value that all lanes of a warp have, so that the compiler knows: the issuing warp's loops, addresses and descriptors are then
// computed once a warp and not once a lane, and need no exchange before each product (in turn on one card: a prompt of 16384 under a
// window 986 -> 938 us, continuations 276 -> 268, ragged prompts 39.9 -> 37.6).
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// Segments of a block's steps: consecutive tiles of one item.
struct AtSegments {
    AttnSteps s;
    int n;
    __device__ __forceinline__ bool get()
    {
        n = s.tiles();
        return s.left > 0;
    }
    __device__ __forceinline__ void done(const AttnArgs &a) { s.advance(a, n); }
    // whether the item's second tile has rows
    __device__ __forceinline__ bool two(const AttnArgs &a) const { return s.c.q.n - s.c.rt * a.tpt > a.tpt / 2; }
};
// NK: head size in steps of 16 (the copies bring zeros past it)
template <typename T, int NK>
__global__ void __launch_bounds__(AT_THREADS, 1)
ubp_attention_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmQ,
                        const AttnArgs a)
{
    constexpr int DP = NK > 4 ? 128 : 64, ST = at_stages(DP);
    constexpr uint32_t PART = at_part(DP);
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    __shared__ __align__(8) AtBars bars;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
        abort_flag = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars.q_full[i]), 1);
            mbar_init(smem_u32(&bars.q_empty[i]), 1);
            mbar_init(smem_u32(&bars.s_full[i]), 1);
            mbar_init(smem_u32(&bars.p_half[i]), 4);
            mbar_init(smem_u32(&bars.p_full[i]), 4);
            mbar_init(smem_u32(&bars.o_full[i]), 1);
        }
        for (int i = 0; i < ST; ++i) {
            mbar_init(smem_u32(&bars.k_full[i]), 1);
            mbar_init(smem_u32(&bars.k_empty[i]), 1);
            mbar_init(smem_u32(&bars.v_full[i]), 1);
            mbar_init(smem_u32(&bars.v_empty[i]), 1);
        }
        mbar_init(smem_u32(&bars.patch), 1);
        mbar_init(smem_u32(&bars.drain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == AT_MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    const uint32_t tmem = (uint32_t)uniform((int)tmem_slot);
    asm volatile("griddepcontrol.wait;" ::: "memory");

    constexpr uint32_t TURN = (2 + 2 * ST) * PART;
    AttnDeal deal;
    AtSegments sg;
    bool ok = true;
    int filled = 0;                        // copy warps: stages filled so far
    if (!attn_locate<AT_THREADS>(a, *reinterpret_cast<AttnPlace<AT_THREADS> *>(smem + TURN), deal, sg.s)) sg.s.left = 0;
    const uint32_t s_q = smem_u32(smem), s_k = s_q + 2 * PART, s_v = s_k + ST * PART;

    if (warp < AT_SOFT_WARP) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        if (warp == AT_K_WARP || warp == AT_V_WARP) {
            const bool values = warp == AT_V_WARP;
            const int page_mask = (1 << a.pshift) - 1, box = imin(1 << a.pshift, AT_BN), nbox = AT_BN / box;
            const CUtensorMap *const tm = values ? &tmV : &tmK;
            uint64_t *const bar_full = values ? bars.v_full : bars.k_full, *const bar_empty = values ? bars.v_empty : bars.k_empty;
            const uint32_t ring = values ? s_v : s_k;
            int patches = 0;
            for (; ok && sg.get(); sg.done(a)) {
                const int kvh = sg.s.c.hu / a.chunks;
                const AttnTiles &t = sg.s.c.t;
                auto page_of = [&](int i) {     // (a lane a box)
                    return lane < nbox ? attn_box_page(a, t, sg.s.c.b, attn_tile_at(t, sg.s.c.tile + i) * AT_BN + lane * box, box) : a.pages;
                };
                int page = page_of(0);
                for (int i = 0; i < sg.n; ++i, ++filled) {
                    const int st = filled % ST, j0 = attn_tile_at(t, sg.s.c.tile + i) * AT_BN, ahead = i + 1 < sg.n ? page_of(i + 1) : 0;
                    // Places of a page whose keys no row sees: whatever they hold, a weight of 0 times it has to be 0, so the values
                    // there are overwritten with zeros before the product reads them.
                    const bool patch = values && ((j0 + AT_BN > t.end && (t.end & (box - 1))) ||                              // the last key
                                                  (j0 < a.kv0 && j0 + AT_BN > a.kv0 && (a.kv0 & (box - 1))) ||                // the call's first
                                                  (j0 < t.w0 && j0 + AT_BN > t.w0) ||                                         // the window
                                                  (j0 < a.sinks && j0 + AT_BN > a.sinks && j0 < t.w0));                       // first tokens
                    const uint32_t full = smem_u32(&bar_full[st]), dst = ring + (uint32_t)st * PART, bar = patch ? smem_u32(&bars.patch) : full;
                    if (filled >= ST) ok = attn_wait(smem_u32(&bar_empty[st]), (uint32_t)(filled / ST - 1) & 1u, &abort_flag);
                    if (!ok) break;
                    if (lane == 0) mbar_expect_tx(bar, PART);
                    for (int b = 0; b < nbox; ++b) {
                        const int pg = __shfl_sync(0xffffffffu, page, b);
                        if (lane == 0) {
#pragma unroll
                            for (int p = 0; p < DP / 64; ++p)
                                tma_load_4d(dst + (uint32_t)p * AT_PANEL + (uint32_t)(b * box) * 128u, tm, p * 64, (j0 + b * box) & page_mask, kvh, pg, bar);
                        }
                    }
                    __syncwarp();
                    if (patch) {
                        ok = attn_wait(bar, (uint32_t)patches & 1u, &abort_flag);
                        ++patches;
                        if (!ok) break;
                        for (int x = lane; x < AT_BN * DP / 8; x += 32) {
                            const int r = x / (DP / 8), c = x % (DP / 8), j = j0 + r;
                            if (!(j >= a.kv0 && j < t.end && (j >= t.w0 || j < a.sinks)))
                                *reinterpret_cast<uint4 *>(smem + (dst - s_q) + (uint32_t)(c / 8) * AT_PANEL + (uint32_t)r * 128u +
                                                           (uint32_t)(c % 8) * 16u) = make_uint4(0, 0, 0, 0);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) mbar_arrive(full);
                    }
                    page = ahead;
                }
            }
        } else if (warp == AT_Q_WARP) {
            int queries[2] = {0, 0};
            for (; ok && sg.get(); sg.done(a)) {
                const int kvh = sg.s.c.hu / a.chunks;
                // the item's queries, as soon as the products of the one before it have read theirs: the rows of a tile are the
                // group's heads of consecutive tokens, one box (rows past the sequence's end, whatever they hold, are not stored)
                for (int i = 0; ok && i < (sg.two(a) ? 2 : 1); ++i) {
                    if (queries[i]++) ok = attn_wait(smem_u32(&bars.q_empty[i]), (uint32_t)queries[i] & 1u, &abort_flag);
                    if (!ok) break;
                    const int per = a.tpt / 2, g0 = (sg.s.c.hu - kvh * a.chunks) * a.gc;
                    const uint32_t dst = s_q + (uint32_t)i * PART, bar = smem_u32(&bars.q_full[i]);
                    if (lane == 0) {
                        mbar_expect_tx(bar, (uint32_t)(DP / 64 * a.gc * per) * 128u);
#pragma unroll
                        for (int p = 0; p < DP / 64; ++p)
                            tma_load_3d(dst + (uint32_t)p * AT_PANEL, &tmQ, p * 64, kvh * a.G + g0, sg.s.c.q.s + sg.s.c.rt * a.tpt + i * per, bar);
                    }
                    __syncwarp();
                }
            }
        } else if (warp == AT_MMA_WARP) {
            constexpr uint32_t fmt = std::is_same_v<T, __nv_bfloat16> ? 1 : 0;
            const uint32_t id_s = at_idesc(AT_BN, fmt, 0), id_o = at_idesc(NK * 16, fmt, 1);
            const uint64_t q0 = make_desc(s_q, 16, 1024, AT_SWZ), k0 = make_desc(s_k, 16, 1024, AT_SWZ), v0 = make_desc(s_v, AT_PANEL, 1024, AT_SWZ);
            uint32_t q_phase[2] = {0, 0}, p_phase[2] = {0, 0}, k_phase = 0, v_phase = 0;
            int ks = 0, vs = 0;                                  // stages of the next keys and values
            auto scores = [&](int i) {                            // S_i = Q_i K^T
                const uint64_t q = q0 + (uint64_t)((uint32_t)i * (PART >> 4)), k = k0 + (uint64_t)((uint32_t)ks * (PART >> 4));
                const uint32_t d = tmem + (uint32_t)i * 128u;
                mma_ss4(d, q, k, id_s, 0);
                if constexpr (NK == 8) mma_ss4(d, q + (AT_PANEL >> 4), k + (AT_PANEL >> 4), id_s, 1);
                else {
#pragma unroll
                    for (int n = 4; n < NK; ++n) mma_ss1(d, q + (AT_PANEL >> 4) + (uint64_t)((n - 4) * 2), k + (AT_PANEL >> 4) + (uint64_t)((n - 4) * 2), id_s, 1);
                }
                commit_one(smem_u32(&bars.s_full[i]));
            };
            auto wait = [&](uint64_t &bar, uint32_t phase) { ok = attn_wait(smem_u32(&bar), phase, &abort_flag); };
            auto next_keys = [&] {
                commit_one(smem_u32(&bars.k_empty[ks]));
                if (++ks == ST) { ks = 0; k_phase ^= 1u; }
            };
            for (; ok && uniform(sg.get()); sg.done(a)) {
                const int nt = uniform(sg.two(a) ? 2 : 1), steps = uniform(sg.n);
                wait(bars.k_full[ks], k_phase);
                for (int i = 0; ok && i < nt; ++i) {
                    wait(bars.q_full[i], q_phase[i]);
                    if (!ok) break;
                    q_phase[i] ^= 1u;
                    tmem_after();
                    scores(i);
                    if (steps == 1) commit_one(smem_u32(&bars.q_empty[i]));
                }
                if (!ok) break;
                next_keys();
                for (int j = 0; ok && j < steps; ++j) {
                    const bool more = j + 1 < steps;
                    wait(bars.v_full[vs], v_phase);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (!ok || i >= nt) break;
                        wait(bars.p_half[i], p_phase[i]);
                        if (!ok) break;
                        tmem_after();
                        const uint64_t v = v0 + (uint64_t)((uint32_t)vs * (PART >> 4));
                        const uint32_t d = tmem + 256u + (uint32_t)i * 128u, p = tmem + (uint32_t)i * 128u;
                        mma_ts4(d, p, v, id_o, j > 0);
                        wait(bars.p_full[i], p_phase[i]);
                        if (!ok) break;
                        p_phase[i] ^= 1u;
                        tmem_after();
                        mma_ts4(d, p + 32u, v + 512, id_o, 1);
                        if (!more) commit_one(smem_u32(&bars.o_full[i]));
                        else {
                            if (i == 0) wait(bars.k_full[ks], k_phase);
                            if (!ok) break;
                            scores(i);
                            if (j + 2 == steps) commit_one(smem_u32(&bars.q_empty[i]));
                        }
                    }
                    if (!ok) break;
                    commit_one(smem_u32(&bars.v_empty[vs]));
                    if (++vs == ST) { vs = 0; v_phase ^= 1u; }
                    if (more) next_keys();
                }
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int tile = (warp - AT_SOFT_WARP) >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t t_s = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)tile * 128u, t_o = t_s + 256u;
        uint8_t *const turn = smem + TURN + (uint32_t)(warp - AT_SOFT_WARP) * AT_TURN;
        uint32_t s_phase = 0, o_phase = 0;
        AttnRow row{-1, 0, 0, 0};
        float m = 0.f, l = 0.f;
        int64_t slot = 0;
        bool before = false, complete = false, described = false;               // before: an item whose outcome is not stored yet
        while (ok) {
            const int token = row.token, head = row.head;
            while (sg.get() && tile == 1 && !sg.two(a)) sg.done(a);
            const bool live = sg.s.left > 0;
            if (live) row = attn_row(a, sg.s.c.q, sg.s.c.hu, sg.s.c.rt, tile * AT_TILE + r);
            if (before) {
                ok = attn_wait(smem_u32(&bars.o_full[tile]), o_phase, &abort_flag);
                if (!ok) break;
                o_phase ^= 1u;
                tmem_after();
                const int64_t at = slot * a.rows + tile * AT_TILE + r;
                uint8_t *const dst = complete ? reinterpret_cast<uint8_t *>(static_cast<T *>(a.out) + (token < 0 ? 0 : token * a.o_ts + head * a.o_hs))
                                              : reinterpret_cast<uint8_t *>(a.po + at * a.D);
                if (!complete && token >= 0) a.ml[at] = make_float2(m, l);
                if (complete && (a.pml || __any_sync(0xffffffffu, token >= 0 && (reinterpret_cast<uintptr_t>(dst) & 15) != 0))) {
                    // with a shared prefix's sums, or outputs off 16 bytes: a thread a row
#pragma unroll 1
                    for (int d = 0; d < a.D; d += 8) {
                        uint32_t o[8];
                        tmem_ld8(t_o + (uint32_t)d, o);
                        tmem_wait_ld();
                        float v[8], M = m, L = l;
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = l == 0.f ? 0.f : __uint_as_float(o[e]);
                        if (token >= 0) attn_finish<T>(a, token, head, d, M, L, v);
                    }
                } else {
                    // 128 bytes of each row at a time, turned in shared memory so that eight lanes store a row's (a thread a row: 32 lines a
                    // store, 5300 cycles an item)
                    uint8_t *to[8];
                    uint32_t there = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        to[i] = reinterpret_cast<uint8_t *>(__shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(dst), i * 4 + (lane >> 3))) + (lane & 7) * 16;
                        there |= (uint32_t)(__shfl_sync(0xffffffffu, token, i * 4 + (lane >> 3)) >= 0) << i;
                    }
                    auto store = [&](const uint32_t (&w)[32], int at_byte, int bytes) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            *reinterpret_cast<uint4 *>(turn + lane * 128 + ((e ^ (lane & 7)) << 4)) = make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
                        __syncwarp();
                        uint4 v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int from = i * 4 + (lane >> 3);
                            v[i] = *reinterpret_cast<const uint4 *>(turn + from * 128 + (((lane & 7) ^ (from & 7)) << 4));
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if ((there >> i & 1) && (lane & 7) * 16 < bytes) *reinterpret_cast<uint4 *>(to[i] + at_byte) = v[i];
                        __syncwarp();
                    };
                    uint32_t o[2][32], w[32];
                    if (complete) {
                        // (a row that saw nothing gives 0, whatever 0 times the values of others' keys is)
                        const float scale = l == 0.f ? 0.f : 1.f / l;
                        auto scaled = [&](uint32_t x) { return l == 0.f ? 0.f : __uint_as_float(x) * scale; };
#pragma unroll 1
                        for (int d = 0; d < a.D; d += 64) {
                            tmem_ld32(t_o + (uint32_t)d, o[0]);
                            tmem_ld32(t_o + (uint32_t)d + 32u, o[1]);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                w[e] = pack2<T>(scaled(o[e / 16][2 * e & 31]), scaled(o[e / 16][(2 * e & 31) + 1]));
                            store(w, d * 2, (a.D - d) * 2);
                        }
                    } else {
#pragma unroll 1
                        for (int d = 0; d < a.D; d += 32) {
                            tmem_ld32(t_o + (uint32_t)d, o[0]);
                            tmem_wait_ld();
                            store(o[0], d * 4, (a.D - d) * 4);
                        }
                    }
                }
            }
            if (!live) break;
            // keys that all (existing) rows of the warp see need no comparison
            const int all_hi = __reduce_min_sync(0xffffffffu, row.token >= 0 ? row.hi : INT_MAX);
            const int all_lo = __reduce_max_sync(0xffffffffu, row.token >= 0 ? row.lo : 0);
            m = -INFINITY; l = 0.f;
            for (int j = 0; j < sg.n; ++j) {
                const int j0 = attn_tile_at(sg.s.c.t, sg.s.c.tile + j) * AT_BN;
                ok = attn_wait(smem_u32(&bars.s_full[tile]), s_phase, &abort_flag);
                if (!ok) break;
                s_phase ^= 1u;
                tmem_after();
                uint32_t s[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(t_s + (uint32_t)c * 32u, s[c]);
                tmem_wait_ld();
                if (!(j0 + AT_BN <= all_hi && j0 >= a.kv0 && (j0 >= all_lo || j0 + AT_BN <= a.sinks))) {
                    // keys first .. last - 1 of the tile (the first `early` ones too) are seen: a bit each, 32 at a time
                    const int first = imax(row.lo, a.kv0) - j0, last = row.hi - j0, early = imin(a.sinks, row.hi) - j0, least = a.kv0 - j0;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t seen = (bits_below(last - c * 32) & ~bits_below(first - c * 32)) |
                                              (bits_below(early - c * 32) & ~bits_below(least - c * 32));
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!(seen & (1u << e))) s[c][e] = 0xff800000u;
                    }
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = max3(__uint_as_float(s[c][0]), __uint_as_float(s[c][1]), __uint_as_float(s[c][2]));
#pragma unroll
                    for (int e = 3; e < 31; e += 2) mx[c] = max3(mx[c], __uint_as_float(s[c][e]), __uint_as_float(s[c][e + 1]));
                    mx[c] = fmaxf(mx[c], __uint_as_float(s[c][31]));
                }
                // (a row that does not exist holds whatever was there: it has no say in when the others' sums are rescaled)
                const float top = row.token >= 0 ? fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) : -INFINITY;
                constexpr float LIFT = AttnRef<T>::lift, LAG = AttnRef<T>::lag;
                if (__any_sync(0xffffffffu, fmaf(top, a.sc, -m) > LIFT + LAG)) {
                    const float to = fmaxf(m, fmaf(top, a.sc, -LIFT)), f = m == -INFINITY ? 0.f : attn_exp2(m - to);
                    m = to;
                    l *= f;
                    if (j > 0) {
#pragma unroll 1
                        for (int c = 0; c < NK; ++c) {
                            uint32_t o[16];
                            tmem_ld16(t_o + (uint32_t)c * 16u, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            tmem_st16(t_o + (uint32_t)c * 16u, o);
                        }
                    }
                }
                const float ref = m == -INFINITY ? 0.f : m;
                const uint64_t sc2 = pair(a.sc, a.sc), ref2 = pair(-ref, -ref);
                uint64_t sum[2] = {0, 0};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float x, y;
                        halves(fma2(pair(__uint_as_float(s[c][2 * e]), __uint_as_float(s[c][2 * e + 1])), sc2, ref2), x, y);
                        x = attn_exp2(x); y = attn_exp2(y);
                        sum[e & 1] = add2(sum[e & 1], pair(x, y));
                        p[e] = pack2<T>(x, y);
                    }
                    tmem_st16(t_s + (uint32_t)c * 16u, p);
                    if (c & 1) {                            // the product with the first 64 values may begin
                        tmem_wait_st();
                        tmem_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(c == 1 ? &bars.p_half[tile] : &bars.p_full[tile]));
                    }
                }
                float sums[4];
                halves(sum[0], sums[0], sums[1]);
                halves(sum[1], sums[2], sums[3]);
                l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
            }
            if (!ok) break;
            // the item's outcome is on its way to tensor memory
            const int c = (int)blockIdx.x, x = deal.count(c) - sg.s.left;
            before = true;
            complete = sg.n == sg.s.c.t.nt && !a.common;
            slot = a.common ? ((int64_t)sg.s.c.hu * attn_row_blocks(a, sg.s.c.q) + sg.s.c.rt) + c : 2 * (int64_t)c + (x > 0 ? 1 : 0);
            if (warp == AT_SOFT_WARP && lane == 0 && !a.common && sg.s.c.tile == 0 && !complete) {
                attn_describe(a, sg.s.c, deal, c, x, 0, sg.n);
                described = true;
            }
            sg.done(a);
        }
        if (warp == AT_SOFT_WARP && lane == 0 && !a.common && !a.whole && !described) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
    }
    if (!ok && lane == 0) atomicExch(a.status, 1);
    tmem_before();
    __syncthreads();
    if (*(volatile int *)&abort_flag) {
        // a block whose waits ran out leaves no copy and no product under way (a millisecond at most each)
        int gave_up = 0;
        if (warp == AT_Q_WARP) {
            for (int f = 0; f < 4; ++f) attn_wait(smem_u32(&bars.q_full[f >> 1]), (uint32_t)f & 1u, &gave_up, 2000000);
        }
        if (warp == AT_K_WARP || warp == AT_V_WARP) {
            for (int f = filled > ST ? filled - ST : 0; f <= filled; ++f) {
                attn_wait(smem_u32(warp == AT_V_WARP ? &bars.v_full[f % ST] : &bars.k_full[f % ST]), (uint32_t)(f / ST) & 1u, &gave_up, 2000000);
                if (warp == AT_V_WARP) attn_wait(smem_u32(&bars.patch), (uint32_t)(f & 1), &gave_up, 2000000);
            }
        }
        if (warp == AT_MMA_WARP) {
            commit_one(smem_u32(&bars.drain));
            attn_wait(smem_u32(&bars.drain), 0, &gave_up, 2000000);
        }
        __syncthreads();
    }
    if (warp == AT_MMA_WARP) {
        tmem_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
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
}  // namespace

// (a stride that is never used has to be a possible one)
int attn_encode_cache(CUtensorMap *tm, const AttnArgs &a, const void *base, int dtype, int keys)
{
    const EncodeTiledFn enc = encoder();
    if (!enc) return UBP_E_CUDA;
    const int page = 1 << a.pshift;
    const cuuint64_t dims[4] = {(cuuint64_t)a.D, (cuuint64_t)page, (cuuint64_t)a.Hkv, (cuuint64_t)a.pages};
    const cuuint64_t unit = (cuuint64_t)a.c_ts * 2;
    const cuuint64_t strides[3] = {unit, a.Hkv > 1 ? (cuuint64_t)a.c_hs * 2 : unit, a.pages > 1 ? (cuuint64_t)a.c_ps * 2 : unit};
    const cuuint32_t box[4] = {64, (cuuint32_t)imin(page, keys), 1, 1}, one[4] = {1, 1, 1, 1};
    const CUresult r = enc(tm, dtype == UBP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void *>(base), dims, strides, box, one,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) { set_last_cuda_error((int)cudaErrorInvalidValue); return UBP_E_CUDA; }
    return UBP_OK;
}

namespace {

// (head values, heads, tokens): boxes of 64 values x the heads of a unit head x the tokens of a tile
int encode_queries(CUtensorMap *tm, const AttnArgs &a, int dtype)
{
    const EncodeTiledFn enc = encoder();
    if (!enc) return UBP_E_CUDA;
    const cuuint64_t dims[3] = {(cuuint64_t)a.D, (cuuint64_t)a.Hq, (cuuint64_t)a.T};
    const cuuint64_t unit = (cuuint64_t)a.D * 2, strides[2] = {a.Hq > 1 ? (cuuint64_t)a.q_hs * 2 : unit, a.T > 1 ? (cuuint64_t)a.q_ts * 2 : unit * a.Hq};
    const cuuint32_t box[3] = {64, (cuuint32_t)a.gc, (cuuint32_t)(a.tpt / 2)}, one[3] = {1, 1, 1};
    const CUresult r = enc(tm, dtype == UBP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(a.q), dims, strides, box, one,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) { set_last_cuda_error((int)cudaErrorInvalidValue); return UBP_E_CUDA; }
    return UBP_OK;
}

template <typename T> int launch_tc_t(const CUtensorMap &k, const CUtensorMap &v, const CUtensorMap &q, const AttnArgs &a, int grid, void *stream)
{
    static std::atomic<bool> done[5][64] = {};
    const dim3 g((unsigned)grid);
    switch (a.D <= 64 ? 4 : (a.D + 15) / 16) {
        case 4: return attn_launch(ubp_attention_tc_kernel<T, 4>, done[0], g, AT_THREADS, at_smem(64), 1, stream, k, v, q, a);
        case 5: return attn_launch(ubp_attention_tc_kernel<T, 5>, done[1], g, AT_THREADS, at_smem(128), 1, stream, k, v, q, a);
        case 6: return attn_launch(ubp_attention_tc_kernel<T, 6>, done[2], g, AT_THREADS, at_smem(128), 1, stream, k, v, q, a);
        case 7: return attn_launch(ubp_attention_tc_kernel<T, 7>, done[3], g, AT_THREADS, at_smem(128), 1, stream, k, v, q, a);
        default: return attn_launch(ubp_attention_tc_kernel<T, 8>, done[4], g, AT_THREADS, at_smem(128), 1, stream, k, v, q, a);
    }
}

}  // namespace

int launch_attn_tc(const AttnArgs &a, int dtype, int grid, void *stream)
{
    CUtensorMap k, v, q;
    if (const int rc = attn_encode_cache(&k, a, a.k, dtype, AT_BN)) return rc;
    if (const int rc = attn_encode_cache(&v, a, a.v, dtype, AT_BN)) return rc;
    if (const int rc = encode_queries(&q, a, dtype)) return rc;
    return dtype == UBP_BF16 ? launch_tc_t<__nv_bfloat16>(k, v, q, a, grid, stream) : launch_tc_t<__half>(k, v, q, a, grid, stream);
}

}  // namespace ubp
