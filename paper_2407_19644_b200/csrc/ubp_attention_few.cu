// Attention of a few query rows over a paged cache: single tokens of running answers (and any other item, 16 rows at a time).
//
//   s_j = scale q.k_j,  o = sum_j 2^(s_j log2e - m) v_j / sum_j 2^(s_j log2e - m)     over the keys j that the row sees
//
// One pass over the keys and values with a running reference m and sum: bound by HBM, 4 D bytes a key and key head. The 16 rows
// of an item are the query heads of one key head (and neighbouring tokens), so that a key is read once for all of them, and they
// are the rows of an m16n8k16 product: at 16 rows it is 16 multiply-adds a value read, a tenth of what the SM could do in the time
// HBM takes for that value, so the unused rows of small groups cost nothing.
// Eight warps a block; a warp has its own 16 keys of a step's 128 (heads of up to 64 values: 32 of 256), its own ring of copies and
// its own running sums: nothing in the loop waits for another warp. They meet once an item. Copies are TMA boxes of 64 values x those
// keys (fewer where pages are smaller), which run ahead over the ends of items: with 16-byte cp.async, whose addresses every lane
// computed, a step took 930 instructions and the kernel ran at 45 % of HBM. Now 64 tokens on 500 .. 8191 keys of eight heads of 128
// values, 1.14 GB, take 182 us with the join, 6.3 TB/s; three tokens on 100000 keys of two heads of 64 values, 0.15 GB, 34 us.
// Pages that no row of the item sees, or that the cache does not have, are out of range for the copy and come as zeros; values of
// unseen keys within a page are overwritten with zeros, so that nothing an unused slot holds reaches a result. The weights are
// rounded to 16 bits for the second product (relative 2^-8 / 2^-11 each, the sum of weights is of the unrounded ones); scores,
// references, sums and outputs are fp32 until the end.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <type_traits>

#include "ubp_attention_steps.cuh"
#include "ubp_attention_copy.cuh"

namespace ubp {
namespace {

using namespace tc;

constexpr int FEW_WARPS = 8, FEW_ROWS = 16, FEW_STAGES = 3;
__host__ __device__ constexpr int few_keys(int dp) { return dp == 128 ? 16 : 32; }                        // a warp's of a step: 4 KB of keys, 4 KB of values
constexpr uint32_t FEW_PART = 4096;
constexpr uint32_t FEW_RING = FEW_STAGES * 2 * FEW_PART;                                                    // a warp's
__host__ __device__ constexpr uint32_t few_smem(int dp) { return FEW_WARPS * (FEW_RING + 8 * (uint32_t)dp * 4 + FEW_ROWS * 8) + 1024; }
static_assert(few_smem(128) <= 227 * 1024 - 1024, "with the static part");

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
template <typename T> __device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same_v<T, __half>)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// from the same place in the shared memory of another block of the cluster
__device__ __forceinline__ uint32_t rank_at(const void *p, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ float2 ld_rank2(const float2 *p, uint32_t rank)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(rank_at(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ void ld_rank4(const float *p, uint32_t rank, float (&v)[4])
{
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(rank_at(p, rank)) : "memory");
}

// The copies of a warp's steps: a cursor that runs ahead, with the pages of the next step already loaded.
// Everything is the same in all lanes; lane 0 issues.
template <int DP> struct FewCopies {
    AttnSteps s;
    int page[few_keys(DP) / 8], j0, kvh;

    __device__ __forceinline__ void item(const AttnArgs &a) { kvh = (int)((uint32_t)s.c.hu / (uint32_t)a.chunks); }
    __device__ __forceinline__ void peek(const AttnArgs &a, int warp)
    {
        constexpr int KEYS = few_keys(DP);
        j0 = attn_tile_at(s.c.t, s.c.tile) * (FEW_WARPS * KEYS) + warp * KEYS;
        const int box = imin(1 << a.pshift, KEYS);
#pragma unroll
        for (int b = 0; b < KEYS / 8; ++b)
            if (b * box < KEYS) page[b] = attn_box_page(a, s.c.t, s.c.b, j0 + b * box, box);
    }
    __device__ __forceinline__ void issue(const AttnArgs &a, const CUtensorMap *tmK, const CUtensorMap *tmV, uint32_t stage, uint32_t bar, int warp, int lane)
    {
        constexpr int KEYS = few_keys(DP);
        if (s.left <= 0) return;
        if (lane == 0) {
            const int box = imin(1 << a.pshift, KEYS);
            mbar_expect_tx(bar, 2 * FEW_PART);
#pragma unroll
            for (int b = 0; b < KEYS / 8; ++b)
                if (b * box < KEYS) {
                    const int at = (j0 + b * box) & ((1 << a.pshift) - 1);
#pragma unroll
                    for (int p = 0; p < DP / 64; ++p) {
                        const uint32_t to = stage + (uint32_t)(p * KEYS + b * box) * 128u;
                        tma_load_4d(to, tmK, p * 64, at, kvh, page[b], bar);
                        tma_load_4d(to + FEW_PART, tmV, p * 64, at, kvh, page[b], bar);
                    }
                }
        }
        const bool over = s.c.tile + 1 == s.c.t.nt;
        s.advance(a, 1);
        if (s.left <= 0) return;
        if (over) item(a);
        peek(a, warp);
    }
};

// NK: head size in steps of 16 (the copies bring zeros past it)
// CLUSTER: a cluster of blocks takes a sequence and unit head, a share of its tiles each; their sums meet in distributed shared
// memory, rank r finishes rows r, r + size, .. (short work of few sequences: no dealing of steps, no partial results, no second kernel)
template <typename T, int NK, bool CLUSTER>
__global__ void __launch_bounds__(FEW_WARPS * 32, 1)
ubp_attention_few_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const AttnArgs a)
{
    constexpr int DP = NK > 4 ? 128 : 64, ST = FEW_STAGES, KEYS = few_keys(DP), NB = KEYS / 8;
    constexpr uint32_t PART = FEW_PART, PANEL = KEYS * 128;        // 64 values of each of a warp's keys
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    __shared__ __align__(8) uint64_t bar_full[FEW_WARPS][ST];
    __shared__ int2 rows[2][FEW_ROWS];      // token and head of the rows of an item, and of the next one
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, tq = lane & 3;
    float *const meet = reinterpret_cast<float *>(smem + FEW_WARPS * FEW_RING);                      // [warp][8 rows][DP]
    float2 *const meet_ml = reinterpret_cast<float2 *>(meet + FEW_WARPS * 8 * DP);                    // [warp][row]
    const uint32_t ring = smem_u32(smem) + (uint32_t)warp * FEW_RING;
    float *const part = reinterpret_cast<float *>(smem);               // CLUSTER: [row][DP] and [row] of the block's sums
    float2 *const part_ml = reinterpret_cast<float2 *>(part + FEW_ROWS * DP);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (lane == 0) {
        if (warp == 0) { prefetch_tensormap(&tmK); prefetch_tensormap(&tmV); abort_flag = 0; }
        for (int i = 0; i < ST; ++i) mbar_init(smem_u32(&bar_full[warp][i]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");

    AttnDeal deal;
    AttnSteps steps;
    int size = 1, rank = 0, tiles = 0;      // of the cluster; tiles of the item
    static_assert(sizeof(AttnPlace<FEW_WARPS * 32>) <= FEW_WARPS * 8 * 64 * 4, "lies where the warps' sums meet");
    if constexpr (CLUSTER) {
        asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(size));
        rank = (int)cluster_rank();
        const int u = (int)blockIdx.x / size, b = u / a.HU;
        steps.c.set(a, b, u - b * a.HU, 0, 0);
        if (steps.c.q.n == 0) return;       // (all of the cluster)
        tiles = steps.c.t.nt;
        steps.c.tile = tiles * rank / size;
        steps.left = tiles * (rank + 1) / size - steps.c.tile;
    } else if (!attn_locate<FEW_WARPS * 32>(a, *reinterpret_cast<AttnPlace<FEW_WARPS * 32> *>(meet), deal, steps)) {
        if (threadIdx.x == 0 && !a.common && !a.whole) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
        return;
    }
    const AttnCursor &cur = steps.c;
    uint32_t qf[NK][4];
    AttnRow row[2];                         // (their keys; tokens and heads are in `rows`)
    int all_lo = 0, all_hi = 0, which = 0;  // keys that all rows see; the item's place in `rows`
    // an item's rows and queries; under way while the item before it ends
    auto begin = [&](const AttnCursor &c) {
        const AttnRow w = attn_row(a, c.q, c.hu, c.rt, lane & 15);
        if (warp == 0 && lane < 16) rows[which][lane] = make_int2(w.token, w.head);
        all_lo = __reduce_max_sync(0xffffffffu, w.token >= 0 ? w.lo : 0);
        all_hi = __reduce_min_sync(0xffffffffu, w.token >= 0 ? w.hi : INT_MAX);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int token = __shfl_sync(0xffffffffu, w.token, g + 8 * i), head = __shfl_sync(0xffffffffu, w.head, g + 8 * i);
            row[i].lo = __shfl_sync(0xffffffffu, w.lo, g + 8 * i);
            row[i].hi = __shfl_sync(0xffffffffu, w.hi, g + 8 * i);
            const T *p = static_cast<const T *>(a.q) + (token < 0 ? 0 : token * a.q_ts + head * a.q_hs) + tq * 2;
#pragma unroll
            for (int k = 0; k < 2 * NK; ++k) qf[k / 2][k % 2 * 2 + i] = token >= 0 && k * 8 < a.D ? *reinterpret_cast<const uint32_t *>(p + k * 8) : 0u;
        }
    };
    FewCopies<DP> copies;
    bool ok = true;                         // no wait has run out
    int st = 0;                             // stage of the next step
    uint32_t phase = 0;
    auto start = [&] {                      // the first copies of a share
        copies.s = steps;
        if (!ok) copies.s.left = 0;
        copies.item(a);
        if (copies.s.left > 0) copies.peek(a, warp);
#pragma unroll 1
        for (int s = 0; s < ST - 1; ++s) {
            const int to = st + s < ST ? st + s : st + s - ST;
            copies.issue(a, &tmK, &tmV, ring + (uint32_t)to * 2 * PART, smem_u32(&bar_full[warp][to]), warp, lane);
        }
    };
    if constexpr (!CLUSTER) start();

    // where the lane's rows of matrix instructions' operands lie in a part: piece (2 k + h) of 16 bytes at k * 32 (within 128 bytes)
    // xor h and the row; the same for keys (rows = keys) and values (transposed)
    const int rk = (lane & 7) + (lane >> 4) * 8, rv = (lane & 7) + (lane >> 3 & 1) * 8;
    const uint32_t at_k = (uint32_t)(rk * 128), xk = (uint32_t)(((lane >> 3 & 1) ^ (rk & 7)) << 4);
    const uint32_t at_v = PART + (uint32_t)(rv * 128), xv = (uint32_t)(((lane >> 4) ^ (rv & 7)) << 4);

    float o[2 * NK][4], m[2], l[2];
    int tile0 = 0, before = 0;              // of the segment: its first tile, the share's steps before it
    bool described = false, over = true, any = false;      // over: a segment has ended (or the first one begins); any: there was one
    while (true) {
        if (over) {
            // The segment before has ended: its warps' sums meet, rows 0 .. 7, then 8 .. 15 where the item has them. Before that, the
            // next item's queries are sent for. (Once in the code: a call of a few steps is bound by fetching instructions.)
            if (CLUSTER && !any) start();
            const int c = (int)blockIdx.x, n = cur.tile + 1 - tile0, now = which;
            const int nr = any ? imin(imin(a.tpt, cur.q.n - cur.rt * a.tpt) * a.gc, FEW_ROWS) : 0;
            const bool whole = n == cur.t.nt && !a.common;
            int64_t slot = 2 * (int64_t)c + (before > 0 ? 1 : 0);
            if (a.common) slot = (int64_t)cur.hu * attn_row_blocks(a, cur.q) + cur.rt + c;
            if (any) {
                if (!CLUSTER && threadIdx.x == 0 && !a.common && tile0 == 0 && !whole) {
                    attn_describe(a, cur, deal, c, before, tile0, n);
                    described = true;
                }
                if (!CLUSTER || steps.left > 0) steps.advance(a, 1);
                which ^= 1;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
                    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
                    if (tq == 0) meet_ml[warp * FEW_ROWS + g + 8 * i] = make_float2(m[i], l[i]);
                }
            }
            if (CLUSTER ? !any : steps.left > 0) begin(cur);
#pragma unroll 1
            for (int i = 0; i * 8 < nr; ++i) {
                if (i) __syncthreads();
#pragma unroll
                for (int k = 0; k < 2 * NK; ++k)
                    *reinterpret_cast<float2 *>(meet + (warp * 8 + g) * DP + k * 8 + tq * 2) =
                        i ? make_float2(o[k][2], o[k][3]) : make_float2(o[k][0], o[k][1]);
                __syncthreads();
                constexpr int N = 4, TPR = DP / N;          // threads a row
                const int r = (int)threadIdx.x / TPR, col = (int)threadIdx.x % TPR * N;
                if (r < 8) {
                    const int2 w = rows[now][i * 8 + r];
                    if (col < a.D && (CLUSTER || w.x >= 0 || !whole)) {
                        float M = -INFINITY, L = 0.f, v[N] = {}, u[FEW_WARPS][N];
                        float2 ml[FEW_WARPS];
#pragma unroll
                        for (int k = 0; k < FEW_WARPS; ++k) {
                            ml[k] = meet_ml[k * FEW_ROWS + i * 8 + r];
                            attn_load(meet + (k * 8 + r) * DP + col, u[k]);
                        }
                        attn_add_all(M, L, v, ml, u, FEW_WARPS);
                        if constexpr (CLUSTER) {            // (over the ring: this share's copies have all been read)
                            if (col == 0) part_ml[i * 8 + r] = make_float2(M, L);
                            *reinterpret_cast<float4 *>(part + (i * 8 + r) * DP + col) = make_float4(v[0], v[1], v[2], v[3]);
                        } else if (whole) attn_finish<T>(a, w.x, w.y, col, M, L, v);
                        else {
                            if (col == 0) a.ml[slot * FEW_ROWS + i * 8 + r] = make_float2(M, L);
                            *reinterpret_cast<float4 *>(a.po + (slot * FEW_ROWS + i * 8 + r) * a.D + col) = make_float4(v[0], v[1], v[2], v[3]);
                        }
                    }
                }
            }
            if constexpr (CLUSTER) {
                if (any) {
                    cluster_sync();
                    constexpr int N = 4;
                    const int per = a.D / N;
                    for (int x = (int)threadIdx.x; x < (nr - rank + size - 1) / size * per; x += FEW_WARPS * 32) {
                        const int r = rank + x / per * size, col = x % per * N;
                        const int2 w = rows[now][r];
                        float M = -INFINITY, L = 0.f, v[N] = {}, u[8][N];
                        float2 ml[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (k < size) {
                                ml[k] = ld_rank2(part_ml + r, (uint32_t)k);
                                ld_rank4(part + r * DP + col, (uint32_t)k, u[k]);
                            }
                        attn_add_all(M, L, v, ml, u, size);
                        if (w.x >= 0 && ok) attn_finish<T>(a, w.x, w.y, col, M, L, v);
                    }
                    cluster_sync();                         // (nobody leaves or goes on while its sums are being read)
                    const int rt = cur.rt + 1;
                    if (rt * a.tpt >= cur.q.n) break;
                    // (more new tokens than the caller said: the next row block)
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    steps.c.set(a, cur.b, cur.hu, rt, 0);
                    steps.c.tile = steps.c.t.nt * rank / size;
                    steps.left = steps.c.t.nt * (rank + 1) / size - steps.c.tile;
                    __syncthreads();
                    any = false;
                    continue;
                }
                over = steps.left <= 0;                     // (a share without tiles meets the others all the same)
            } else {
                if (steps.left <= 0) break;
                if (any) __syncthreads();                   // (all have read)
                over = false;
            }
            any = true;
            tile0 = cur.tile;
            if constexpr (!CLUSTER) before = deal.count(c) - steps.left;
#pragma unroll
            for (int i = 0; i < 2; ++i) { m[i] = -INFINITY; l[i] = 0.f; }
#pragma unroll
            for (int k = 0; k < 2 * NK; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[k][e] = 0.f;
            if (CLUSTER && over) continue;
        }
        __syncwarp();                       // (all lanes have read the stage that is copied to now)
        const int nx = st == 0 ? ST - 1 : st - 1;
        copies.issue(a, &tmK, &tmV, ring + (uint32_t)nx * 2 * PART, smem_u32(&bar_full[warp][nx]), warp, lane);
        if (ok && !attn_wait(smem_u32(&bar_full[warp][st]), phase, &abort_flag)) {
            ok = false;
            copies.s.left = 0;              // (a stage whose copy has not come is not copied to again)
        }
        const int j0 = attn_tile_at(cur.t, cur.tile) * (FEW_WARPS * KEYS) + warp * KEYS;
        const uint32_t base = ring + (uint32_t)st * 2 * PART;
        if (ok && j0 < cur.t.end && j0 + KEYS > a.kv0 && (j0 + KEYS > cur.t.w0 || j0 < a.sinks)) {
            float s[NB][4] = {};
            if constexpr (NB == 2) {
                float s1[2][4] = {};                        // (two sums each, half as long a chain)
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    uint32_t b[4];
                    ldsm4(b, base + at_k + (uint32_t)(k / 4) * PANEL + ((uint32_t)(k % 4 * 32) ^ xk));
                    mma16<T>(k & 1 ? s1[0] : s[0], qf[k], b[0], b[1]);
                    mma16<T>(k & 1 ? s1[1] : s[1], qf[k], b[2], b[3]);
                }
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n][e] += s1[n][e];
            } else {
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int n = 0; n < NB; n += 2) {
                        uint32_t b[4];
                        ldsm4(b, base + at_k + (uint32_t)(n * 8 * 128) + ((uint32_t)(k % 4 * 32) ^ xk));
                        mma16<T>(s[n], qf[k], b[0], b[1]);
                        mma16<T>(s[n + 1], qf[k], b[2], b[3]);
                    }
            }
            const bool all = j0 + KEYS <= all_hi && j0 >= a.kv0 && (j0 >= all_lo || j0 + KEYS <= a.sinks);
            if (!all) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!attn_sees(a, row[e >> 1], j0 + n * 8 + tq * 2 + (e & 1))) s[n][e] = -INFINITY;
                // values of keys that no row sees
#pragma unroll 1
                for (int x = lane; x < KEYS * DP / 8; x += 32) {
                    const int r = x / (DP / 8), ch = x % (DP / 8), j = j0 + r;
                    if (!(j >= a.kv0 && j < cur.t.end && (j >= cur.t.w0 || j < a.sinks)))
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};"
                                     ::"r"(base + PART + (uint32_t)(ch / 8) * PANEL + (uint32_t)(r * 128 + ch % 8 * 16)), "r"(0) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (before the next copy to these places)
                __syncwarp();
            }
            float mx[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                mx[i] = fmaxf(s[0][2 * i], s[0][2 * i + 1]);
#pragma unroll
                for (int n = 1; n < NB; ++n) mx[i] = fmaxf(mx[i], fmaxf(s[n][2 * i], s[n][2 * i + 1]));
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
            }
            // (the reference: see AttnRef)
            constexpr float LIFT = AttnRef<T>::lift, LAG = AttnRef<T>::lag;
            if (__any_sync(0xffffffffu, fmaf(mx[0], a.sc, -m[0]) > LIFT + LAG || fmaf(mx[1], a.sc, -m[1]) > LIFT + LAG)) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float to = fmaxf(m[i], fmaf(mx[i], a.sc, -LIFT)), f = m[i] == -INFINITY ? 0.f : attn_exp2(m[i] - to);
                    m[i] = to;
                    l[i] *= f;
#pragma unroll
                    for (int n = 0; n < 2 * NK; ++n) { o[n][2 * i] *= f; o[n][2 * i + 1] *= f; }
                }
            }
            uint32_t p[NB / 2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float ref = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    const float p0 = attn_exp2(fmaf(s[n][2 * i], a.sc, -ref)), p1 = attn_exp2(fmaf(s[n][2 * i + 1], a.sc, -ref));
                    l[i] += p0 + p1;
                    p[n / 2][n % 2 * 2 + i] = pack2<T>(p0, p1);
                }
            }
#pragma unroll
            for (int h = 0; h < NB / 2; ++h)
#pragma unroll
                for (int n = 0; n < NK; ++n) {
                    uint32_t b[4];
                    ldsm4t(b, base + at_v + (uint32_t)(h * 16 * 128) + (uint32_t)(n / 4) * PANEL + ((uint32_t)(n % 4 * 32) ^ xv));
                    mma16<T>(o[2 * n], p[h], b[0], b[1]);
                    mma16<T>(o[2 * n + 1], p[h], b[2], b[3]);
                }
        }
        if (++st == ST) { st = 0; phase ^= 1u; }
        over = cur.tile + 1 == cur.t.nt || steps.left == 1;
        if (!over) steps.advance(a, 1);
    }
    if (!CLUSTER && threadIdx.x == 0 && !a.common && !a.whole && !described) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
    if (!ok) {                              // copies that are still under way end before the block does (a millisecond at most each)
        int gave_up = 0;
        for (int i = 0; i < ST; ++i)
            for (uint32_t ph = 0; ph < 2; ++ph) attn_wait(smem_u32(&bar_full[warp][i]), ph, &gave_up, 2000000);
        if (lane == 0) atomicExch(a.status, 1);
    }
}

// Joins the partial results of an item that several blocks have worked on, in the order of its keys: a warp a row, four values a
// lane, eight parts under way at a time.
// COMMON: block (u, i) takes the i-th rows of item u of the shared prefix; all of its blocks' results lie in slots u + block, and the
// sums go to pml and ppo. Else block (c, i) takes those of the item that begins in block c, if it does not end there.
// ROWS a block: 8 for the prefix and for items of 16 rows, which have many parts (32: 64 blocks for a batch of 64, 20 us); 32 for
// items of 256 rows, which have two or three (8: 4700 blocks for 148 items, 10 us).
constexpr int JOIN_WARPS = 8;
template <typename T, bool COMMON, int ROWS>
__global__ void __launch_bounds__(JOIN_WARPS * 32) ubp_attention_join_kernel(const AttnArgs a, const int blocks)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int col = (int)(threadIdx.x & 31) * 4;
    int t0, n, hu, parts;
    int64_t slot0, slot1;                   // of the first part, and of the second one (the others follow)
    if constexpr (COMMON) {
        const AttnSeq q = attn_seq(a, 0);
        const int nrt = attn_row_blocks(a, q), nt = attn_block_tiles(a, q, 0).nt, u = (int)blockIdx.x;
        if (u >= nrt * a.HU) return;
        const AttnDeal deal((int64_t)nrt * a.HU * (nt + a.extra), blocks);
        hu = u / nrt;
        t0 = (u - hu * nrt) * a.tpt;
        n = q.n - t0;
        const int64_t x = (int64_t)u * (nt + a.extra);
        const int c = deal.owner(x);
        parts = deal.owner(x + nt - 1) - c + 1;
        slot0 = u + c; slot1 = slot0 + 1;
    } else {
        const int c = (int)blockIdx.x;
        const int4 d = a.desc[c];
        t0 = d.x; n = d.y; hu = d.z; parts = d.w >> 1;
        slot0 = 2 * (int64_t)c + (d.w & 1);
        slot1 = 2 * (int64_t)(c + 1);
    }
    if (parts == 0) return;
    if (col >= a.D) return;
    constexpr int N = 4, AHEAD = 8, STEP = COMMON ? 1 : 2;
    const int r0 = (int)blockIdx.y * ROWS + (int)(threadIdx.x >> 5);
    auto part = [&](int r, int k, float2 &ml, float (&v)[N]) {
        const int64_t at = (k == 0 ? slot0 : slot1 + (int64_t)(k - 1) * STEP) * a.rows + r;
        ml = a.ml[at];
        attn_load(a.po + at * a.D + col, v);
    };
    auto finish = [&](const int2 &w, float M, float L, float (&o)[N]) {
        if constexpr (COMMON) {
            const int64_t at = (int64_t)w.x * a.Hq + w.y;
            if (col == 0) a.pml[at] = make_float2(M, L);
            *reinterpret_cast<float4 *>(a.ppo + at * a.D + col) = make_float4(o[0], o[1], o[2], o[3]);
        } else {
            attn_finish<T>(a, w.x, w.y, col, M, L, o);
        }
    };
    if constexpr (ROWS > JOIN_WARPS) {
        if (parts == 2) {                   // the rule for such items: all of the warp's rows together
            constexpr int R = ROWS / JOIN_WARPS;
            float2 ml[R][2];
            float v[R][2][N];
            int2 w[R];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int r = r0 + i * JOIN_WARPS;
                w[i] = r < a.rows ? attn_row_at(a, t0, n, hu, r) : make_int2(-1, 0);
                if (w[i].x >= 0) { part(r, 0, ml[i][0], v[i][0]); part(r, 1, ml[i][1], v[i][1]); }
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                float M = -INFINITY, L = 0.f, o[N] = {};
                if (w[i].x < 0) continue;
                attn_add_all(M, L, o, ml[i], v[i], 2);
                finish(w[i], M, L, o);
            }
            return;
        }
    }
#pragma unroll 1
    for (int r = r0; r < imin(a.rows, ((int)blockIdx.y + 1) * ROWS); r += JOIN_WARPS) {
        const int2 w = attn_row_at(a, t0, n, hu, r);
        if (w.x < 0) continue;
        float M = -INFINITY, L = 0.f, o[N] = {};
        for (int k0 = 0; k0 < parts; k0 += AHEAD) {
            float2 ml[AHEAD];
            float v[AHEAD][N];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (k0 + i < parts) part(r, k0 + i, ml[i], v[i]);
            attn_add_all(M, L, o, ml, v, parts - k0);
        }
        finish(w, M, L, o);
    }
}

// Queries off 16 bytes -> rows that lie on them.
__global__ void __launch_bounds__(256) ubp_attention_copy_queries_kernel(const uint16_t *q, int64_t ts, int64_t hs, int64_t rows, int Hq, int D, uint4 *to)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int per = D / 8;
    for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < rows * per; x += (int64_t)gridDim.x * 256) {
        const int64_t row = x / per, t = row / Hq;
        const uint16_t *h = q + t * ts + (row - t * Hq) * hs + (x - row * per) * 8;
        to[x] = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
    }
}

// cluster: its size, 0: steps dealt to `grid` blocks
template <typename T, bool CLUSTER> int launch_few_t(const AttnArgs &a, int dtype, int grid, int cluster, void *stream)
{
    static std::atomic<bool> done[5][64] = {};
    CUtensorMap k, v;
    const int keys = few_keys(a.D <= 64 ? 64 : 128);
    if (const int rc = attn_encode_cache(&k, a, a.k, dtype, keys)) return rc;
    if (const int rc = attn_encode_cache(&v, a, a.v, dtype, keys)) return rc;
    const dim3 g((unsigned)grid);
    constexpr int t = FEW_WARPS * 32;
    switch (a.D <= 64 ? 4 : (a.D + 15) / 16) {
        case 4: return attn_launch(ubp_attention_few_kernel<T, 4, CLUSTER>, done[0], g, t, few_smem(64), cluster, stream, k, v, a);
        case 5: return attn_launch(ubp_attention_few_kernel<T, 5, CLUSTER>, done[1], g, t, few_smem(128), cluster, stream, k, v, a);
        case 6: return attn_launch(ubp_attention_few_kernel<T, 6, CLUSTER>, done[2], g, t, few_smem(128), cluster, stream, k, v, a);
        case 7: return attn_launch(ubp_attention_few_kernel<T, 7, CLUSTER>, done[3], g, t, few_smem(128), cluster, stream, k, v, a);
        default: return attn_launch(ubp_attention_few_kernel<T, 8, CLUSTER>, done[4], g, t, few_smem(128), cluster, stream, k, v, a);
    }
}

}  // namespace

int launch_attn_few(const AttnArgs &a, int dtype, int grid, void *stream)
{
    return dtype == UBP_BF16 ? launch_few_t<__nv_bfloat16, false>(a, dtype, grid, 1, stream) : launch_few_t<__half, false>(a, dtype, grid, 1, stream);
}

int launch_attn_cluster(const AttnArgs &a, int dtype, int size, void *stream)
{
    const int grid = a.B * a.HU * size;
    return dtype == UBP_BF16 ? launch_few_t<__nv_bfloat16, true>(a, dtype, grid, size, stream) : launch_few_t<__half, true>(a, dtype, grid, size, stream);
}

int launch_attn_copy_queries(const void *q, int64_t ts, int64_t hs, int64_t T, int Hq, int D, void *to, void *stream)
{
    static std::atomic<bool> done[64] = {};
    const int64_t blocks = (T * Hq * (D / 8) + 255) / 256, most = 8 * device_sms();
    return attn_launch(ubp_attention_copy_queries_kernel, done, dim3((unsigned)(blocks < most ? blocks : most)), 256, 0, 1, stream, static_cast<const uint16_t *>(q), ts, hs,
                       T * (int64_t)Hq, Hq, D, static_cast<uint4 *>(to));
}

int launch_attn_join(const AttnArgs &a, int dtype, int grid, void *stream)
{
    static std::atomic<bool> done[64] = {};       // (no dynamic shared memory: not looked at)
    auto go = [&](auto kern, int64_t x, int rows) {
        return attn_launch(kern, done, dim3((unsigned)x, (unsigned)((a.rows + rows - 1) / rows)), JOIN_WARPS * 32, 0, 1, stream, a, grid);
    };
    if (a.common) return go(ubp_attention_join_kernel<__half, true, 8>, (int64_t)((a.T + a.tpt - 1) / a.tpt) * a.HU, 8);
    if (a.rows == FEW_ROWS)
        return dtype == UBP_BF16 ? go(ubp_attention_join_kernel<__nv_bfloat16, false, 8>, grid, 8) : go(ubp_attention_join_kernel<__half, false, 8>, grid, 8);
    return dtype == UBP_BF16 ? go(ubp_attention_join_kernel<__nv_bfloat16, false, 32>, grid, 32) : go(ubp_attention_join_kernel<__half, false, 32>, grid, 32);
}

}  // namespace ubp
