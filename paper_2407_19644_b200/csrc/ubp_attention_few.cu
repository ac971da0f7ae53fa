// Attention of a few query rows over a paged cache: single tokens of running answers (and any other item, 16 rows at a time).
//
//   s_j = scale q.k_j,  o = sum_j 2^(s_j log2e - m) v_j / sum_j 2^(s_j log2e - m)     over the keys j that the row sees
//
// One pass over the keys and values with a running reference m and sum: bound by HBM, 4 D bytes a key and key head. The 16 rows
// of an item are the query heads of one key head (and neighbouring tokens), so that a key is read once for all of them, and they
// are the rows of an m16n8k16 product: at 16 rows it is 16 multiply-adds a value read, a tenth of what the SM could do in the time
// HBM takes for that value, so the unused rows of small groups cost nothing.
// Eight warps a block; a warp has its own 16 keys of a step's 128, its own ring of copies (16-byte cp.async, so that any strides,
// pages and ends of sequences are taken row by row) and its own running sums: nothing in the loop waits for another warp. They
// meet once an item. Copies run ahead over the ends of items.
// Keys outside what any row of the item sees are not read: their places hold zeros, so that nothing an unused slot of a page
// holds reaches a result. The weights are rounded to 16 bits for the second product (relative 2^-9 / 2^-12 each, the sum of
// weights is of the unrounded ones); scores, references, sums and outputs are fp32 until the end.
#include <cuda_runtime.h>

#include <type_traits>

#include "ubp_attention_steps.cuh"

namespace ubp {
namespace {

constexpr int FEW_WARPS = 8, FEW_KEYS = 16, FEW_ROWS = 16;
constexpr int FEW_BN = FEW_WARPS * FEW_KEYS;
static_assert(FEW_ROWS == 16 && FEW_BN == 128, "as the launch fills AttnArgs");
__host__ __device__ constexpr int few_stages(int dp) { return dp == 128 ? 3 : 6; }
__host__ __device__ constexpr int few_part(int dp) { return FEW_KEYS * dp * 2; }                    // keys (or values) of a warp's step
__host__ __device__ constexpr int few_ring(int dp) { return few_stages(dp) * 2 * few_part(dp); }     // a warp's
__host__ __device__ constexpr int few_smem(int dp) { return FEW_WARPS * (few_ring(dp) + 8 * dp * 4 + FEW_ROWS * 8); }

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool valid)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
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
// two neighbouring elements, whatever their alignment
template <typename T> __device__ __forceinline__ uint32_t load_pair(const T *p)
{
    if ((reinterpret_cast<uintptr_t>(p) & 3) == 0) return *reinterpret_cast<const uint32_t *>(p);
    const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
    return (uint32_t)h[0] | (uint32_t)h[1] << 16;
}

// The copies of a warp's steps: a cursor that runs ahead, with the page of the next step's keys already loaded.
template <typename T, int DP> struct FewCopies {
    AttnCursor c;
    int64_t left;            // steps that are not issued yet
    int page0, page1;        // pages of the step's first and last eight keys
    int j0;

    __device__ __forceinline__ int page_of(const AttnArgs &a, int j) const
    {
        return j < c.t.end ? a.table[(a.common ? 0 : (int64_t)c.b * a.ldt) + (j >> a.pshift)] : -1;
    }
    __device__ __forceinline__ void peek(const AttnArgs &a, int warp)
    {
        j0 = attn_tile_at(c.t, c.tile) * FEW_BN + warp * FEW_KEYS;
        page0 = page_of(a, j0);
        page1 = a.pshift > 3 ? page0 : page_of(a, j0 + 8);
    }
    __device__ __forceinline__ void issue(const AttnArgs &a, uint32_t stage, int warp, int lane)
    {
        if (left > 0) {
            constexpr int CH = DP / 8, RPI = 32 / CH;
            const int ch = lane % CH;
            const int kvh = c.hu / a.chunks;
            if (ch * 8 < (a.D + 15) / 16 * 16) {
#pragma unroll
                for (int i = 0; i < FEW_KEYS / RPI; ++i) {
                    const int r = i * RPI + lane / CH, j = j0 + r, page = r < 8 ? page0 : page1;
                    const bool in = ch * 8 < a.D && j >= a.kv0 && j < c.t.end && (j >= c.t.w0 || j < a.sinks) && (uint32_t)page < (uint32_t)a.pages;
                    const int64_t at = in ? page * a.c_ps + kvh * a.c_hs + (j & ((1 << a.pshift) - 1)) * a.c_ts + ch * 8 : 0;
                    const uint32_t to = stage + (uint32_t)(r * DP * 2 + ((ch ^ (r & 7)) << 4));
                    cp16(to, static_cast<const T *>(a.k) + at, in);
                    cp16(to + few_part(DP), static_cast<const T *>(a.v) + at, in);
                }
            }
            --left;
            c.next(a, left > 0);
            if (left > 0) peek(a, warp);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
};

template <typename T, int DP>
__global__ void __launch_bounds__(FEW_WARPS * 32, 1) ubp_attention_few_kernel(const AttnArgs a)
{
    constexpr int ST = few_stages(DP), NK = DP / 16;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ AttnPlace place;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, tq = lane & 3;
    float *const meet = reinterpret_cast<float *>(smem + FEW_WARPS * few_ring(DP));                  // [warp][8 rows][DP]
    float2 *const meet_ml = reinterpret_cast<float2 *>(meet + FEW_WARPS * 8 * DP);                    // [warp][row]
    const uint32_t ring = smem_at(smem) + (uint32_t)(warp * few_ring(DP));

    int64_t total, first, count;
    int grid;
    AttnCursor cur;
    if (!attn_locate(a, place, total, first, count, grid, cur)) {
        if (threadIdx.x == 0 && !a.common) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
        return;
    }
    FewCopies<T, DP> copies;
    copies.c = cur;
    copies.left = count;
    copies.peek(a, warp);
    for (int s = 0; s < ST - 1; ++s) copies.issue(a, ring + (uint32_t)(s * 2 * few_part(DP)), warp, lane);

    uint32_t qf[NK][4];
    float o[DP / 8][4], m[2], l[2];
    AttnRow row[2];
    int tile0 = cur.tile, st = 0;
    bool fresh = true;
    for (int64_t step = 0; step < count; ++step) {
        __syncwarp();                       // (all lanes have read the stage that is copied to now)
        copies.issue(a, ring + (uint32_t)((st + ST - 1) % ST * 2 * few_part(DP)), warp, lane);
        if (fresh) {
            fresh = false;
            tile0 = cur.tile;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                row[i] = attn_row(a, cur.q, cur.hu, cur.rt, g + 8 * i);
                m[i] = -INFINITY; l[i] = 0.f;
                const T *p = static_cast<const T *>(a.q) + (row[i].token < 0 ? 0 : row[i].token * a.q_ts + row[i].head * a.q_hs);
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int d = k * 16 + h * 8 + tq * 2;
                        qf[k][h * 2 + i] = row[i].token >= 0 && d < a.D ? load_pair<T>(p + d) : 0u;
                    }
            }
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
        __syncwarp();
        const int j0 = attn_tile_at(cur.t, cur.tile) * FEW_BN + warp * FEW_KEYS;
        const uint32_t ks = ring + (uint32_t)(st * 2 * few_part(DP)), vs = ks + few_part(DP);
        if (j0 < cur.t.end && (j0 + FEW_KEYS > cur.t.w0 || j0 < a.sinks)) {
            float s[2][4] = {};
            {
                const int r = (lane & 7) + (lane >> 4) * 8;
                const uint32_t at = ks + (uint32_t)(r * DP * 2);
#pragma unroll
                for (int k = 0; k < NK; ++k)
                    if (k * 16 < a.D) {
                        uint32_t b[4];
                        ldsm4(b, at + (uint32_t)(((2 * k + (lane >> 3 & 1)) ^ (r & 7)) << 4));
                        mma16<T>(s[0], qf[k], b[0], b[1]);
                        mma16<T>(s[1], qf[k], b[2], b[3]);
                    }
            }
            float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[n][e] = attn_sees(a, row[e >> 1], j0 + n * 8 + tq * 2 + (e & 1)) ? s[n][e] * a.sc : -INFINITY;
                    mx[e >> 1] = fmaxf(mx[e >> 1], s[n][e]);
                }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
            }
            // The reference only moves when a score lies more than 2^8 above it: weights stay below 2^8, sums far from overflow.
            if (__any_sync(0xffffffffu, mx[0] > m[0] + 8.f || mx[1] > m[1] + 8.f)) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float to = fmaxf(m[i], mx[i]), f = m[i] == -INFINITY ? 0.f : attn_exp2(m[i] - to);
                    m[i] = to;
                    l[i] *= f;
#pragma unroll
                    for (int n = 0; n < DP / 8; ++n) { o[n][2 * i] *= f; o[n][2 * i + 1] *= f; }
                }
            }
            uint32_t p[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float ref = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float p0 = attn_exp2(s[n][2 * i] - ref), p1 = attn_exp2(s[n][2 * i + 1] - ref);
                    l[i] += p0 + p1;
                    p[n * 2 + i] = pack2<T>(p0, p1);
                }
            }
            {
                const int r = (lane & 7) + (lane >> 3 & 1) * 8;
                const uint32_t at = vs + (uint32_t)(r * DP * 2);
#pragma unroll
                for (int n = 0; n < NK; ++n)
                    if (n * 16 < a.D) {
                        uint32_t b[4];
                        ldsm4t(b, at + (uint32_t)(((2 * n + (lane >> 4)) ^ (r & 7)) << 4));
                        mma16<T>(o[2 * n], p, b[0], b[1]);
                        mma16<T>(o[2 * n + 1], p, b[2], b[3]);
                    }
            }
        }
        st = st + 1 == ST ? 0 : st + 1;
        const bool last = step + 1 == count;
        if (cur.tile + 1 == cur.t.nt || last) {
            // ---- the warps' sums meet: rows 0 .. 7, then 8 .. 15 where the item has them
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
                if (tq == 0) meet_ml[warp * FEW_ROWS + g + 8 * i] = make_float2(m[i], l[i]);
            }
            const int nr = imin(imin(a.tpt, cur.q.n - cur.rt * a.tpt) * a.gc, FEW_ROWS), n = cur.tile + 1 - tile0;
            const bool whole = n == cur.t.nt && !a.common;
            const int c = (int)blockIdx.x;
            int64_t slot = 2 * (int64_t)c + (step + 1 - n > 0 ? 1 : 0);
            if (a.common) slot = (int64_t)cur.hu * attn_row_blocks(a, cur.q) + cur.rt + c;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (i * 8 >= nr) break;
                if (i) __syncthreads();
#pragma unroll
                for (int k = 0; k < DP / 8; ++k)
                    *reinterpret_cast<float2 *>(meet + (warp * 8 + g) * DP + k * 8 + tq * 2) = make_float2(o[k][2 * i], o[k][2 * i + 1]);
                __syncthreads();
                constexpr int N = 4, TPR = DP / N;          // threads a row
                for (int x = (int)threadIdx.x; x < 8 * TPR; x += FEW_WARPS * 32) {
                    const int r = x / TPR, col = x % TPR * N;
                    const AttnRow w = attn_row(a, cur.q, cur.hu, cur.rt, i * 8 + r);
                    if (col < a.D && (w.token >= 0 || !whole)) {
                        float M = -INFINITY, L = 0.f, v[N] = {};
#pragma unroll
                        for (int k = 0; k < FEW_WARPS; ++k) {
                            const float2 ml = meet_ml[k * FEW_ROWS + i * 8 + r];
                            float u[N];
                            attn_load(meet + (k * 8 + r) * DP + col, u);
                            attn_add(M, L, v, ml.x, ml.y, u);
                        }
                        if (whole) attn_finish<T>(a, w, col, M, L, v);
                        else {
                            if (col == 0) a.ml[slot * FEW_ROWS + i * 8 + r] = make_float2(M, L);
                            *reinterpret_cast<float4 *>(a.po + (slot * FEW_ROWS + i * 8 + r) * a.D + col) = make_float4(v[0], v[1], v[2], v[3]);
                        }
                    }
                }
            }
            __syncthreads();
            if (last && threadIdx.x == 0 && !a.common) attn_describe(a, cur, total, grid, c, first, first + step + 1 - n, tile0, n);
            fresh = true;
        }
        cur.next(a, !last);
    }
}

// Joins the partial results of an item that several blocks have worked on: block (c, i) rows 16 i .. 16 i + 15 of the item that
// begins in block c, in the order of its keys.
template <typename T>
__global__ void __launch_bounds__(256) ubp_attention_join_kernel(const AttnArgs a)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int c = (int)blockIdx.x;
    const int4 d = a.desc[c];
    const int parts = d.w >> 1;
    if (parts == 0) return;
    const AttnSeq q = attn_seq(a, d.x);
    constexpr int N = 4;
    const int per = a.D / N;
    for (int x = (int)threadIdx.x; x < 16 * per; x += 256) {
        const int r = (int)blockIdx.y * 16 + x / per, col = x % per * N;
        const AttnRow w = attn_row(a, q, d.y, d.z, r);
        if (w.token < 0) continue;
        float M = -INFINITY, L = 0.f, o[N] = {};
        for (int k = 0; k < parts; ++k) {
            const int64_t at = (2 * (int64_t)(c + k) + (k == 0 ? (d.w & 1) : 0)) * a.rows + r;
            const float2 ml = a.ml[at];
            float v[N];
            attn_load(a.po + at * a.D + col, v);
            attn_add(M, L, o, ml.x, ml.y, v);
        }
        attn_finish<T>(a, w, col, M, L, o);
    }
}

int attn_fail(cudaError_t e) { set_last_cuda_error((int)e); return UBP_E_CUDA; }

template <typename K>
int launch_after(K kern, dim3 grid, int threads, size_t smem, const AttnArgs &a, void *stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, a);
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? UBP_OK : attn_fail(e);
}

template <typename T, int DP> int launch_few_t(const AttnArgs &a, int grid, void *stream)
{
    const auto kern = ubp_attention_few_kernel<T, DP>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, few_smem(DP));
    if (e != cudaSuccess) return attn_fail(e);
    return launch_after(kern, dim3((unsigned)grid), FEW_WARPS * 32, few_smem(DP), a, stream);
}

}  // namespace

int launch_attn_few(const AttnArgs &a, int dtype, int grid, void *stream)
{
    if (dtype == UBP_BF16) return a.D <= 64 ? launch_few_t<__nv_bfloat16, 64>(a, grid, stream) : launch_few_t<__nv_bfloat16, 128>(a, grid, stream);
    return a.D <= 64 ? launch_few_t<__half, 64>(a, grid, stream) : launch_few_t<__half, 128>(a, grid, stream);
}

int launch_attn_join(const AttnArgs &a, int dtype, int grid, void *stream)
{
    const dim3 g((unsigned)grid, (unsigned)((a.rows + 15) / 16));
    return dtype == UBP_BF16 ? launch_after(ubp_attention_join_kernel<__nv_bfloat16>, g, 256, 0, a, stream)
                             : launch_after(ubp_attention_join_kernel<__half>, g, 256, 0, a, stream);
}

}  // namespace ubp
