// Device side of the attention kernels' schedule: where a block starts, which rows an item has, and the join of partial results.
#ifndef UBP_ATTENTION_STEPS_CUH_
#define UBP_ATTENTION_STEPS_CUH_

#include "ubp_attention.h"
#include "ubp_types.cuh"

namespace ubp {

__device__ __forceinline__ float attn_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct AttnPlace { int64_t warp[32]; int64_t rem; int b; };

// Steps of sequence b (none where !valid); called by whole warps. A lane counts its own sequence's row blocks while they are few,
// the warp counts those of long prompts together.
__device__ __forceinline__ int64_t attn_seq_steps(const AttnArgs &a, int b, bool valid)
{
    const int lane = threadIdx.x & 31;
    int n = 0;
    AttnSeq q{0, 0, 0};
    if (valid) { q = attn_seq(a, b); n = attn_row_blocks(a, q); }
    int64_t c = 0;
    if (n <= 2)
        for (int rt = 0; rt < n; ++rt) c += attn_block_tiles(a, q, rt).nt;
    for (uint32_t big = __ballot_sync(0xffffffffu, n > 2); big; big &= big - 1) {
        const int src = __ffs(big) - 1;
        AttnSeq w;
        w.s = __shfl_sync(0xffffffffu, q.s, src);
        w.n = __shfl_sync(0xffffffffu, q.n, src);
        w.len = __shfl_sync(0xffffffffu, q.len, src);
        const int m = attn_row_blocks(a, w);
        int64_t s = 0;
        for (int rt = lane; rt < m; rt += 32) s += attn_block_tiles(a, w, rt).nt;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == src) c = s;
    }
    return c * a.HU;
}

// The cursor at step rem of sequence b; called by whole warps.
__device__ __forceinline__ void attn_place(const AttnArgs &a, int b, int64_t rem, AttnCursor &cur)
{
    const int lane = threadIdx.x & 31;
    const AttnSeq q = attn_seq(a, b);
    const int m = attn_row_blocks(a, q);
    if (m == 1) {
        const int n = attn_block_tiles(a, q, 0).nt, hu = rem >> 32 ? (int)(rem / n) : (int)((uint32_t)rem / (uint32_t)n);
        cur.set(a, b, hu, 0, (int)(rem - (int64_t)hu * n));
        return;
    }
    int64_t per = 0;
    for (int i = lane; i < m; i += 32) per += attn_block_tiles(a, q, i).nt;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) per += __shfl_xor_sync(0xffffffffu, per, o);
    const int hu = (int)(rem / per);
    int rt = 0;
    rem -= (int64_t)hu * per;
    for (int i = 0; i < m; i += 32) {
        const int n = i + lane < m ? attn_block_tiles(a, q, i + lane).nt : 0;
        int64_t x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        const uint32_t in = __ballot_sync(0xffffffffu, x > rem);
        if (in) {
            const int src = __ffs(in) - 1;
            rem -= __shfl_sync(0xffffffffu, x - n, src);
            rt = i + src;
            break;
        }
        rem -= __shfl_sync(0xffffffffu, x, 31);
    }
    cur.set(a, b, hu, rt, (int)rem);
}

// The block's steps, [first, first + count), and the cursor at the first one. Called by all threads of the block (a multiple of
// 32); returns false, to all of them, if there is nothing to do.
__device__ __forceinline__ bool attn_locate(const AttnArgs &a, AttnPlace &sh, AttnDeal &deal, int64_t &first, int64_t &count, AttnCursor &cur)
{
    const int nt = (int)blockDim.x, tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = nt >> 5;
    const int nb = a.common ? 1 : a.B;
    if (nb <= 32) {                     // every warp for itself: no barrier
        const int64_t mine = attn_seq_steps(a, lane, lane < nb);
        int64_t x = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        deal = AttnDeal(__shfl_sync(0xffffffffu, x, 31), (int)gridDim.x);
        const int c = (int)blockIdx.x;
        if (c >= deal.grid) return false;
        first = deal.first(c);
        count = deal.count(c);
        const int b = __ffs(__ballot_sync(0xffffffffu, x > first)) - 1;
        attn_place(a, b, first - __shfl_sync(0xffffffffu, x - mine, b), cur);
        return true;
    }
    int64_t total = 0, mine = 0, before = 0;       // steps of this thread's sequence, and of all sequences before it in the chunk
    auto scan = [&](int base) {         // -> steps of the chunk of nt sequences from base on
        const int b = base + tid;
        mine = attn_seq_steps(a, b, b < nb);
        int64_t x = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        __syncthreads();
        if (lane == 31) sh.warp[warp] = x;
        __syncthreads();
        int64_t w = 0, all = 0;
        for (int i = 0; i < nw; ++i) {
            const int64_t v = sh.warp[i];
            if (i < warp) w += v;
            all += v;
        }
        before = w + x - mine;
        return all;
    };
    for (int base = 0; base < nb; base += nt) total += scan(base);
    deal = AttnDeal(total, (int)gridDim.x);
    const int c = (int)blockIdx.x;
    if (c >= deal.grid) return false;
    first = deal.first(c);
    count = deal.count(c);
    int64_t at = first;
    for (int base = 0; base < nb; base += nt) {
        const int64_t all = nb > nt ? scan(base) : total;
        if (at < all) {
            if (at >= before && at < before + mine) { sh.b = base + tid; sh.rem = at - before; }
            break;
        }
        at -= all;
    }
    __syncthreads();
    attn_place(a, sh.b, sh.rem, cur);
    return true;
}

// sequence of a token, -1 for one behind the last
__device__ __forceinline__ int attn_seq_of(const int32_t *starts, int B, int t)
{
    int lo = 0, hi = B;                  // largest b with starts[b] <= t
    if (starts[0] > t) return -1;
    while (hi - lo > 1) {
        const int m = lo + (hi - lo) / 2;
        if (starts[m] <= t) lo = m;
        else hi = m;
    }
    return t < starts[lo + 1] ? lo : -1;
}

// Row r of a row block with n tokens from token t0 on: its token (-1 if the row does not exist) and query head.
__device__ __forceinline__ int2 attn_row_at(const AttnArgs &a, int t0, int n, int hu, int r)
{
    const int per = a.rows / a.tiles, tile = r >= per ? 1 : 0, i = r - tile * per, tpt = a.tpt / a.tiles;
    const int ti = (int)((uint32_t)i / (uint32_t)a.gc), kvh = (int)((uint32_t)hu / (uint32_t)a.chunks);
    const int g = (hu - kvh * a.chunks) * a.gc + i - ti * a.gc, t = tile * tpt + ti;
    return ti < tpt && g < a.G && t < n ? make_int2(t0 + t, kvh * a.G + g) : make_int2(-1, 0);
}

// A row of an item: its token among the call's, its query head, and the keys that it sees: j < hi and (j >= lo or j < sinks), of
// [kv0, kv1). A row that does not exist has token -1 and sees nothing.
struct AttnRow { int token, head, lo, hi; };
__device__ __forceinline__ AttnRow attn_row(const AttnArgs &a, const AttnSeq &q, int hu, int rt, int r)
{
    const int2 at = attn_row_at(a, q.s + rt * a.tpt, q.n - rt * a.tpt, hu, r);
    AttnRow w{at.x, at.y, 0, 0};
    if (w.token < 0) return w;
    int pos = q.len - q.n + w.token - q.s;
    if (a.common) {
        const int t = w.token, b = a.starts ? attn_seq_of(a.starts, a.B, t) : t;
        if (b < 0) { w.token = -1; return w; }
        const int s = a.starts ? imax(a.starts[b], 0) : t, e = a.starts ? imin(a.starts[b + 1], a.T) : t + 1;
        pos = imin(imax(a.lengths[b], 0), a.cap) - (e - s) + (t - s);
    }
    w.hi = imin(pos + 1, a.kv1);
    w.lo = a.window > 0 ? imax(pos - a.window + 1, 0) : 0;
    return w;
}
__device__ __forceinline__ bool attn_sees(const AttnArgs &a, const AttnRow &w, int j)
{
    return j < w.hi && j >= a.kv0 && (j >= w.lo || j < a.sinks);
}

// One more partial result (reference m, sum l, N values) onto (M, L, o). A reference of -inf stands for no score above it: the sum
// is 0 then, or NaN where a score was NaN, which stays.
template <int N> __device__ __forceinline__ void attn_add(float &M, float &L, float (&o)[N], float m, float l, const float (&v)[N])
{
    const float to = fmaxf(M, m);
    const float x = M == -INFINITY ? L : attn_exp2(M - to), y = m == -INFINITY ? l : attn_exp2(m - to);
    L = L * x + l * y;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = (x == 0.f ? 0.f : o[i] * x) + (y == 0.f ? 0.f : v[i] * y);
    M = to;
}
template <int N> __device__ __forceinline__ void attn_load(const float *p, float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float4 f = *reinterpret_cast<const float4 *>(p + i);
        v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
    }
}
template <typename T, int N> __device__ __forceinline__ void attn_store(T *p, const float (&v)[N])
{
    static_assert(N == 4 || N == 8, "");
    if ((reinterpret_cast<uintptr_t>(p) & (N * sizeof(T) - 1)) == 0) {
        if constexpr (N == 8) store8<T>(p, v);
        else *reinterpret_cast<uint2 *>(p) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = from_f32<T>(v[i]);
    }
}
// Finished sums of a row, from column col on, to the output: o / L, 0 where nothing was seen.
template <typename T, int N> __device__ __forceinline__ void attn_finish(const AttnArgs &a, int token, int head, int col, float M, float L, float (&o)[N])
{
    if (a.pml) {
        const int64_t at = (int64_t)token * a.Hq + head;
        const float2 ml = a.pml[at];
        float v[N];
        attn_load(a.ppo + at * a.D + col, v);
        attn_add(M, L, o, ml.x, ml.y, v);
    }
    const float r = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] *= r;
    attn_store(static_cast<T *>(a.out) + token * a.o_ts + head * a.o_hs + col, o);
}

// What block c leaves behind for the join: its last item if that begins here and ends in a later block, as {first token, tokens,
// unit head, 2 * blocks that share it + (the item is not the block's first segment)}.
// x: the block's steps before its last segment, n: that segment's tiles, tile0: the first of them.
__device__ __forceinline__ void attn_describe(const AttnArgs &a, const AttnCursor &at, const AttnDeal &deal, int c, int64_t x, int tile0, int n)
{
    int4 d = make_int4(0, 0, 0, 0);
    if (tile0 == 0 && n < at.t.nt) {
        const int last = deal.owner(deal.first(c) + x + at.t.nt - 1);
        d = make_int4(at.q.s + at.rt * a.tpt, at.q.n - at.rt * a.tpt, at.hu, (last - c + 1) << 1 | (x > 0 ? 1 : 0));
    }
    a.desc[c] = d;
}

}  // namespace ubp
#endif
