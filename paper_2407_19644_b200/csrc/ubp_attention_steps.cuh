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

// A row's reference m lies `lift` below a score that was its largest at some time (in powers of two), and only moves when a score is
// more than `lag` above that one, so that sums are rarely rescaled: weights 2^(s - m) stay below 2^(lift + lag), and the largest is
// 2^lift or more. In bf16 a weight has the same relative error wherever it lies. f16 has 2^-24 as its smallest step, and the sum of
// weights takes them unrounded: with the reference at the largest score, a first token far above the rest whose value is near 0
// (8192 keys, scores N(0, 1), the first one 14 / 16 / 18 above 0) left relative errors of 0.008 / 0.05 / 0.3; 2^7 higher, 0.0004 /
// 0.0006 / 0.0044, where unrounded weights give 0.0002 / 0.0006 / 0.0040 (the outputs' rounding). What is compared with `lag` is the
// exponent as it is computed, by one fused product and difference, so that only the reference's own rounding, half a unit of the
// scores, can lift a weight: with scores (of base 2) below 2^28 f16's stay below their overflow, below 2^31 bf16's.
template <typename T> struct AttnRef { static constexpr float lift = 0.f, lag = 8.f; };
template <> struct AttnRef<__half> { static constexpr float lift = 7.f, lag = 5.f; };

// Shared memory of attn_locate, for blocks of NT threads.
template <int NT> struct AttnPlace { int warp[2][32]; int pre[NT + 1]; int b, rt, before, from, to; };

// The block's share of the steps, from its first one on. Called by all threads of the block, NT of them (a multiple of 32); false, to all
// of them, if there is nothing to do (or the steps of a unit head pass 32 bits). Row blocks (of all sequences, a thread each) are counted
// and summed in parallel, for one unit head: all of a sequence's have equal steps, so that step x lies in the sequence that x / HU lies in.
template <int NT>
__device__ __forceinline__ bool attn_locate(const AttnArgs &a, AttnPlace<NT> &sh, AttnDeal &deal, AttnSteps &steps)
{
    constexpr int NW = NT / 32;
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5, c = (int)blockIdx.x;
    const int nb = a.common ? 1 : a.B;
    int64_t first = 0;
    auto warp_sum = [&](int x) {        // inclusive
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        return x;
    };
    auto begin = [&](int64_t total) {
        if (total > INT_MAX) return false;      // (only starts that do not ascend get there: see the host's limit)
        deal = AttnDeal(total * a.HU, (int)gridDim.x);
        if (c >= deal.grid) return false;
        first = deal.first(c);
        steps.left = deal.count(c);
        return true;
    };
    if (nb <= 32) {                     // a few sequences of one row block each: every warp for itself, no barrier
        AttnSeq q{0, 0, 0};
        if (lane < nb) q = attn_seq(a, lane);
        const int blocks = attn_row_blocks(a, q);
        if (!__any_sync(0xffffffffu, blocks > 1)) {
            const int mine = blocks ? attn_block_tiles(a, q, 0).nt + a.extra : 0, x = warp_sum(mine);
            if (!begin(__shfl_sync(0xffffffffu, x, 31))) return false;
            const int b = __ffs(__ballot_sync(0xffffffffu, (int64_t)x * a.HU > first)) - 1;
            steps.c.set(a, b, 0, 0, 0);
            const uint32_t rem = (uint32_t)(first - (int64_t)__shfl_sync(0xffffffffu, x - mine, b) * a.HU), per = (uint32_t)__shfl_sync(0xffffffffu, mine, b);
            steps.c.hu = (int)(rem / per);
            steps.c.tile = (int)(rem - (uint32_t)steps.c.hu * per);
            steps.seek(a);
            return true;
        }
    }
    int turn = 0;
    auto scan = [&](int v, int &all) {  // -> sum before this thread
        const int x = warp_sum(v);
        if (lane == 31) sh.warp[turn][warp] = x;
        __syncthreads();
        const int w = lane < NW ? sh.warp[turn][lane] : 0, ws = warp_sum(w);
        turn ^= 1;
        all = __shfl_sync(0xffffffffu, ws, 31);
        return __shfl_sync(0xffffffffu, ws - w, warp) + x - v;
    };
    if (nb <= NT) {                     // sequences of one row block each, a thread a sequence
        AttnSeq q{0, 0, 0};
        if (tid < nb) q = attn_seq(a, tid);
        const int blocks = attn_row_blocks(a, q);
        if (!__syncthreads_or(blocks > 1)) {
            const int mine = blocks ? attn_block_tiles(a, q, 0).nt + a.extra : 0;
            int all;
            const int before = scan(mine, all);
            if (!begin(all)) return false;
            if ((int64_t)before * a.HU <= first && (int64_t)(before + mine) * a.HU > first) { sh.b = tid; sh.before = before; sh.to = mine; }
            __syncthreads();
            steps.c.set(a, sh.b, 0, 0, 0);
            const uint32_t rem = (uint32_t)(first - (int64_t)sh.before * a.HU), per = (uint32_t)sh.to;
            steps.c.hu = (int)(rem / per);
            steps.c.tile = (int)(rem - (uint32_t)steps.c.hu * per);
            __syncthreads();            // (sh may be something else from here on)
            steps.seek(a);
            return true;
        }
    }
    // all row blocks, NT at a time: visit(b, rt, steps before it, its steps) for this thread's; returns all steps
    auto walk = [&](auto &&visit) {
        int64_t sum = 0;
        for (int base = 0; base < nb; base += NT) {
            const int b = base + tid;
            AttnSeq q{0, 0, 0};
            if (b < nb) q = attn_seq(a, b);
            int blocks;
            const int at = scan(attn_row_blocks(a, q), blocks);
            sh.pre[tid] = at;
            if (tid == 0) sh.pre[NT] = blocks;
            __syncthreads();
            for (int i0 = 0; i0 < blocks; i0 += NT) {
                const int i = i0 + tid;
                int s = 0, nt = 0, all;
                if (i < blocks) {
                    for (int hi = imin(NT, nb - base); hi - s > 1;) {       // last sequence that begins at i or before (of empty ones: the one behind them)
                        const int m = (s + hi) / 2;
                        if (sh.pre[m] <= i) s = m;
                        else hi = m;
                    }
                    nt = attn_block_tiles(a, attn_seq(a, base + s), i - sh.pre[s]).nt + a.extra;
                }
                const int before = scan(nt, all);
                if (nt) visit(base + s, i - sh.pre[s], sum + before, nt);
                sum += all;
            }
            __syncthreads();
        }
        return sum;
    };
    int kb = -1, krt = 0, kbefore = 0, knt = 0;
    const int64_t total = walk([&](int b, int rt, int64_t before, int nt) { kb = b; krt = rt; kbefore = (int)before; knt = nt; });
    if (!begin(total)) return false;
    const bool once = nb <= NT && sh.pre[NT] <= NT;         // (this thread still has its row block, the only one)
    auto again = [&](auto &&visit) {
        if (!once) walk(visit);
        else if (kb >= 0) visit(kb, krt, (int64_t)kbefore, knt);
        __syncthreads();
    };
    // the sequence of the first step; its steps for one unit head; the row block
    const int64_t y = first / a.HU;
    again([&](int b, int, int64_t before, int nt) { if (y >= before && y < before + nt) sh.b = b; });
    const int b = sh.b;
    const AttnSeq q = attn_seq(a, b);
    const int last = attn_row_blocks(a, q) - 1;
    again([&](int b_, int rt, int64_t before, int nt) {
        if (b_ == b && rt == 0) sh.from = (int)before;
        if (b_ == b && rt == last) sh.to = (int)before + nt;
    });
    const int from = sh.from;
    const int64_t rem = first - (int64_t)from * a.HU;
    const int hu = rem >> 32 ? (int)(rem / (sh.to - from)) : (int)((uint32_t)rem / (uint32_t)(sh.to - from));
    const int64_t z = from + (rem - (int64_t)hu * (sh.to - from));
    again([&](int b_, int rt, int64_t before, int nt) { if (b_ == b && z >= before && z < before + nt) { sh.rt = rt; sh.before = (int)before; } });
    steps.c.set(a, b, hu, sh.rt, (int)z - sh.before);
    __syncthreads();                    // (sh may be something else from here on)
    steps.seek(a);
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
    w.lo = a.window > 0 ? imax(imax(pos, 0) - a.window + 1, 0) : 0;
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
// The first `k` of K partial results onto (M, L, o): one common reference, so that no exponential waits for another.
template <int K, int N> __device__ __forceinline__ void attn_add_all(float &M, float &L, float (&o)[N], const float2 (&ml)[K], const float (&v)[K][N], int k)
{
    float to = M, y[K];
#pragma unroll
    for (int i = 0; i < K; ++i) to = i < k ? fmaxf(to, ml[i].x) : to;
    const float x = M == -INFINITY ? L : attn_exp2(M - to);
    L *= x;
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = x == 0.f ? 0.f : o[j] * x;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        if (i >= k) break;
        y[i] = ml[i].x == -INFINITY ? ml[i].y : attn_exp2(ml[i].x - to);
        L = fmaf(ml[i].y, y[i], L);
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] += y[i] == 0.f ? 0.f : v[i][j] * y[i];
    }
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
// Finished sums of a row, from column col on, to the output: o / L, 0 where nothing was seen. (A single part's sums of such a row may hold
// 0 times infinity; attn_add and attn_add_all leave them out.)
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
