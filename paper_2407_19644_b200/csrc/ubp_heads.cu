// Rows of a query, key and value projection -> queries, and keys and values in a paged cache, in one pass: the norm of each query
// and key head, the position rotation, the copy to the pages.
//
//   u = x / sqrt(mean(x^2) + eps) * gamma                                   query and key heads, where a gamma is given
//   (u_i, u_j) -> (u_i cos - u_j sin, u_j cos + u_i sin)                     j = i + r / 2, i < r / 2; or (i, j) = (2 i, 2 i + 1)
//
// Bound by HBM: every value is read once and written once (2 + 2 bytes), and a token's rotation (r fp32 numbers) is read once for
// all its heads. A thread holds two 16-byte pieces of a head that are rotated into one another, so that no pair needs another
// thread; D / 16 threads share a head, and their part of the rotation stays in registers from head to head. Statistics, rotation
// and products are fp32, each value is rounded once.
// Measured: 16384 tokens of 48 heads of 128 values with norms 73 us, 5.6 TB/s; 1531 tokens of 20 heads of 80 in rows off 16 bytes 6.6
// us; one token of 48 heads 2.3.
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "ubp_attention.h"
#include "ubp_f32x2.cuh"
#include "ubp_types.cuh"

namespace ubp {

int check_cache(const ubp_cache_t *c, int64_t T, int q_heads);

namespace {

struct HeadArgs {
    const void *qkv;
    int64_t ld;
    const void *q_gamma, *k_gamma;
    const float *rot;               // [positions][r]: cosines, then sines; null: no rotation
    int64_t ldrot;
    int positions, r, interleaved;
    float eps;
    void *q;
    int64_t q_ts, q_hs;
    void *k, *v;
    int64_t c_ps, c_hs, c_ts;
    const int32_t *table, *lengths, *starts;
    int64_t ldt;
    int pages, pshift, cap;
    int T, B, Hq, Hkv, D;
    float inv_d;
};

// Sequence of token t, -1 for one behind the last; called by whole warps: 32 places of the starts at a time.
__device__ __forceinline__ int seq_of(const HeadArgs &a, int t)
{
    if (!a.starts) return t;
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = a.B;
    while (true) {
        const int step = (hi - lo + 31) / 32, i = lo + lane * step;
        const uint32_t in = __ballot_sync(0xffffffffu, i < hi && a.starts[i < hi ? i : lo] <= t);
        if (!in) return -1;
        lo += (31 - __clz(in)) * step;
        hi = imin(hi, lo + step);
        if (step == 1) break;
    }
    return t < a.starts[lo + 1] ? lo : -1;
}

// Where a token stands: its position (-1: none that the rotation has) and its place in a page (-1: it has none).
struct Place { int pos; int64_t at; };
__device__ __forceinline__ Place place_of(const HeadArgs &a, int b, int pos)
{
    Place p{-1, -1};
    if (pos < 0 || (a.rot && pos >= a.positions)) return p;
    p.pos = pos;
    if (pos < a.cap) {
        const int page = a.table[b * a.ldt + (pos >> a.pshift)];
        if ((uint32_t)page < (uint32_t)a.pages) p.at = page * a.c_ps + (pos & ((1 << a.pshift) - 1)) * a.c_ts;
    }
    return p;
}

// Eight values as they lie in memory <-> four fp32 pairs
template <typename T> __device__ __forceinline__ void pairs_of(const uint4 &w, uint64_t (&v)[4])
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<T>(u[i]);
        v[i] = pair(f.x, f.y);
    }
}
template <typename T> __device__ __forceinline__ uint4 packed(const uint64_t (&v)[4])
{
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        halves(v[i], a, b);
        u[i] = pack2<T>(a, b);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

constexpr int HEADS_BLOCKS = 6;         // an SM holds
// TPH: threads a head (a power of two, D / 16 of them at work). A block takes consecutive tokens, whose sequence and position
// follow from one another, and its groups of TPH threads a token's heads in turns, AHEAD of a group's together.
// STAGED: rows of qkv off 16 bytes come through shared memory, whole 16-byte lines of memory (all of a turn's under way together)
// and single elements at the ends, so that everything behind is the same (all elements singly: 7.6 us where it takes 6.6; with three
// heads of a group together, whose lines do not fit the registers, 9.4).
template <typename T, int TPH, bool INTER, bool STAGED, int AHEAD>
__global__ void __launch_bounds__(128, HEADS_BLOCKS) ubp_heads_kernel(const HeadArgs a, const int per)
{
    constexpr int GROUPS = 128 / TPH;
    __shared__ __align__(16) T stage[STAGED ? AHEAD * GROUPS * TPH * 16 : 8];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int H = a.Hq + 2 * a.Hkv, part = threadIdx.x % TPH, group = threadIdx.x / TPH, rp = a.r / 16;
    const int64_t t0 = (int64_t)blockIdx.x * per;
    const int end = (int)(t0 + per < a.T ? t0 + per : a.T);
    const bool live = part < a.D / 16;
    // the thread's two pieces of a head
    const int c0 = 8 * (INTER || part >= rp ? 2 * part : part), c1 = INTER || part >= rp ? c0 + 8 : c0 + 8 * rp;
    uint4 cur[AHEAD][2];
    const int stride = (int)gridDim.y * GROUPS * AHEAD, h_first = (int)blockIdx.y * GROUPS * AHEAD;
    auto fetch = [&](int t, int h0) {   // heads h0 + i * GROUPS + group of token t
        const T *row = static_cast<const T *>(a.qkv) + t * a.ld;
        if constexpr (STAGED) {
            const int first = h0 * a.D, n = imin(AHEAD * GROUPS, H - h0) * a.D;
            const T *const src = row + first;
            const int head = imin(n, (int)((16 - (reinterpret_cast<uintptr_t>(src) & 15)) & 15) / 2), body = (n - head) / 8, rest = n - head - 8 * body;
            constexpr int V = (AHEAD * GROUPS * TPH * 16 / 8 + 127) / 128;
            uint4 w[V];
#pragma unroll
            for (int i = 0; i < V; ++i)
                if ((int)threadIdx.x + i * 128 < body) w[i] = reinterpret_cast<const uint4 *>(src + head)[threadIdx.x + i * 128];
            const int edge = (int)threadIdx.x < head ? (int)threadIdx.x : head + 8 * body + (int)threadIdx.x - head;
            uint16_t x = 0;
            if ((int)threadIdx.x < head + rest) x = reinterpret_cast<const uint16_t *>(src)[edge];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i)
                if ((int)threadIdx.x + i * 128 < body) {
                    uint16_t *const to = reinterpret_cast<uint16_t *>(stage) + head + 8 * ((int)threadIdx.x + i * 128);
                    const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) { to[2 * k] = (uint16_t)u[k]; to[2 * k + 1] = (uint16_t)(u[k] >> 16); }
                }
            if ((int)threadIdx.x < head + rest) reinterpret_cast<uint16_t *>(stage)[edge] = x;
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int k = i * GROUPS + group;
            if (live && h0 + k < H) {
                const T *p = STAGED ? stage + k * a.D : row + (int64_t)(h0 + k) * a.D;
                cur[i][0] = *reinterpret_cast<const uint4 *>(p + c0);
                cur[i][1] = *reinterpret_cast<const uint4 *>(p + c1);
            }
        }
    };
    int t = (int)t0;
    int b = -1, s = 0, e = 0, len = 0;  // sequence of the token, its rows s .. e - 1
    Place pl{-1, -1};
    bool rotated = false;
    // the thread's part of the token's rotation: cosines, sines, and the sines' negatives (neighbouring pairs: (c, c) and (-s, s))
    uint64_t cs[INTER ? 8 : 4], sn[INTER ? 8 : 4], ns[INTER ? 1 : 4];
    for (int h0 = h_first; t < end;) {
        fetch(t, h0);
        if (h0 == h_first) {            // a token begins
            if (b < 0 || t >= e) {
                b = seq_of(a, t);
                s = t; e = t + 1;
                if (b >= 0) {
                    if (a.starts) { s = imax(a.starts[b], 0); e = imin(a.starts[b + 1], a.T); }
                    len = imax(a.lengths[b], 0);
                }
            }
            pl = b >= 0 ? place_of(a, b, len - (e - s) + (t - s)) : Place{-1, -1};
            rotated = a.rot && part < rp && pl.pos >= 0;
            if (rotated) {
                const float *p = a.rot + pl.pos * a.ldrot + 8 * part;
                float c[8], n[8];
                load8(p, c);
                load8(p + a.r / 2, n);
                if constexpr (INTER) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) { cs[j] = pair(c[j], c[j]); sn[j] = pair(-n[j], n[j]); }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        cs[j] = pair(c[2 * j], c[2 * j + 1]);
                        sn[j] = pair(n[2 * j], n[2 * j + 1]);
                        ns[j] = pair(-n[2 * j], -n[2 * j + 1]);
                    }
                }
            }
        }
        const int now = h0, tok = t;
        h0 += stride;
        if (h0 >= H) { h0 = h_first; ++t; }
        if (b < 0) continue;            // (a token of no sequence)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int h = now + i * GROUPS + group;
            const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv, on = live && h < H;
            const T *gamma = static_cast<const T *>(is_q ? a.q_gamma : is_k ? a.k_gamma : nullptr);
            uint64_t x[4], y[4], z = 0;
            if (on && (is_q || is_k)) {
                pairs_of<T>(cur[i][0], x);
                pairs_of<T>(cur[i][1], y);
                if (gamma) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) z = fma2(x[j], x[j], fma2(y[j], y[j], z));
                }
            }
            float sum, half;
            halves(z, sum, half);
            sum += half;
#pragma unroll
            for (int o = TPH / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (!on) continue;
            if (is_q || is_k) {
                if (gamma) {
                    const float r = rsqrtf(fmaf(sum, a.inv_d, a.eps));
                    const uint64_t r2 = pair(r, r);
                    uint64_t g[4];
                    pairs_of<T>(*reinterpret_cast<const uint4 *>(gamma + c0), g);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = mul2(x[j], mul2(r2, g[j]));
                    pairs_of<T>(*reinterpret_cast<const uint4 *>(gamma + c1), g);
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[j] = mul2(y[j], mul2(r2, g[j]));
                }
                if (rotated) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if constexpr (INTER) {
                            float u, w;
                            halves(x[j], u, w);
                            x[j] = fma2(pair(w, u), sn[j], mul2(x[j], cs[j]));
                            halves(y[j], u, w);
                            y[j] = fma2(pair(w, u), sn[4 + j], mul2(y[j], cs[4 + j]));
                        } else {
                            const uint64_t u = x[j];
                            x[j] = fma2(y[j], ns[j], mul2(u, cs[j]));
                            y[j] = fma2(u, sn[j], mul2(y[j], cs[j]));
                        }
                    }
                }
                if (gamma || rotated) { cur[i][0] = packed<T>(x); cur[i][1] = packed<T>(y); }
            }
            T *p;
            if (is_q) {
                p = static_cast<T *>(a.q) + tok * a.q_ts + h * a.q_hs;
                if (pl.pos < 0) cur[i][0] = cur[i][1] = make_uint4(0, 0, 0, 0);
            } else {
                if (pl.at < 0) continue;
                p = static_cast<T *>(is_k ? a.k : a.v) + pl.at + (is_k ? h - a.Hq : h - a.Hq - a.Hkv) * a.c_hs;
            }
            *reinterpret_cast<uint4 *>(p + c0) = cur[i][0];
            *reinterpret_cast<uint4 *>(p + c1) = cur[i][1];
        }
    }
}

// Any layout: a warp a head, single elements.
template <typename T>
__global__ void __launch_bounds__(128) ubp_heads_any_kernel(const HeadArgs a)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int t = (int)blockIdx.x, b = seq_of(a, t), lane = threadIdx.x & 31;
    if (b < 0) return;
    const int first = a.starts ? imax(a.starts[b], 0) : t, last = a.starts ? imin(a.starts[b + 1], a.T) : t + 1;
    const Place pl = place_of(a, b, imax(a.lengths[b], 0) - (last - first) + (t - first));
    const int H = a.Hq + 2 * a.Hkv, half = a.r / 2;
    const float *rot = a.rot && pl.pos >= 0 ? a.rot + pl.pos * a.ldrot : nullptr;
    for (int h = (int)blockIdx.y * 4 + (threadIdx.x >> 5); h < H; h += (int)gridDim.y * 4) {
        const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
        const T *x = static_cast<const T *>(a.qkv) + t * a.ld + (int64_t)h * a.D;
        const T *gamma = static_cast<const T *>(is_q ? a.q_gamma : is_k ? a.k_gamma : nullptr);
        T *p;
        if (is_q) p = static_cast<T *>(a.q) + t * a.q_ts + h * a.q_hs;
        else {
            if (pl.at < 0) continue;
            p = static_cast<T *>(is_k ? a.k : a.v) + pl.at + (is_k ? h - a.Hq : h - a.Hq - a.Hkv) * a.c_hs;
        }
        if (is_q && pl.pos < 0) {
            for (int i = lane; i < a.D; i += 32) p[i] = from_f32<T>(0.f);
            continue;
        }
        float r = 1.f;
        if (gamma) {
            float sum = 0.f;
            for (int i = lane; i < a.D; i += 32) { const float u = to_f32<T>(x[i]); sum = fmaf(u, u, sum); }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            r = rsqrtf(fmaf(sum, a.inv_d, a.eps));
        }
        auto at = [&](int i) { return gamma ? to_f32<T>(x[i]) * (r * to_f32<T>(gamma[i])) : to_f32<T>(x[i]); };
        const int turned = rot && (is_q || is_k) ? half : 0;
        for (int i = lane; i < turned; i += 32) {
            const int i0 = a.interleaved ? 2 * i : i, i1 = a.interleaved ? 2 * i + 1 : i + half;
            const float u = at(i0), w = at(i1), c = rot[i], s = rot[half + i];
            p[i0] = from_f32<T>(u * c - w * s);
            p[i1] = from_f32<T>(w * c + u * s);
        }
        for (int i = 2 * turned + lane; i < a.D; i += 32) p[i] = from_f32<T>(at(i));
    }
}

template <typename K, typename... A> int launch(K kern, dim3 grid, void *stream, const HeadArgs &a, A... more)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(128);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, a, more...);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { set_last_cuda_error((int)e); return UBP_E_CUDA; }
    return UBP_OK;
}

// kind: 2 = 16-byte accesses, 1 = rows of qkv element by element, 0 = single elements
template <typename T> int launch_heads(const HeadArgs &a, int kind, void *stream)
{
    const int H = a.Hq + 2 * a.Hkv, sms = device_sms();
    if (kind == 0) {
        const int64_t want = std::max<int64_t>(1, (int64_t)8 * sms / a.T);
        return launch(ubp_heads_any_kernel<T>, dim3((unsigned)a.T, (unsigned)std::min<int64_t>((H + 3) / 4, want)), stream, a);
    }
    auto by = [&](auto tph, auto inter) {
        constexpr int P = decltype(tph)::value;
        constexpr bool I = decltype(inter)::value;
        const int heads = 128 / P;              // a block's side by side
        // Few tokens: a head a group of threads, a block for every `heads` of them (one token of 48 heads 2.3 us, 3.1 with three heads a
        // group). Many: all of a token's heads in one block, consecutive tokens, as many blocks as the SMs hold.
        if ((int64_t)a.T * ((H + heads - 1) / heads) <= 8 * sms) {
            const dim3 g((unsigned)a.T, (unsigned)((H + heads - 1) / heads));
            return kind == 2 ? launch(ubp_heads_kernel<T, P, I, false, 1>, g, stream, a, 1) : launch(ubp_heads_kernel<T, P, I, true, 1>, g, stream, a, 1);
        }
        const int per = (a.T + HEADS_BLOCKS * sms - 1) / (HEADS_BLOCKS * sms);
        const dim3 g((unsigned)((a.T + per - 1) / per));
        return kind == 2 ? launch(ubp_heads_kernel<T, P, I, false, 3>, g, stream, a, per) : launch(ubp_heads_kernel<T, P, I, true, 2>, g, stream, a, per);
    };
    auto by_size = [&](auto inter) { return a.D <= 64 ? by(std::integral_constant<int, 4>{}, inter) : by(std::integral_constant<int, 8>{}, inter); };
    return a.interleaved ? by_size(std::true_type{}) : by_size(std::false_type{});
}

bool on(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace
}  // namespace ubp

extern "C" int ubp_rotate_append(const ubp_cache_t *cache, const void *qkv, int64_t ld, int64_t T, int q_heads, const void *q_gamma,
                                 const void *k_gamma, float eps, const float *rotation, int64_t rotation_stride, int64_t positions, int rotated,
                                 int interleaved, void *q, int64_t q_token_stride, int64_t q_head_stride, void *stream)
{
    using namespace ubp;
    if (const int rc = check_cache(cache, T, q_heads)) return rc;
    const int D = cache->head_dim;
    if (rotation && (rotated < 2 || rotated % 2 || rotated > D || positions < 1 || (positions > 1 && rotation_stride < rotated))) return UBP_E_ARG;
    if (!(eps >= 0.f)) return UBP_E_ARG;
    if (T == 0 || cache->batch == 0) return UBP_OK;
    if (!qkv || !q || !on(qkv, 2) || !on(q, 2) || !on(q_gamma, 2) || !on(k_gamma, 2) || !on(rotation, 4)) return UBP_E_ARG;
    const int64_t width = (int64_t)(q_heads + 2 * (int64_t)cache->kv_heads) * D;
    if (width > INT32_MAX) return UBP_E_UNSUPPORTED;
    if ((T > 1 && (ld < width || q_token_stride < D)) || (q_heads > 1 && q_head_stride < D)) return UBP_E_ARG;
    // (blocks read rows that others may have written already: the queries' own place in qkv, where a head is read and written by the same
    // threads, or a place apart)
    const HeadPlaces to(q, q_token_stride, q_head_stride, q_heads, D);
    const bool own = q == qkv && (T == 1 || q_token_stride == ld) && (q_heads == 1 || q_head_stride == D);
    if (places_repeat(to, T) || (!own && places_meet(to, HeadPlaces(qkv, ld, 0, 1, width), T))) return UBP_E_ARG;
    HeadArgs a{};
    a.qkv = qkv; a.ld = ld; a.q_gamma = q_gamma; a.k_gamma = k_gamma; a.eps = eps;
    a.rot = rotation; a.ldrot = rotation_stride; a.positions = (int)std::min<int64_t>(positions, INT32_MAX); a.r = rotation ? rotated : 0;
    a.interleaved = interleaved != 0;
    a.q = q; a.q_ts = q_token_stride; a.q_hs = q_head_stride;
    a.k = cache->k; a.v = cache->v;
    a.c_ps = cache->page_stride; a.c_hs = cache->head_stride; a.c_ts = cache->token_stride;
    a.table = cache->table; a.lengths = cache->lengths; a.starts = cache->starts; a.ldt = cache->table_stride;
    a.pages = (int)cache->pages;
    while ((1 << a.pshift) < cache->page_size) ++a.pshift;
    a.cap = (int)std::min<int64_t>((int64_t)cache->table_width << a.pshift, INT32_MAX);
    a.T = (int)T; a.B = (int)cache->batch; a.Hq = q_heads; a.Hkv = cache->kv_heads; a.D = D;
    a.inv_d = 1.f / (float)D;
    const bool pieces = D % 16 == 0 && a.r % 16 == 0 && on(q, 16) && (T == 1 || q_token_stride % 8 == 0) && (q_heads == 1 || q_head_stride % 8 == 0) &&
                        on(q_gamma, 16) && on(k_gamma, 16) && (!rotation || (on(rotation, 16) && (positions == 1 || rotation_stride % 4 == 0)));
    // (queries over their own place in unaligned rows would be such rows' neighbours' too early: they are off 16 bytes then, kind 0)
    const int kind = !pieces ? 0 : on(qkv, 16) && (T == 1 || ld % 8 == 0) ? 2 : 1;
    return cache->dtype == UBP_BF16 ? launch_heads<__nv_bfloat16>(a, kind, stream) : launch_heads<__half>(a, kind, stream);
}
