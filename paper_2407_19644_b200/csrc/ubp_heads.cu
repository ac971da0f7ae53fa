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
#include <cuda_runtime.h>

#include <algorithm>

#include "ubp_attention.h"
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
__device__ __forceinline__ Place place_of(const HeadArgs &a, int b, int t)
{
    Place p{-1, -1};
    int s = t, n = 1;
    if (a.starts) {
        s = imin(imax(a.starts[b], 0), a.T);
        n = imin(imax(a.starts[b + 1], s), a.T) - s;
    }
    const int pos = imax(a.lengths[b], 0) - n + (t - s);
    if (pos < 0 || (a.rot && pos >= a.positions)) return p;
    p.pos = pos;
    if (pos < a.cap) {
        const int page = a.table[b * a.ldt + (pos >> a.pshift)];
        if ((uint32_t)page < (uint32_t)a.pages) p.at = page * a.c_ps + (pos & ((1 << a.pshift) - 1)) * a.c_ts;
    }
    return p;
}

// TPH: threads a head (a power of two, D / 16 of them at work)
template <typename T, int TPH, bool INTER>
__global__ void __launch_bounds__(128) ubp_heads_kernel(const HeadArgs a)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int GROUPS = 128 / TPH;
    const int t = (int)blockIdx.x, b = seq_of(a, t);
    if (b < 0) return;
    const Place pl = place_of(a, b, t);
    const int part = threadIdx.x % TPH, rp = a.r / 16;
    const bool live = part < a.D / 16, rotated = a.rot && part < rp;
    // the thread's two pieces of a head
    const int c0 = 8 * (INTER || part >= rp ? 2 * part : part), c1 = INTER || part >= rp ? c0 + 8 : c0 + 8 * rp;
    float cs[8], sn[8];
    if (rotated && pl.pos >= 0) {
        const float *p = a.rot + pl.pos * a.ldrot + 8 * part;
        load8(p, cs);
        load8(p + a.r / 2, sn);
    }
    const T *row = static_cast<const T *>(a.qkv) + t * a.ld;
    const int H = a.Hq + 2 * a.Hkv;
    for (int h = (int)blockIdx.y * GROUPS + threadIdx.x / TPH; h < (H + GROUPS - 1) / GROUPS * GROUPS; h += (int)gridDim.y * GROUPS) {
        const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv, on = live && h < H;
        float x[8], y[8];
        if (on) { load8(row + (int64_t)h * a.D + c0, x); load8(row + (int64_t)h * a.D + c1, y); }
        const T *gamma = static_cast<const T *>(is_q ? a.q_gamma : is_k ? a.k_gamma : nullptr);
        float sum = 0.f;
        if (on && gamma) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], fmaf(y[i], y[i], sum));
        }
#pragma unroll
        for (int o = TPH / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (!on) continue;
        if (gamma) {
            const float r = rsqrtf(sum / (float)a.D + a.eps);
            float g[8];
            load8(gamma + c0, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= r * g[i];
            load8(gamma + c1, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= r * g[i];
        }
        if (rotated && pl.pos >= 0 && (is_q || is_k)) {
            if constexpr (INTER) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float u = x[2 * i], w = y[2 * i];
                    x[2 * i] = u * cs[i] - x[2 * i + 1] * sn[i];
                    x[2 * i + 1] = x[2 * i + 1] * cs[i] + u * sn[i];
                    y[2 * i] = w * cs[4 + i] - y[2 * i + 1] * sn[4 + i];
                    y[2 * i + 1] = y[2 * i + 1] * cs[4 + i] + w * sn[4 + i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = x[i];
                    x[i] = u * cs[i] - y[i] * sn[i];
                    y[i] = y[i] * cs[i] + u * sn[i];
                }
            }
        }
        T *p;
        if (is_q) {
            p = static_cast<T *>(a.q) + t * a.q_ts + h * a.q_hs;
            if (pl.pos < 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = y[i] = 0.f;
            }
        } else {
            if (pl.at < 0) continue;
            p = static_cast<T *>(is_k ? a.k : a.v) + pl.at + (is_k ? h - a.Hq : h - a.Hq - a.Hkv) * a.c_hs;
        }
        store8<T>(p + c0, x);
        store8<T>(p + c1, y);
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
    const Place pl = place_of(a, b, t);
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
            r = rsqrtf(sum / (float)a.D + a.eps);
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

template <typename K> int launch(K kern, dim3 grid, const HeadArgs &a, void *stream)
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
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, a);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { set_last_cuda_error((int)e); return UBP_E_CUDA; }
    return UBP_OK;
}

template <typename T> int launch_heads(const HeadArgs &a, bool vec, void *stream)
{
    const int H = a.Hq + 2 * a.Hkv, sms = device_sms();
    // One head a group of threads while the call has few tokens, so that one token's heads are under way together; all of a
    // token's heads in one block otherwise, whose threads then load its rotation once.
    auto grid = [&](int groups) {
        const int64_t most = (H + groups - 1) / groups, want = std::max<int64_t>(1, (int64_t)8 * sms / a.T);
        return dim3((unsigned)a.T, (unsigned)std::min(most, want));
    };
    if (!vec) return launch(ubp_heads_any_kernel<T>, grid(4), a, stream);
    if (a.D <= 64) return a.interleaved ? launch(ubp_heads_kernel<T, 4, true>, grid(32), a, stream) : launch(ubp_heads_kernel<T, 4, false>, grid(32), a, stream);
    return a.interleaved ? launch(ubp_heads_kernel<T, 8, true>, grid(16), a, stream) : launch(ubp_heads_kernel<T, 8, false>, grid(16), a, stream);
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
    const bool vec = D % 16 == 0 && a.r % 16 == 0 && on(qkv, 16) && (T == 1 || ld % 8 == 0) && on(q, 16) && (T == 1 || q_token_stride % 8 == 0) &&
                     (q_heads == 1 || q_head_stride % 8 == 0) && on(q_gamma, 16) && on(k_gamma, 16) &&
                     (!rotation || (on(rotation, 16) && (positions == 1 || rotation_stride % 4 == 0)));
    return cache->dtype == UBP_BF16 ? launch_heads<__nv_bfloat16>(a, vec, stream) : launch_heads<__half>(a, vec, stream);
}
