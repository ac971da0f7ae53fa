// C entry points of the attention operators: argument checks, choice of kernel and grid, workspace.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "ubp_attention.h"
#include "ubp_types.cuh"

namespace ubp {
__device__ int attn_status_word;         // 1: a bounded wait ran out

namespace {

// its address on the current device (found once a device)
int status_word(int **p)
{
    static std::atomic<int *> known[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev < 64 && (*p = known[dev])) return UBP_OK;
    void *q = nullptr;
    if (e == cudaSuccess) e = cudaGetSymbolAddress(&q, attn_status_word);
    if (e != cudaSuccess) { set_last_cuda_error((int)e); return UBP_E_CUDA; }
    *p = static_cast<int *>(q);
    if (dev < 64) known[dev] = *p;
    return UBP_OK;
}

bool on(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int log2_of(int n) { int s = 0; while ((1 << s) < n) ++s; return s; }

}  // namespace

// What every call on a cache asks of it. B sequences; T new tokens.
int check_cache(const ubp_cache_t *c, int64_t T, int q_heads)
{
    if (!c) return UBP_E_ARG;
    if (c->dtype != UBP_BF16 && c->dtype != UBP_F16) return UBP_E_ARG;
    if (c->batch < 0 || T < 0 || c->kv_heads < 1 || q_heads < 1 || c->head_dim < 1) return UBP_E_ARG;
    if (c->page_size < 1 || c->pages < 1 || c->table_width < 1) return UBP_E_ARG;
    if (q_heads % c->kv_heads) return UBP_E_ARG;
    if (!c->starts && c->batch != T) return UBP_E_ARG;
    if (c->head_dim % 8 || c->head_dim > 128 || c->page_size < 8 || (c->page_size & (c->page_size - 1))) return UBP_E_UNSUPPORTED;
    // (the kernels count tokens and sequences in 32 bits, up to a block's or a warp's share past the last one)
    constexpr int64_t most = INT32_MAX - 4096;
    if (T > most || c->batch > most || c->pages > INT32_MAX) return UBP_E_UNSUPPORTED;
    if (T == 0 || c->batch == 0) return UBP_OK;
    if (!c->k || !c->v || !c->table || !c->lengths) return UBP_E_ARG;
    if (!on(c->k, 16) || !on(c->v, 16) || !on(c->table, 4) || !on(c->lengths, 4) || !on(c->starts, 4)) return UBP_E_ARG;
    const int D = c->head_dim;
    if (c->page_stride % 8 || c->head_stride % 8 || c->token_stride % 8) return UBP_E_ARG;
    if (c->token_stride < D || (c->kv_heads > 1 && c->head_stride < D) || (c->pages > 1 && c->page_stride < D)) return UBP_E_ARG;
    if (c->batch > 1 && c->table_stride < c->table_width) return UBP_E_ARG;
    return UBP_OK;
}

namespace {

// Rows of an item and how the heads of a group are dealt to them.
void set_rows(AttnArgs &a, int rows, int tiles)
{
    const int per = rows / tiles;
    a.bsh = tiles == 1 && a.D <= 64 ? 8 : 7;
    a.rows = rows; a.tiles = tiles;
    a.chunks = (a.G + per - 1) / per;
    a.gc = (a.G + a.chunks - 1) / a.chunks;
    a.HU = a.Hq / a.G * a.chunks;
    a.tpt = per / a.gc * tiles;
    a.extra = tiles == 2 ? 2 : 3;
}

// Bytes of a shared prefix that are read again for the other sequences (mostly from L2) in the time that a call of its own for the
// prefix and the join of its sums take. bf16, read again / a call of its own, us: 8 MB 17.0 / 21.8, 25 MB 11.7 / 24.3, 57 MB 18.0 /
// 27.5, 66 MB 24.9 / 28.3, 123 MB 27.8 / 28.4, 131 MB 32.9 / 27.7, 197 MB 41.0 / 29.8, 254 MB 46.8 / 33.4, 516 MB 84 / 45.
constexpr double ATTN_PREFIX_BYTES = 120e6;
// Clusters of blocks of 16 rows: as many blocks as run at once (15 clusters of eight; 16 of them took 11.5 us instead of 6.3), and
// tiles a block, by the longest that the table or the window allows. One token on 8 key heads of 128 values, cluster / steps dealt,
// us: 500 keys 7.0 / 8.6, 2000 8.1 / 10.5, 4000 10.3 / 11.6, 8000 (eight tiles a block) 15.1 / 14.2; four sequences of 500 7.2 / 9.9, of
// 4000 (eight tiles) 16.9 / 16.8; twelve of 500 (one block each) 9.8 / 12.9; 100 of 700 keys on one head of 64 values 7.9 / 11.9.
constexpr int64_t ATTN_CLUSTER_BLOCKS = 120, ATTN_CLUSTER_TILES = 6;

// Items of at most this many tiles (of 256 rows, of 16 rows), by the longest that the table or the window allows, are not cut: the most
// that a block then has to do more than the others is one item, and cuts cost about as much (segments' ends, partial results, the
// join). Left whole / cut, us, 32 heads on 8 of 128 values unless said: 256 rows: 7 prompts of 1 .. 901 on 12 / 4 heads, window 300
// (7 tiles) 27.7 / 37.7, one of 512 (6) 17.5 / 23.1, one of 16384 with a window of 512 (8) 239 / 282, 4096 with 1024 (12) 100.6 / 100.1,
// 1400 (13) 36.7 / 42.4, 20 of 100 on up to 1600 (14) 65.7 / 75.6, 8 of them 43.8 / 43.1, 2000 and 1500 on 16 / 4 heads (17) 54.0 /
// 51.1, 8192 (66) 562 / 511. 16 rows: 64 tokens on up to 400 keys (5) 24.1 / 25.8, 17 on 500 (6) 10.3 / 13.9, 32 with a window of 512 (8)
// 22.2 / 24.6, 64 on 900 (9) 37.3 / 36.8, 32 on 1500 (13) 34.1 / 26.3.
constexpr int64_t ATTN_WHOLE_TILES = 14, ATTN_WHOLE_FEW = 8;

// A call's kernels, grids and the layout of its workspace; the same for the size query and the call.
struct AttnCall {
    AttnArgs own, common;
    bool own_tc = false, common_tc = false;
    int cluster = 0;                    // blocks of a cluster that share a sequence and unit head; 0: steps are dealt
    bool has_common = false;
    int own_grid = 0, common_grid = 0;
    AttnSpace own_space{}, common_space{}, row_space{};
    size_t q_bytes = 0, bytes = 0;      // queries off 16 bytes are copied first
};

int attn_plan(const ubp_cache_t *c, const void *q, int64_t q_ts, int64_t q_hs, int64_t T, int q_heads, float scale, int window, int sinks,
              int64_t prefix, int64_t max_new, AttnCall &p)
{
    const int sms = device_sms();
    AttnArgs a{};
    a.T = (int)T; a.B = (int)c->batch; a.Hq = q_heads; a.Hkv = c->kv_heads; a.G = q_heads / c->kv_heads; a.D = c->head_dim;
    a.k = c->k; a.v = c->v;
    a.c_ps = c->page_stride; a.c_hs = c->head_stride; a.c_ts = c->token_stride;
    a.table = c->table; a.ldt = c->batch > 1 ? c->table_stride : 0;
    a.lengths = c->lengths; a.starts = c->starts;
    a.pages = (int)c->pages; a.pshift = log2_of(c->page_size);
    a.cap = (int)std::min<int64_t>((int64_t)c->table_width << a.pshift, INT32_MAX - 4096);
    a.sc = scale * 1.44269504088896340736f;
    a.window = window; a.sinks = window > 0 ? sinks : 0;
    a.kv0 = (int)prefix; a.kv1 = INT32_MAX;
    p.own_tc = std::min<int64_t>(max_new, T) * a.G > 16;
    if (p.own_tc) set_rows(a, 256, 2);
    else set_rows(a, 16, 1);
    // more blocks than steps would have nothing to do
    const int64_t seen = window > 0 ? std::min<int64_t>(a.cap, (int64_t)window + sinks + a.tpt + (2 << a.bsh)) : a.cap;
    const int64_t items = (a.T / a.tpt + (int64_t)a.B) * a.HU;
    const int64_t tiles = (seen >> a.bsh) + 2 + a.extra;
    // (the kernels count the steps of a unit head, and a block's, in 32 bits)
    if (items / a.HU > INT32_MAX / tiles || ((a.cap >> a.bsh) + 2) > INT32_MAX / a.HU || items * tiles / sms >= INT32_MAX)
        return UBP_E_UNSUPPORTED;
    p.own_grid = (int)std::min<int64_t>(sms, items * tiles);
    if (!on(q, 16) || (T > 1 && q_ts % 8) || (q_heads > 1 && q_hs % 8)) p.q_bytes = ((size_t)T * q_heads * a.D * 2 + 255) / 256 * 256;
    p.bytes = p.q_bytes;
    // A shared prefix is read for all sequences at once only where reading it again for each -- what a window leaves of it -- takes
    // longer than that saves.
    const double each = window > 0 ? std::min<double>((double)prefix, (double)window + sinks) : (double)prefix;
    const bool again = prefix > 0 && (a.B * each - (double)prefix) * a.Hkv * a.D * 4.0 < ATTN_PREFIX_BYTES;
    if (again) { a.kv0 = 0; a.shared = (int)prefix; }
    // Few sequences and short work: a cluster of up to eight blocks for each sequence and unit head.
    if (!p.own_tc && (prefix == 0 || again)) {
        const int64_t units = (int64_t)a.B * a.HU, reach = (seen >> a.bsh) + 2;
        int size = 8;
        while (size > 1 && units * size > ATTN_CLUSTER_BLOCKS) size /= 2;
        if (units * size <= ATTN_CLUSTER_BLOCKS && reach <= (int64_t)ATTN_CLUSTER_TILES * size) p.cluster = size;
    }
    const int64_t reach = ((prefix > 0 && !again ? std::min(seen, a.cap - prefix) : seen) >> a.bsh) + 2;
    const bool whole = reach <= (p.own_tc ? ATTN_WHOLE_TILES : ATTN_WHOLE_FEW);
    if (!p.cluster && !whole) {
        p.own_space = attn_space(p.own_grid, 2 * (int64_t)p.own_grid, a.rows, a.D);
        p.bytes += p.own_space.total;
    }
    if (prefix > 0 && !again) {
        AttnArgs b = a;
        b.common = 1;
        b.kv0 = 0; b.kv1 = (int)prefix;
        p.common_tc = T * b.G > 16;
        if (p.common_tc) set_rows(b, 256, 2);
        else set_rows(b, 16, 1);
        const int64_t units = (int64_t)((b.T + b.tpt - 1) / b.tpt) * b.HU;
        const int nt = (int)((prefix + (1 << b.bsh) - 1) >> b.bsh) + b.extra;
        p.common_grid = (int)std::min<int64_t>(sms, units * nt);
        if (units + p.common_grid > INT32_MAX || units / b.HU > INT32_MAX / nt || units * nt / sms >= INT32_MAX) return UBP_E_UNSUPPORTED;
        p.common_space = attn_space(0, units + p.common_grid, b.rows, b.D);
        p.row_space = attn_space(0, T, q_heads, b.D);          // a row's sums over the prefix
        p.bytes += p.common_space.total + p.row_space.total;
        p.common = b;
    }
    p.has_common = prefix > 0 && !again;
    p.own = a;
    p.own.whole = whole;
    return UBP_OK;
}

int check_attention(const ubp_cache_t *c, int64_t T, int q_heads, float scale, int window, int sinks, int64_t prefix, int64_t max_new)
{
    if (const int rc = check_cache(c, T, q_heads)) return rc;
    if (!(scale > 0.f) || !std::isfinite(scale) || window < 0 || sinks < 0 || max_new < 1) return UBP_E_ARG;
    if (prefix < 0 || prefix > (int64_t)c->table_width * c->page_size) return UBP_E_ARG;
    if (prefix > INT32_MAX - 4096) return UBP_E_UNSUPPORTED;
    return UBP_OK;
}

}  // namespace
}  // namespace ubp

extern "C" size_t ubp_attention_workspace_size(const ubp_cache_t *cache, const void *q, int64_t q_token_stride, int64_t q_head_stride, int64_t T,
                                               int q_heads, int window, int sinks, int64_t prefix, int64_t max_new)
{
    if (ubp::check_attention(cache, T, q_heads, 1.f, window, sinks, prefix, max_new) || T == 0 || cache->batch == 0) return 0;
    ubp::AttnCall p;
    return ubp::attn_plan(cache, q, q_token_stride, q_head_stride, T, q_heads, 1.f, window, sinks, prefix, max_new, p) ? 0 : p.bytes;
}

extern "C" int ubp_attention_choice(const ubp_cache_t *cache, int64_t T, int q_heads, int64_t prefix, int64_t max_new, int *kernel,
                                    int *prefix_kernel)
{
    using namespace ubp;
    if (const int rc = check_attention(cache, T, q_heads, 1.f, 0, 0, prefix, max_new)) return rc;
    if (!kernel || !prefix_kernel) return UBP_E_ARG;
    AttnCall p;
    if (T == 0 || cache->batch == 0) { *kernel = 0; *prefix_kernel = -1; return UBP_OK; }
    if (const int rc = attn_plan(cache, nullptr, 0, 0, T, q_heads, 1.f, 0, 0, prefix, max_new, p)) return rc;
    *kernel = p.own_tc ? 1 : p.cluster ? 2 : 0;
    *prefix_kernel = p.has_common ? (int)p.common_tc : -1;
    return UBP_OK;
}

extern "C" int ubp_attention(const ubp_cache_t *cache, const void *q, int64_t q_token_stride, int64_t q_head_stride, int64_t T, int q_heads,
                             float scale, int window, int sinks, int64_t prefix, int64_t max_new, void *out, int64_t out_token_stride,
                             int64_t out_head_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace ubp;
    if (const int rc = check_attention(cache, T, q_heads, scale, window, sinks, prefix, max_new)) return rc;
    if (T == 0 || cache->batch == 0) return UBP_OK;
    if (!q || !out || !on(q, 2) || !on(out, 2)) return UBP_E_ARG;
    const int D = cache->head_dim;
    if ((q_heads > 1 && (q_head_stride < D || out_head_stride < D)) || (T > 1 && (q_token_stride < D || out_token_stride < D))) return UBP_E_ARG;
    // (blocks read whole groups' queries, of other tokens and heads than they have written)
    const HeadPlaces to(out, out_token_stride, out_head_stride, q_heads, D);
    if (places_repeat(to, T) || places_meet(to, HeadPlaces(q, q_token_stride, q_head_stride, q_heads, D), T)) return UBP_E_ARG;
    AttnCall p;
    if (const int rc = attn_plan(cache, q, q_token_stride, q_head_stride, T, q_heads, scale, window, sinks, prefix, max_new, p)) return rc;
    if (p.bytes && (!workspace || !on(workspace, 256))) return UBP_E_ARG;
    if (workspace_bytes < p.bytes) return UBP_E_SPACE;
    int *status = nullptr;
    if (const int rc = status_word(&status)) return rc;
    uint8_t *w = static_cast<uint8_t *>(workspace);
    auto finish = [&](AttnArgs &a, const AttnSpace &s) {
        a.status = status;
        a.q = q; a.q_ts = q_token_stride; a.q_hs = q_head_stride;
        a.out = out; a.o_ts = out_token_stride; a.o_hs = out_head_stride;
        a.desc = reinterpret_cast<int4 *>(w);
        a.ml = reinterpret_cast<float2 *>(w + s.ml);
        a.po = reinterpret_cast<float *>(w + s.po);
        w += s.total;
    };
    if (p.q_bytes) {
        if (const int rc = launch_attn_copy_queries(q, q_token_stride, q_head_stride, T, q_heads, D, w, stream)) return rc;
        q = w;
        q_head_stride = D;
        q_token_stride = (int64_t)q_heads * D;
    }
    w += p.q_bytes;
    finish(p.own, p.own_space);
    if (p.cluster) return launch_attn_cluster(p.own, cache->dtype, p.cluster, stream);
    if (p.has_common) {
        finish(p.common, p.common_space);
        p.own.pml = p.common.pml = reinterpret_cast<float2 *>(w + p.row_space.ml);
        p.own.ppo = p.common.ppo = reinterpret_cast<float *>(w + p.row_space.po);
        if (const int rc = (p.common_tc ? launch_attn_tc : launch_attn_few)(p.common, cache->dtype, p.common_grid, stream)) return rc;
        if (const int rc = launch_attn_join(p.common, cache->dtype, p.common_grid, stream)) return rc;
    }
    if (const int rc = (p.own_tc ? launch_attn_tc : launch_attn_few)(p.own, cache->dtype, p.own_grid, stream)) return rc;
    return p.own.whole ? UBP_OK : launch_attn_join(p.own, cache->dtype, p.own_grid, stream);
}

extern "C" int ubp_attention_check(void *stream)
{
    int v = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(&v, ubp::attn_status_word, sizeof v, 0, cudaMemcpyDeviceToHost, static_cast<cudaStream_t>(stream));
    if (e == cudaSuccess) e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) { ubp::set_last_cuda_error((int)e); return UBP_E_CUDA; }
    return v ? UBP_E_DEVICE : UBP_OK;
}

extern "C" int ubp_attention_clear_status(void *stream)
{
    const int v = 0;
    cudaError_t e = cudaMemcpyToSymbolAsync(ubp::attn_status_word, &v, sizeof v, 0, cudaMemcpyHostToDevice, static_cast<cudaStream_t>(stream));
    if (e == cudaSuccess) e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) { ubp::set_last_cuda_error((int)e); return UBP_E_CUDA; }
    return UBP_OK;
}
