// Attention over a paged cache: what its kernels share -- arguments, the tiles a row block has to visit, and how the steps of a
// call are dealt to the blocks of a grid.
//
// Rows. The query heads that share a key head are rows of one product, together with neighbouring tokens: row r of a row block is
// token r / gc, head r % gc of a group of gc query heads ("unit head"; a group is the Hq / Hkv heads of a key head, cut into
// pieces of at most the row block's rows). An item is (sequence, unit head, row block); its steps are the tiles of keys that some
// of its rows see, at least one (an item whose rows see nothing still writes its zeros).
//
// Steps. All items of a call lie one behind the other -- sequence by sequence, unit head by unit head, row block by row block --
// and block c of G takes the c-th share of their steps: every block gets the same number to within one whatever the lengths are,
// which only the device knows. An item that ends up with several blocks is joined by a second kernel from their partial results.
// An item counts for `extra` steps more than its tiles: what its beginning and end take. Without them, blocks that got many short
// items (the first rows of a prompt, short sequences of a batch) took twice as long as the others. (With the heads inside the row
// blocks, a long prompt of eight key heads took 1.58 times as long, in an early form of the kernel: the blocks at work then read
// eight times as many different keys at a time.) For few sequences and short work a cluster of blocks takes all of an item instead;
// items of few tiles are left whole.
#ifndef UBP_ATTENTION_H_
#define UBP_ATTENTION_H_

#include <cuda_runtime.h>

#include <climits>
#include <cstddef>
#include <cstdint>

#include "ubp.h"

#define UBP_HD __host__ __device__ __forceinline__

namespace ubp {

struct AttnArgs {
    const void *q;
    int64_t q_ts, q_hs;             // strides of q between tokens and heads (elements; rows on 16 bytes)
    void *out;
    int64_t o_ts, o_hs;
    const void *k, *v;
    int64_t c_ps, c_hs, c_ts;       // strides of the cache between pages, heads and tokens
    const int32_t *table;
    int64_t ldt;
    const int32_t *lengths;
    const int32_t *starts;          // null: one new token a sequence
    int pages, pshift, cap;         // cap: tokens a table row holds
    int T, B, Hq, Hkv, G, D;
    int rows;                       // rows of a row block, and tokens (rows / gc) of each of its `tiles` tiles
    int tiles;                      // row tiles of a row block (each rows / tiles rows)
    int gc, chunks, HU;             // heads of a unit head, unit heads of a key head, unit heads in all
    int tpt;                        // tokens a row block takes
    int bsh;                        // keys a step takes: 1 << bsh
    int extra;                      // steps that an item counts for beside its tiles
    int whole;                      // 1: items are not cut; a block takes those that begin in its share
    float sc;                       // scale * log2(e)
    int window, sinks;
    int kv0, kv1;                   // keys outside [kv0, kv1) are left out (a shared prefix is a call of its own)
    int shared;                     // keys below it lie in the pages of table row 0 (boxes of a copy that lie below it as a whole)
    int common;                     // 1: the rows are all tokens of all sequences, the pages those of table row 0
    // partial results: rows x {reference maximum, sum} and rows x D of a slot
    float2 *ml;
    float *po;
    int *status;                    // of the device: 1 once a bounded wait has run out
    int4 *desc;                     // [grid] the item that begins in a block and does not end there (AttnPart)
    // the shared prefix's results of each row, [T][Hq] and [T][Hq][D] (null without one): written by its join, read by the others
    float2 *pml;
    float *ppo;
};

UBP_HD int imin(int a, int b) { return a < b ? a : b; }
UBP_HD int imax(int a, int b) { return a > b ? a : b; }

// new tokens of sequence b: [s, s + n) of the call's; len tokens in all (numbers that make no sense are cut to what does)
struct AttnSeq { int s, n, len; };
UBP_HD AttnSeq attn_seq(const AttnArgs &a, int b)
{
    AttnSeq q;
    if (a.common) {
        q.s = 0;
        q.n = a.starts ? imin(imax(a.starts[a.B], 0), a.T) : a.T;
        q.len = a.kv1;
        return q;
    }
    if (a.starts) {
        q.s = imin(imax(a.starts[b], 0), a.T);
        q.n = imin(imax(a.starts[b + 1], q.s), a.T) - q.s;
    } else {
        q.s = b; q.n = 1;
    }
    q.len = imin(imax(a.lengths[b], 0), a.cap);
    return q;
}

// The tiles of keys that a row block with positions p0 .. p1 visits: ns from s0 on (first tokens), the rest from lo on.
// Keys below w0 are seen by none of the rows unless they are among the first `sinks`, keys from `end` on by none.
struct AttnTiles { int s0, ns, lo, nt, w0, end; };
UBP_HD AttnTiles attn_tiles(const AttnArgs &a, int p0, int p1)
{
    AttnTiles t;
    const int up = (1 << a.bsh) - 1;
    t.end = imin(p1 + 1, a.kv1);
    t.w0 = a.window > 0 && !a.common ? imax(a.kv0, imax(p0, 0) - a.window + 1) : a.kv0;
    t.s0 = a.kv0 >> a.bsh;
    t.lo = t.w0 >> a.bsh;
    t.ns = 0;
    if (t.end <= a.kv0) { t.end = a.kv0; t.lo = t.s0; t.nt = 1; return t; }
    if (t.lo > t.s0 && a.sinks > a.kv0) t.ns = imin(((imin(a.sinks, t.end) + up) >> a.bsh) - t.s0, t.lo - t.s0);
    t.nt = imax(1, t.ns + imax(0, ((t.end + up) >> a.bsh) - t.lo));
    return t;
}
UBP_HD int attn_tile_at(const AttnTiles &t, int i) { return i < t.ns ? t.s0 + i : t.lo + i - t.ns; }

UBP_HD int attn_row_blocks(const AttnArgs &a, const AttnSeq &q) { return (q.n + a.tpt - 1) / a.tpt; }
UBP_HD AttnTiles attn_block_tiles(const AttnArgs &a, const AttnSeq &q, int rt)
{
    if (a.common) return attn_tiles(a, 0, a.kv1 - 1);
    const int first = q.len - q.n + rt * a.tpt, last = q.len - q.n + imin(q.n, (rt + 1) * a.tpt) - 1;
    return attn_tiles(a, first, last);
}

// Where a block is in its steps: an item, and the next of its tiles.
struct AttnCursor {
    int b, hu, rt, tile;
    AttnSeq q;
    AttnTiles t;
    UBP_HD void set(const AttnArgs &a, int b_, int hu_, int rt_, int tile_)
    {
        b = b_; hu = hu_; rt = rt_; tile = tile_;
        q = attn_seq(a, b);
        t = attn_block_tiles(a, q, rt);
    }
    UBP_HD void next_item(const AttnArgs &a)        // (only while steps are left: there is a next item)
    {
        tile = 0;
        if (q.n <= a.tpt && hu + 1 < a.HU) { ++hu; return; }           // (the same rows of other heads: the same tiles)
        if (++rt * a.tpt >= q.n) {
            rt = 0;
            if (++hu == a.HU) {
                hu = 0;
                do q = attn_seq(a, ++b); while (q.n == 0);
            }
        }
        t = attn_block_tiles(a, q, rt);
    }
};

// The steps of a block that are left: a cursor at the next tile, and how many steps its share still holds (extras included; if
// items are not cut, all tiles of the last item that begins in it).
struct AttnSteps {
    AttnCursor c;
    int left;
    UBP_HD void seek(const AttnArgs &a)             // a share may begin in an item's extras
    {
        if (left > 0 && (c.tile >= c.t.nt || (a.whole && c.tile > 0))) skip(a);
        else if (a.whole) left = imax(left, left > 0 ? c.t.nt : 0);
    }
    UBP_HD void skip(const AttnArgs &a)             // the rest of the item's steps
    {
        left -= c.t.nt + a.extra - c.tile;
        if (left <= 0) return;
        c.next_item(a);
        if (a.whole) left = imax(left, c.t.nt);
    }
    UBP_HD int tiles() const { return imin(c.t.nt - c.tile, left); }      // of the item, in this share
    UBP_HD void advance(const AttnArgs &a, int n)   // past n tiles
    {
        c.tile += n;
        left -= n;
        if (left > 0 && c.tile == c.t.nt) skip(a);
    }
};

// How `total` steps are dealt to `grid` blocks (grid <= total): the first r blocks take q + 1, the others q.
struct AttnDeal {
    int64_t q;
    int r, grid;
    UBP_HD AttnDeal() : q(0), r(0), grid(0) {}
    UBP_HD AttnDeal(int64_t total, int blocks)
    {
        grid = total < (int64_t)blocks ? (int)total : blocks;
        if (total >> 32) { q = total / grid; r = (int)(total - q * grid); }
        else if (grid) { q = (uint32_t)total / (uint32_t)grid; r = (int)((uint32_t)total - (uint32_t)q * (uint32_t)grid); }
        else { q = 0; r = 0; }
    }
    UBP_HD int64_t first(int c) const { return q * c + imin(c, r); }
    UBP_HD int count(int c) const { return (int)q + (c < r ? 1 : 0); }      // (the launch refuses calls of more)
    UBP_HD int owner(int64_t x) const       // block that has step x
    {
        const int64_t y = x - (q + 1) * r;
        return y < 0 ? (int)(x / (q + 1)) : r + (int)(y / q);
    }
};

// slots of partial results that a call needs, and its workspace: [desc][ml][po]
struct AttnSpace { size_t ml, po, total; };
inline AttnSpace attn_space(int64_t grid, int64_t slots, int rows, int D)
{
    AttnSpace s;
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    s.ml = up((size_t)grid * sizeof(int4));
    s.po = s.ml + up((size_t)slots * rows * sizeof(float2));
    s.total = s.po + up((size_t)slots * rows * D * sizeof(float));
    return s;
}

// ---- places of operands. Heads of T tokens: n pieces of w 16-bit elements a token, hs apart, tokens ts apart (a stride that is never
// used may be anything).
struct HeadPlaces {
    const void *p;
    int64_t ts, hs, n, w;
    HeadPlaces(const void *p_, int64_t ts_, int64_t hs_, int64_t n_, int64_t w_) : p(p_), ts(ts_), hs(hs_), n(n_), w(w_)
    {
        if (hs == w) { w *= n; n = 1; }
    }
    int64_t end(int64_t T) const { return (T > 1 ? (T - 1) * ts : 0) + (n > 1 ? (n - 1) * hs : 0) + w; }
};
// whether pieces of w and v elements, the first x behind the second, meet for some two of T tokens
inline bool pieces_meet(int64_t x, int64_t w, int64_t v, int64_t ts, int64_t T)
{
    if (T == 1) return x > -w && x < v;
    const int64_t y = -w - x;                                      // the first i with x + i ts > -w, of -(T - 1) .. T - 1
    int64_t i = (y >= 0 ? y / ts : -((-y + ts - 1) / ts)) + 1;
    if (i < 1 - T) i = 1 - T;
    return i < T && x + i * ts < v;
}
// Whether an element of a is one of b, of any two tokens. Where they lie among one another with different strides between tokens, that
// counts as if it were so.
inline bool places_meet(const HeadPlaces &a, const HeadPlaces &b, int64_t T)
{
    const int64_t d = (static_cast<const char *>(a.p) - static_cast<const char *>(b.p)) / 2;
    if (d >= b.end(T) || -d >= a.end(T)) return false;
    if (T > 1 && a.ts != b.ts) return true;
    for (int64_t h = 0; h < a.n; ++h)
        for (int64_t g = 0; g < b.n; ++g)
            if (pieces_meet(d + h * a.hs - g * b.hs, a.w, b.w, a.ts, T)) return true;
    return false;
}
// whether heads of different tokens share elements
inline bool places_repeat(const HeadPlaces &a, int64_t T)
{
    if (T == 1) return false;
    if (a.n == 1) return a.ts < a.w;
    if (a.ts >= (a.n - 1) * a.hs + a.w || a.hs >= (T - 1) * a.ts + a.w) return false;
    for (int64_t h = 1; h < a.n; ++h)
        if (pieces_meet(h * a.hs, a.w, a.w, a.ts, T)) return true;
    return false;
}

// ---- launches; both kernels follow the same scheme and leave the same partial results
int launch_attn_few(const AttnArgs &a, int dtype, int grid, void *stream);       // 16 rows an item (ubp_attention_few.cu)
int launch_attn_cluster(const AttnArgs &a, int dtype, int size, void *stream);    // the same, a cluster of blocks a sequence and unit head
int launch_attn_tc(const AttnArgs &a, int dtype, int grid, void *stream);        // 256 rows an item (ubp_attention_tc.cu)
int launch_attn_copy_queries(const void *q, int64_t ts, int64_t hs, int64_t T, int Hq, int D, void *to, void *stream);      // -> [T][Hq][D]
int launch_attn_join(const AttnArgs &a, int dtype, int grid, void *stream);       // `grid`: the kernel's before it
int device_sms();
void set_last_cuda_error(int e);

}  // namespace ubp
#endif
