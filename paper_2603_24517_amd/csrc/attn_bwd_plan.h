// How the work of a call of attn_bwd() is cut into items and dealt to workgroups: plain integer arithmetic on sizes, for the host that plans and the
// kernels that look their items up, without HIP's headers, so that it can be compiled and checked on its own.
#ifndef PAPER_2603_24517_ATTN_BWD_PLAN_H
#define PAPER_2603_24517_ATTN_BWD_PLAN_H

#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/attn.h"

#ifdef __HIP__
#define BWD_FN __host__ __device__ inline __attribute__((always_inline))
#else
#define BWD_FN inline
#endif

namespace attn_bwd_plan {
namespace {        // (nothing of it is exported by the library)

constexpr int HD = 128;
constexpr int ROW_BYTES = HD * 2;
constexpr int BT = 32;                          // streamed rows per step
constexpr int ITEM_ROWS = 128;                  // held rows of an item, 32 per wavefront
constexpr size_t PART_BYTES = 32 * HD * sizeof(float);     // what one wavefront leaves of one sum

// n / d for n < 2^31 with constants found on the host
struct Div { uint32_t mul, shift; };
inline Div make_div(uint32_t d)
{
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    return {(uint32_t)(((1ull << 32) * ((1ull << l) - d)) / d + 1), l};
}
BWD_FN int fast_div(int n, Div d) { return (int)(((uint32_t)((uint64_t)(uint32_t)n * d.mul >> 32) + (uint32_t)n) >> d.shift); }

// The items of one kind.  A tile's steps (streamed tiles, of all heads of a group) are cut into pieces of at most `most`, so that a call of few or
// uneven tiles fills the chip; a tile of several pieces leaves FP32 parts, which attn_bwd_join adds up.
struct Role {
    int groups, tiles, splits;      // grid: groups x tiles x splits (the largest number of pieces)
    int most;
    int items, per_xcd;             // of all XCDs and of one (of all, where they do not keep to their own groups)
    int window, per_window;         // groups whose tiles are dealt out together, and their items
    int last, rest;                 // the last window (of an XCD's), which may be longer, and its groups
    Div d_window, d_per_tile, d_per_window, d_rest, d_per_rest_tile;
};
struct Sizes {
    int B, Hq, Hkv, Sq, Skv, G, qtiles;
    int pack_log2, chunks;          // rows items: query heads of a group side by side, and how many such chunks a group has
    int off;                        // key j valid for row i iff j <= i + off (without the mask: always true)
    Role keys, rows;
    int xcd_groups;                 // 0, or the K/V heads (of all batch entries) that each XCD keeps to
    bool together;                  // behind each window's keys items come its rows items; otherwise all rows items come last
    Div d_both;                     // items of a window, of both kinds
    Div d_hkv, d_chunks, d_g;
    int join_keys;                  // workgroups of attn_bwd_join for dk and dv
};

// Query tiles in front of a tile's first key (keys items); steps of a tile.
BWD_FN int keys_skip(const Sizes &p, int tile)
{
    const int first = tile * ITEM_ROWS - p.off;             // first row that sees the tile's first key
    return first > 0 ? (first / BT < p.qtiles ? first / BT : p.qtiles) : 0;
}
BWD_FN int keys_steps(const Sizes &p, int tile) { return (p.qtiles - keys_skip(p, tile)) * p.G; }
BWD_FN int rows_steps(const Sizes &p, int tile)
{
    const int end = (tile + 1) * (ITEM_ROWS >> p.pack_log2);
    const int last = (end < p.Sq ? end : p.Sq) - 1 + p.off;      // last key that the tile's last row sees
    return last < 0 ? 0 : (last < p.Skv - 1 ? last : p.Skv - 1) / BT + 1;
}
BWD_FN int pieces(int steps, int most) { return steps <= most ? 1 : (steps + most - 1) / most; }
// Steps [first, first + count) of a tile's that piece `piece` of `n_pieces` takes.
BWD_FN void piece_steps(int steps, int n_pieces, int piece, int &first, int &count)
{
    first = (int)((unsigned)steps * (unsigned)piece / (unsigned)n_pieces);
    count = (int)((unsigned)steps * (unsigned)(piece + 1) / (unsigned)n_pieces) - first;
}

// Batch entry, head and first of the 32 rows that a wavefront of an item holds.
BWD_FN void find_rows(const Sizes &p, bool keys, int group, int tile, int wave, int &b, int &head, int &x0)
{
    const int bh = keys ? group : fast_div(group, p.d_chunks);
    b = fast_div(bh, p.d_hkv);
    head = bh - b * p.Hkv;
    x0 = tile * ITEM_ROWS + wave * 32;
    if (!keys) {
        head = head * p.G + ((group - bh * p.chunks) << p.pack_log2) + (wave & ((1 << p.pack_log2) - 1));
        x0 = tile * (ITEM_ROWS >> p.pack_log2) + (wave >> p.pack_log2) * 32;
    }
}

// Which item of a kind has number n in its order (together: in that of window w): window by window, longest tiles first.
BWD_FN void find_item(const Role &r, bool together, int n, int w, int first, int &group, int &tile, int &piece)
{
    if (!together) {
        w = fast_div(n, r.d_per_window);
        w = w < r.last ? w : r.last;
        n -= w * r.per_window;
    }
    const bool last = w == r.last;
    const int window = last ? r.rest : r.window;
    tile = fast_div(n, last ? r.d_per_rest_tile : r.d_per_tile);
    n -= tile * window * r.splits;
    piece = fast_div(n, last ? r.d_rest : r.d_window);
    group = first + w * r.window + n - piece * window;
}

// The item of workgroup n.  The hardware deals workgroups round-robin to the 8 XCDs, each with an L2 of its own; where the groups (batch entries x K/V heads)
// divide among them, an XCD keeps to its own groups, a window of them at a time, so that the tiles of a group, which stream the same data, meet in one L2.
struct Item {
    bool keys;
    int group, tile, piece;
};
BWD_FN Item which_item(const Sizes &p, int n)
{
    int first = 0, w = 0, of_keys = p.keys.per_xcd;
    if (p.xcd_groups) {
        first = (n & 7) * p.xcd_groups;
        n >>= 3;
        if (p.together) {
            w = fast_div(n, p.d_both);
            w = w < p.keys.last ? w : p.keys.last;
            n -= w * (p.keys.per_window + p.rows.per_window);
            of_keys = w == p.keys.last ? p.keys.rest * p.keys.tiles * p.keys.splits : p.keys.per_window;
        }
    }
    Item item;
    item.keys = n < of_keys;
    if (item.keys) {
        find_item(p.keys, p.together, n, w, first, item.group, item.tile, item.piece);
    } else {
        find_item(p.rows, p.together, n - of_keys, w, first * p.chunks, item.group, item.tile, item.piece);
        item.tile = p.rows.tiles - 1 - item.tile;
    }
    return item;
}

// ----------------------------------------------------------------------------------------------------------- host
struct Plan {
    Sizes p;                                    // sizes and roles
    size_t stats, part_kv, part_q, total;       // bytes: the workspace's three parts
};

inline int check_sizes(int B, int Hq, int Hkv, int Sq, int Skv, int D)
{
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Skv <= 0 || D <= 0) return ATTN_E_SHAPE;
    if (Hq % Hkv != 0) return ATTN_E_SHAPE;
    if (D != HD) return ATTN_E_UNSUPPORTED;
    if ((long long)Sq + Skv >= (1ll << 31) - 1024 || Hq > 32768 || Hkv > 32768) return ATTN_E_UNSUPPORTED;
    return ATTN_OK;
}

// Workgroups that are resident at a time on the device that this is written for, two per compute unit: how items are cut (and so what the
// workspace needs) does not ask the device.
constexpr int CUS = 256, PLACES = 2 * CUS;
// Microseconds: a step alone on a compute unit, and how much longer it takes beside another; an item beside its steps; how much of the last items
// stands out behind a full chip; the launch and the bytes per microsecond of adding up parts.  Fitted to 100 calls of this range, each cut in
// up to 90 ways: the choice is 2.1 % off the best of those on average, 18 % at most.
constexpr double KEYS_STEP = 0.75, ROWS_STEP = 0.69, SHARED = 1.38, ITEM = 3.8, LAST = 0.7, JOIN = 4.6, JOIN_BYTES = 7.9e6;
constexpr int MOST_PIECES = 32;
constexpr double CACHE_BYTES = 192e6;      // three quarters of the memory-side cache

// The order of the items.  Windows are as many groups as an XCD's 64 places take, or up to half as many again where windows of that size are equal; otherwise they
// are of one size but for the last, which takes what is left over as well: a last window that is shorter instead ends with one long tile to a place
// (13 x 4096, 8 heads, masked: 1425 us, one window for all 1376, this 1368).  One window for all, which is what a count without divisors
// came to before / these windows, us: 131 x 500, 8 heads 702 / 586; 53 x 1000, 16 heads 1649 / 1487; 13 x 4096, 32 on 8, masked 5550 / 5269; 11 x 4096,
// 8 heads 2126 / 2115; of 20 calls with such counts all are faster, 6.0 % on average.
inline int fit_window(int groups, int per_group)
{
    const int wanted = (PLACES / 8 + per_group - 1) / per_group, windows = groups / wanted;
    if (windows < 2) return groups;
    for (int window = wanted; 2 * window <= 3 * wanted; ++window)
        if (groups % window == 0) return window;
    return groups / windows;
}
inline void deal(Sizes &p)
{
    const int groups = p.keys.groups, both = p.keys.tiles * p.keys.splits + p.chunks * p.rows.tiles * p.rows.splits;
    p.xcd_groups = groups % 8 == 0 ? groups / 8 : 0;
    // Keys and rows items read the same inputs.  Side by side they find them in L2, which pays where a few tiles to a group leave the rest of the
    // traffic to memory and the cache behind the L2s does not hold the inputs, unless an item is so long that it must not start late: more than a
    // quarter of a place's work.  Together / apart, inputs from memory, us: 96 x 300, 16 heads, masked 338 / 382; 210 x 198, 8 heads, masked 227 / 257;
    // 27 x 642, 24 heads 564 / 583; 34 x 840, 32 on 8 heads 1354 / 1432; longer items 4 x 2401, 32 on 4, masked 865 / 727; smaller inputs 512 x 64, 4 heads,
    // masked 90 / 86.  40 drawn calls that are dealt together: 5.9 % faster on average, 0.5 to 11.5 %.
    p.together = false;
    if (p.xcd_groups && both < PLACES / 8 && 2.0 * ROW_BYTES * ((double)p.G * p.Sq + p.Skv) * groups > CACHE_BYTES) {
        double all = 0;
        int longest = 0;
        for (int t = 0; t < p.keys.tiles; ++t) {
            const int n = keys_steps(p, t);
            all += n;
            longest = n > longest ? n : longest;
        }
        for (int t = 0; t < p.rows.tiles; ++t) {
            const int n = rows_steps(p, t);
            all += (double)n * p.chunks;
            longest = n > longest ? n : longest;
        }
        p.together = 4.0 * longest * PLACES <= all * groups;
    }
    for (Role *r : {&p.keys, &p.rows}) {
        const int heads = r == &p.keys ? 1 : p.chunks, per_group = r->tiles * r->splits;
        r->items = r->groups * per_group;
        r->per_xcd = p.xcd_groups ? r->items / 8 : r->items;
        r->window = r->groups;
        if (p.together)
            r->window = fit_window(p.xcd_groups, both) * heads;
        else if (p.xcd_groups)      // all groups of an XCD at once, longest tiles first, while that is few rounds
            r->window = r->per_xcd <= 4 * PLACES / 8 ? p.xcd_groups * heads : fit_window(p.xcd_groups * heads, per_group);
        r->per_window = r->window * per_group;
        const int of_xcd = p.xcd_groups ? p.xcd_groups * heads : r->groups;
        r->last = of_xcd / r->window - 1;
        r->rest = of_xcd - r->last * r->window;
        r->d_window = make_div(r->window);
        r->d_per_tile = make_div(r->window * r->splits);
        r->d_rest = make_div(r->rest);
        r->d_per_rest_tile = make_div(r->rest * r->splits);
        r->d_per_window = make_div(r->per_window);
    }
    p.d_both = make_div(p.keys.per_window + p.rows.per_window);
}

inline int make_plan(int B, int Hq, int Hkv, int Sq, int Skv, int causal, Plan &r)
{
    Sizes &p = r.p;
    const int G = Hq / Hkv;
    p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.Sq = Sq; p.Skv = Skv; p.G = G;
    p.pack_log2 = G % 4 == 0 ? 2 : G % 2 == 0 ? 1 : 0;
    p.chunks = G >> p.pack_log2;
    p.qtiles = (Sq + BT - 1) / BT;
    // (i + INT32_MAX - Sq - 256 is above every key for i >= 0 and within 32 bits for the i < Sq + 256 of a tile)
    p.off = causal ? Skv - Sq : INT32_MAX - Sq - 256;
    const int pos = ITEM_ROWS >> p.pack_log2;
    const int tk = (Skv + ITEM_ROWS - 1) / ITEM_ROWS, tr = (Sq + pos - 1) / pos;
    // A rows item holds rows of 4 heads at most: 2^25 heads or more are 2^23 items or more, and below that no product here leaves 64 bits.
    if ((long long)B * Hq >= (1ll << 25)) return ATTN_E_UNSUPPORTED;
    const long long nk = (long long)B * Hkv * tk, nr = (long long)B * Hkv * p.chunks * tr;
    // (A launch has fewer than 2^32 threads.  Fewer than 2^23 rows items also bound the rows with figures, 32 of a head in line, to less than 2^30, four
    // threads each, and the steps of a keys tile to less than 2^25)
    if (nk >= (1ll << 23) || nr >= (1ll << 23)) return ATTN_E_UNSUPPORTED;
    p.d_hkv = make_div(Hkv);
    p.d_chunks = make_div(p.chunks);
    p.d_g = make_div(G);
    p.keys = {B * Hkv, tk, 1, INT32_MAX};
    p.rows = {B * Hkv * p.chunks, tr, 1, INT32_MAX};

    // Calls of few tiles for the chip, or of uneven ones, are cut: the pair of piece lengths whose estimate is the shortest.
    const int long_k = keys_steps(p, 0), long_r = rows_steps(p, tr - 1), short_r = rows_steps(p, 0);
    if (nk + nr < 4 * PLACES) {
        double all_k = 0, all_r = 0;
        for (int t = 0; t < tk; ++t) all_k += keys_steps(p, t);
        for (int t = 0; t < tr; ++t) all_r += rows_steps(p, t);
        all_k *= p.keys.groups;
        all_r *= p.rows.groups;
        const double kv_bytes = 2.0 * B * Skv * Hkv * HD * 4, q_bytes = (double)B * Sq * Hq * HD * 4;
        double best = INFINITY;
        int best_k = 1, best_r = 1;
        for (int sk = 1; sk <= MOST_PIECES; sk += sk < 8 ? 1 : sk / 4) {
            const int mk = (long_k + sk - 1) / sk;
            if (sk > 1 && mk < 3) break;
            for (int sr = 1; sr <= MOST_PIECES; sr += sr < 8 ? 1 : sr / 4) {
                const int mr = (long_r + sr - 1) / sr;
                if (sr > 1 && mr < 4) break;
                const double pk = sk > 1 ? all_k / mk : nk, pr = sr > 1 ? all_r / mr : nr, n = pk + pr;       // pieces, about
                const double more = n <= CUS ? 0 : n >= PLACES ? 1 : (n - CUS) / (PLACES - CUS), slow = 1 + (SHARED - 1) * more;
                const double k = slow * KEYS_STEP, q = slow * ROWS_STEP, ik = ITEM + k * mk, ir = ITEM + q * mr;
                double us = (all_k * k + all_r * q + n * ITEM) / PLACES;
                if (n > PLACES) us += LAST * (ITEM + q * (sr > 1 ? mr : short_r));
                if (us < ik) us = ik;
                if (us < ir) us = ir;
                if (sk > 1 || sr > 1) us += JOIN + 2 * ((sk > 1 ? sk * kv_bytes : 0) + (sr > 1 ? sr * q_bytes : 0)) / JOIN_BYTES;
                if (us < best) {
                    best = us;
                    best_k = sk;
                    best_r = sr;
                }
            }
        }
        if (best_k > 1) {
            p.keys.most = (long_k + best_k - 1) / best_k;
            p.keys.splits = pieces(long_k, p.keys.most);
        }
        if (best_r > 1) {
            p.rows.most = (long_r + best_r - 1) / best_r;
            p.rows.splits = pieces(long_r, p.rows.most);
        }
    }
    deal(p);
    auto pad = [](size_t n) { return (n + 255) / 256 * 256; };
    r.stats = pad((size_t)B * Hq * p.qtiles * 2 * BT * sizeof(float));
    p.join_keys = p.keys.splits > 1 ? (int)nk * 8 : 0;
    r.part_kv = p.keys.splits > 1 ? (size_t)p.keys.items * 8 * PART_BYTES : 0;
    r.part_q = p.rows.splits > 1 ? (size_t)p.rows.items * 4 * PART_BYTES : 0;
    r.total = r.stats + r.part_kv + r.part_q;
    return ATTN_OK;
}

}  // namespace
}  // namespace attn_bwd_plan

#undef BWD_FN
#endif
