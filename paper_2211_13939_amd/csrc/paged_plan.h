// What an attention call to a paged cache becomes: which requests share a launch, which kernel takes them, what is read apart and in which parts.  Host code, no HIP calls.
#pragma once
#include <algorithm>
#include <cmath>
#include <utility>

#include "past_kernels.h"

namespace tts {

constexpr int PAGED_MAX_TILES = 1 << 23;             // of a call: a grid has fewer than 2^32 threads, and XCDs' shares of the tiles may be of different heights
constexpr int PAGED_MAX_SPLITS = 256;                // parts of one sequence
// Requests of so many rows and more are a kernel's for many rows, if their call has two and a half tiles of 16 for every compute unit (the lines of cross attention, where they were measured)
constexpr int PAGED_MANY_ROWS = 33;
inline bool paged_many(long long few_tiles, int n_cu) { return 2 * few_tiles >= 5LL * n_cu; }

// Room for parts, in parts of 16 rows: more than a launch is split into, and enough for a tile of each of its requests and key heads beside their prefixes'.
inline int paged_room(int n_kv_heads) { return 4096 + PAGED_BATCH * n_kv_heads; }

// How requests of few rows, gathered, are cut into tiles of 16 rows and parts of their keys.
enum class PagedPools { NONE, TILES, APART };        // prefixes: ahead of their requests' own rows; tiles of theirs in the same launch; a launch of their own behind this
struct PagedCut {
    PagedPools pools;
    int share;                           // length of a part, 0: whole sequences
    double ns;                           // what it should take
};
// A workgroup's way from its launch to its first keys and from the last ones to its results (3.2 us measured, with one step); a step of its waves: the matrix pipe's (two waves a SIMD take turns), or its
// keys' and values' way, by latency: 45 GB/s to a workgroup of four waves from the last-level cache, 28 from memory, 70 and 43 to one of eight.
struct PagedCosts {
    int keys, held;                      // of a wave's step; workgroups of four waves that a compute unit holds
    double step[2];                      // ns, of workgroups of four waves and of eight
};
constexpr double PAGED_START = 3500;
inline PagedCosts paged_costs(int d, int element_bytes, bool far)
{
    const int keys = element_bytes == 2 ? 32 : 16, held = d == 64 ? 4 : element_bytes == 2 ? 3 : 2;
    const double pipe = element_bytes == 2 ? 2.5 * d + 80 : 6.8 * d, bytes = 8.0 * keys * d * element_bytes;
    return {keys, held, {std::max({700.0, pipe, bytes / (far ? 28 : 45)}), std::max({700.0, 2 * pipe, 2 * bytes / (far ? 43 : 70)})}};
}
constexpr int PAGED_JOIN_PARTS = 40;                 // that a row's last one joins; of more a kernel of its own does

// Entities of a launch: tiles (of all key heads) over a sequence each.
struct PagedTiles {
    int n = 0;
    int tiles[PAGED_BATCH + PAGED_POOLS], len[PAGED_BATCH + PAGED_POOLS];
    void add(int rows, int kv, int length)
    {
        tiles[n] = (rows + 15) / 16 * kv;
        len[n++] = length;
    }
};
inline PagedTiles paged_tiles(const PagedArgs& a, PagedPools pools)
{
    PagedTiles t;
    for (int i = 0; i < a.n; ++i) {
        const int g = prefix_of(a.req[i]);
        t.add(a.row[i + 1] - a.row[i], a.n_kv_heads, own_len_of(a.req[i]) + (pools == PagedPools::NONE && g >= 0 ? up16(a.pool[g].len) : 0));
    }
    if (pools == PagedPools::TILES)
        for (int g = 0; g < a.n_pools; ++g) t.add(a.row[a.pool[g].end] - a.row[a.pool[g].begin], a.n_kv_heads, a.pool[g].len);
    return t;
}

// The cheapest cut with prefixes so.  `unique`: bytes that have to come from memory at least.
inline PagedCut paged_cut(const PagedArgs& a, PagedPools pools, int element_bytes, int n_cu, double unique, int room)
{
    const int d = paged_width(a.head_dim);
    const PagedCosts c = paged_costs(d, element_bytes, unique > 128e6);
    const PagedTiles t = paged_tiles(a, pools);
    PagedCut best{pools, 0, 1e30};
    int longest = 0;
    double keys = 0;
    for (int i = 0; i < t.n; ++i) {
        longest = std::max(longest, t.len[i]);
        keys += (double)t.tiles[i] * t.len[i];
    }
    int whole = 64;
    while (whole < longest) whole *= 2;
    for (int log = log2_of(whole); log >= 6; --log) {
        long long items = 0;
        for (int i = 0; i < t.n; ++i) items += (long long)t.tiles[i] * (((std::max(t.len[i], 1) - 1) >> log) + 1);
        const int parts = std::max(1, (longest + (1 << log) - 1) >> log);
        const bool eight = items <= n_cu;
        if ((parts > 1 || pools != PagedPools::NONE) && items > room) break;
        if (parts > PAGED_MAX_SPLITS) break;
        const double at_once = (double)n_cu * (eight ? 1 : c.held), per = (eight ? 8 : 4) * c.keys, step = c.step[eight];
        // what bounds it, of which none hides another altogether: the longest part; all of them, one behind the other; memory's rate and the L2s'
        const double bounds[4] = {PAGED_START + std::ceil(std::min(longest, 1 << log) / per) * step, items > at_once ? (items * (PAGED_START + 0.5 * step) + keys / per * step) / at_once : 0,
                                  unique / 4800 + 2500, 2.0 * keys * a.head_dim * element_bytes / 9000 + 2500};
        double ns = 0;
        for (double x : bounds) ns += x * x * x;
        ns = std::cbrt(ns);
        const int meet = parts + (pools == PagedPools::TILES);
        if (meet > 1) ns += meet <= PAGED_JOIN_PARTS ? 2500 + 100 * meet : 6000;
        if (ns < best.ns) best = PagedCut{pools, parts > 1 ? 1 << log : 0, ns};
        if (items > 2 * at_once && parts > 1) break;
    }
    return best;
}
// The longest sequence's parts of one length, where that makes no more of them for others.
inline void even_parts(const PagedArgs& a, PagedCut& cut)
{
    if (!cut.share) return;
    const PagedTiles t = paged_tiles(a, cut.pools);
    int longest = 0;
    for (int i = 0; i < t.n; ++i) longest = std::max(longest, t.len[i]);
    const int parts = (longest - 1) / cut.share + 1, even = ((longest + parts - 1) / parts + 31) / 32 * 32;
    if (even == cut.share) return;
    long long items = 0, evenly = 0;
    for (int i = 0; i < t.n; ++i) {
        items += (long long)t.tiles[i] * paged_parts(t.len[i], cut.share);
        evenly += (long long)t.tiles[i] * paged_parts(t.len[i], even);
    }
    if (evenly <= items) cut.share = even;
}

// Numbers of a launch's tiles; pools: of prefixes of their own in it.
inline void plan_paged_few(PagedArgs& a, const PagedCut& cut)
{
    a.pooled = cut.pools != PagedPools::NONE && a.n_pools;
    a.share = a.pool_share = cut.share;
    a.height = a.pool_height = PAGED_FEW_ROWS;
    const bool pools = a.pooled && cut.pools == PagedPools::TILES;
    long long items = 0;
    int most = 1;
    a.per = 0;
    for (int i = 0; i < a.n; ++i) {
        a.req[i].first = (int)items;
        const int parts = paged_parts(paged_len(a, a.req[i]), cut.share), mine = (a.row[i + 1] - a.row[i] + 15) / 16 * a.n_kv_heads * parts;
        a.per = i == 0 || a.per == mine ? mine : 0;
        most = std::max(most, parts);
        items += mine;
    }
    a.pool_first = (int)items;
    if (pools)
        for (int g = 0; g < a.n_pools; ++g) {
            const int parts = paged_parts(a.pool[g].len, cut.share);
            a.pool[g].first = (int)items;
            most = std::max(most, parts + 1);
            items += (long long)((a.row[a.pool[g].end] - a.row[a.pool[g].begin] + 15) / 16) * a.n_kv_heads * parts;
        }
    a.items = (int)items;
    if (a.per > 4096) a.per = 0;         // (128 requests' tiles times those of one: less than 2^32)
    a.by_per = by_of(a.per);
    a.join = (pools || (!a.pooled && most > 1)) && most <= PAGED_JOIN_PARTS;
    a.subs = most <= 4 ? 1 : 4;
    a.pool_parts = a.parts + (size_t)a.pool_first * paged_part_floats(16, paged_width(a.head_dim));
}

// Shares of the XCDs: tiles in runs of equal work.  `entry(i, tiles, each)` gives the i-th entry's tiles and one's work.
template <typename Entry> int plan_runs(PagedArgs& a, int first, int n, Entry entry)
{
    double work = 0, done = 0;
    for (int i = 0; i < n; ++i) {
        const auto [tiles, each] = entry(i);
        work += (double)tiles * each;
    }
    int x = 1, at = first;
    a.start[0] = first;
    for (int i = 0; i < n; ++i) {
        const auto [tiles, each] = entry(i);
        for (; x < 8 && done + (double)tiles * each >= work * x / 8; ++x)
            a.start[x] = std::min(at + tiles, std::max(a.start[x - 1], at + (int)((work * x / 8 - done) / each + 0.5)));
        at += tiles;
        done += (double)tiles * each;
    }
    for (; x <= 8; ++x) a.start[x] = at;
    return at;
}

// The split of a launch's sequences into parts of one length: shortest that `most` workgroups go through at once.  0: none.
template <typename Items> int paged_share(double keys, long long tiles, int longest, int most, Items items)
{
    if (2 * tiles > most) return 0;
    double share = std::max({keys / (most - 0.5 * tiles), (double)longest / PAGED_MAX_SPLITS, 128.0});
    auto whole = [](double s) { return ((int)std::ceil(s) + 63) / 64 * 64; };      // (tiles of 64 keys, steps of 32)
    while (share < longest && items(whole(share)) > most) share *= 1.0625;
    if (share >= longest) return 0;
    const int parts = (longest - 1) / whole(share) + 1, even = whole((longest - 1) / parts + 1);
    return items(even) <= most ? even : whole(share);
}

// Prefixes' tiles of many rows, in a launch of their own behind that of the requests' own rows.
inline int pool_rows(const PagedArgs& a, int g) { return a.row[a.pool[g].end] - a.row[a.pool[g].begin]; }
// Their height, 0: no room for the parts.
inline int paged_pool_height(const PagedArgs& a, int n_cu)
{
    int most = 0;
    for (int g = 0; g < a.n_pools; ++g) most = std::max(most, pool_rows(a, g));
    const int height = most > 64 ? 128 : 64;
    long long tiles = 0, own = 0;
    for (int g = 0; g < a.n_pools; ++g) tiles += (pool_rows(a, g) + height - 1) / height * a.n_kv_heads;
    for (int i = 0; i < a.n; ++i) own += (a.row[i + 1] - a.row[i] + 15) / 16 * a.n_kv_heads;
    return tiles * height <= (paged_room(a.n_kv_heads) - std::max<long long>(own, 8 * n_cu)) * PAGED_FEW_ROWS ? height : 0;
}
// What they should take, with the kernel that joins their rows: a tile's 64 keys 1.2 us of a compute unit (0.85 with heads of 64), its part's way out with them (512 rows of 8 heads over
// 16001 keys, in 16 parts, 48 us), then some ten parts of every row.
inline double paged_pools_ns(const PagedArgs& a, int height, int n_cu)
{
    double work = 0;
    for (int g = 0; g < a.n_pools; ++g) work += (double)((pool_rows(a, g) + height - 1) / height) * a.n_kv_heads * (a.pool[g].len / 64 + 1);
    return 9000 + work * (a.head_dim > 64 ? 1200 : 850) / n_cu + 5000 + (double)a.rows * a.n_kv_heads * 10 * 520 / 3500;
}
inline void plan_paged_pools(PagedArgs& a, int height, int n_cu)
{
    const int d = paged_width(a.head_dim);
    auto tiles_of = [&](int g) { return (pool_rows(a, g) + height - 1) / height * a.n_kv_heads; };
    double keys = 0;
    long long tiles = 0;
    int longest = 0;
    for (int g = 0; g < a.n_pools; ++g) {
        keys += (double)tiles_of(g) * a.pool[g].len;
        tiles += tiles_of(g);
        longest = std::max(longest, a.pool[g].len);
    }
    const long long room = ((long long)paged_room(a.n_kv_heads) - a.pool_first) * PAGED_FEW_ROWS / height;
    auto cut = [&](int share) {
        long long items = 0;
        for (int g = 0; g < a.n_pools; ++g) {
            a.pool[g].first = a.pool_first + (int)items;
            items += (long long)tiles_of(g) * paged_parts(a.pool[g].len, share);
        }
        return items;
    };
    a.pool_height = height;
    a.pool_share = paged_share(keys, tiles, longest, (int)std::min<long long>(room, (d == 128 ? 2 : 3) * n_cu), cut);
    a.items = a.pool_first + (int)cut(a.pool_share);
    a.pool_parts = a.parts + (size_t)a.pool_first * paged_part_floats(PAGED_FEW_ROWS, d);
    plan_runs(a, a.pool_first, a.n_pools, [&](int g) { return std::pair<int, double>(tiles_of(g) * paged_parts(a.pool[g].len, a.pool_share), a.pool_share ? a.pool_share : a.pool[g].len); });
}

// Requests of many rows, gathered, in tiles of 128 over whole sequences or parts of them: a tile's 64 keys by themselves and with the compute unit full (one request of 512 and of 1024 rows,
// 32 heads of 128 that share 8, 17.4 and 28.1 us; of 2048 behind 4096 187).  Tiles of 64, where requests have no more rows, are no faster (32 requests of 40 rows over 700 to 2400
// 46.6 us, in tiles of 128 42.1; 64 of 64 over 300 22.1 / 22.4), nor are such of 256 (4 of 512 over 1024 40.7 / 42.6, 2 of 4096 289 / 294, one of 512 over 2560 72 / 56).
constexpr int PAGED_MANY_HEIGHT = 128;
struct PagedManyCosts { double start, alone, full; };
constexpr PagedManyCosts paged_many_costs(int d) { return d == 128 ? PagedManyCosts{6500, 1250, 970} : PagedManyCosts{5500, 900, 690}; }
inline double paged_keys(const PagedArgs& a, int i)      // that a tile of the i-th request takes on average
{
    const int q = (a.row[i + 1] - a.row[i]) / (a.n_heads / a.n_kv_heads);
    return paged_len(a, a.req[i]) - (a.causal ? std::min(q, own_len_of(a.req[i])) / 2 : 0);
}
// One request of 128 rows over 4224 keys takes 86 us whole and 29.7 in 8 parts, one of 512 over 2560 56 and 49.6 in two.
inline PagedCut paged_many_cut(const PagedArgs& a, int n_cu, double unique)
{
    constexpr int height = PAGED_MANY_HEIGHT;
    const int d = paged_width(a.head_dim);
    const PagedManyCosts c = paged_many_costs(d);
    const long long room = (long long)paged_room(a.n_kv_heads) * PAGED_FEW_ROWS / height;
    const double held = d == 128 ? 2 : 3;
    int longest = 0;
    double work = 0;                     // tiles' 64 keys
    for (int i = 0; i < a.n; ++i) {
        longest = std::max(longest, paged_len(a, a.req[i]));
        work += (double)((a.row[i + 1] - a.row[i] + height - 1) / height) * a.n_kv_heads * (paged_keys(a, i) / 64 + 1);
    }
    PagedCut best{PagedPools::NONE, 0, 1e30};
    for (int parts = 1; parts <= 64; parts += std::max(1, parts / 4)) {
        const int share = parts == 1 ? 0 : ((longest + parts - 1) / parts + 63) / 64 * 64;
        if (parts > 1 && share < 128) break;
        long long items = 0;
        for (int i = 0; i < a.n; ++i) items += (long long)((a.row[i + 1] - a.row[i] + height - 1) / height) * a.n_kv_heads * paged_parts(paged_len(a, a.req[i]), share);
        if (parts > 1 && items > room) break;
        const double one = std::min<double>(items, n_cu * held) > n_cu ? std::max(c.alone, 2 * c.full) : c.alone;
        const double bounds[3] = {c.start + ((share ? share : longest) + 63) / 64 * one, items > n_cu ? (work * c.full + items * c.start / held) / n_cu : 0, unique / 4800 + 2500};
        double ns = 0;
        for (double x : bounds) ns += x * x * x;
        ns = std::cbrt(ns);
        if (parts > 1) ns += 5000 + (double)a.rows * a.n_kv_heads * parts * 4 * (d + 2) * 2 / 3500;
        if (ns < best.ns) best = PagedCut{PagedPools::NONE, share, ns};
    }
    return best;
}
inline void plan_paged_many(PagedArgs& a, const PagedCut& cut)
{
    constexpr int height = PAGED_MANY_HEIGHT;
    constexpr int OWN = 160;             // a tile's own cost, in keys (measured for cross attention)
    auto tiles_of = [&](int i) { return (a.row[i + 1] - a.row[i] + height - 1) / height * a.n_kv_heads * paged_parts(paged_len(a, a.req[i]), a.share); };
    a.pooled = false;
    a.share = a.pool_share = cut.share;
    a.per = 0;
    a.join = false;
    a.height = a.pool_height = height;
    int at = 0;
    for (int i = 0; i < a.n; ++i) {
        a.req[i].first = at;
        at += tiles_of(i);
    }
    a.items = a.pool_first = at;
    plan_runs(a, 0, a.n, [&](int i) { return std::pair<int, double>(tiles_of(i), OWN + paged_keys(a, i) / paged_parts(paged_len(a, a.req[i]), a.share)); });
}

}  // namespace tts
