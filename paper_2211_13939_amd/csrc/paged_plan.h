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

// Requests of few rows, gathered: tiles and parts.  n_cu: compute units; pools: whether prefixes' tiles are of 16 rows, too, in the same launch.
inline void plan_paged_few(PagedArgs& a, int element_bytes, int n_cu, bool pools)
{
    const int d = paged_width(a.head_dim);
    auto tiles_of = [](int rows) { return (long long)(rows + 15) / 16; };
    auto rows_of = [&](int i) { return a.row[i + 1] - a.row[i]; };
    int longest = 0;
    long long tiles = 0;
    double keys = 0;
    auto more = [&](long long n, int len) {
        tiles += n * a.n_kv_heads;
        keys += (double)n * a.n_kv_heads * len;
        longest = std::max(longest, len);
    };
    for (int i = 0; i < a.n; ++i) more(tiles_of(rows_of(i)), paged_len(a, i));
    if (pools)
        for (int g = 0; g < a.n_pools; ++g) more(tiles_of(a.row[a.pool[g].end] - a.row[a.pool[g].begin]), a.pool[g].len);
    auto cut = [&](int share) {
        long long items = 0;
        for (int i = 0; i < a.n; ++i) {
            a.req[i].first = (int)items;
            items += tiles_of(rows_of(i)) * a.n_kv_heads * paged_parts(paged_len(a, i), share);
        }
        a.pool_first = (int)items;
        if (pools)
            for (int g = 0; g < a.n_pools; ++g) {
                a.pool[g].first = (int)items;
                items += tiles_of(a.row[a.pool[g].end] - a.row[a.pool[g].begin]) * a.n_kv_heads * paged_parts(a.pool[g].len, share);
            }
        return items;
    };
    // Whether parts pay: what a compute unit has to bring of whole sequences goes by latency, parts come at memory's rate but have to be joined (measured for cross attention; where prefixes are
    // read apart there is something to join anyhow).
    const double row = 2.0 * a.head_dim * element_bytes, all = keys * row, rate = all <= 256 << 20 ? 45e3 : d == 64 ? 22e3 : 32e3;
    const double here = (longest + (double)((tiles - 1) / n_cu) * keys / tiles) * row;
    const bool alike = longest * (double)tiles <= 1.25 * keys;
    const int most = (d == 128 ? 2 : alike ? 4 : 8) * n_cu;
    a.share = 0;
    if ((pools && a.n_pools) || here / rate > 1.1 * all / 5.1e6 + 5) a.share = paged_share(keys, tiles, longest, most, cut);
    a.pool_share = a.share;
    a.pool_height = PAGED_FEW_ROWS;
    a.items = (int)cut(a.share);
    a.pool_parts = a.parts + (size_t)a.pool_first * paged_part_floats(16, d);
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

// Prefixes' tiles of many rows, in a launch of their own behind that of the requests' own rows.
inline int pool_rows(const PagedArgs& a, int g) { return a.row[a.pool[g].end] - a.row[a.pool[g].begin]; }
// Their height, 0: tiles of 16 serve (few rows of each, short ones, or no room for the parts).
inline int paged_pool_height(const PagedArgs& a, int n_cu)
{
    int most = 0;
    for (int g = 0; g < a.n_pools; ++g)
        if (a.pool[g].len >= 512) most = std::max(most, pool_rows(a, g));
    if (most < 64) return 0;
    const int height = most > 64 ? 128 : 64;
    long long tiles = 0, own = 0;
    for (int g = 0; g < a.n_pools; ++g) tiles += (pool_rows(a, g) + height - 1) / height * a.n_kv_heads;
    for (int i = 0; i < a.n; ++i) own += (a.row[i + 1] - a.row[i] + 15) / 16 * a.n_kv_heads;
    return tiles * height <= (paged_room(a.n_kv_heads) - std::max<long long>(own, 8 * n_cu)) * PAGED_FEW_ROWS ? height : 0;
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

// Requests of many rows, gathered: the height of a tile.
inline int plan_paged_many(PagedArgs& a, int n_cu)
{
    constexpr int OWN = 160;             // a tile's own cost, in keys (measured for cross attention)
    long long large = 0;
    int longest = 0;
    for (int i = 0; i < a.n; ++i) {
        large += (long long)(a.row[i + 1] - a.row[i] + 255) / 256 * a.n_kv_heads;
        longest = std::max(longest, paged_len(a, i));
    }
    const int height = longest >= 1024 && large >= n_cu - n_cu / 4 ? 256 : 128;
    auto tiles_of = [&](int i) { return (a.row[i + 1] - a.row[i] + height - 1) / height * a.n_kv_heads; };
    int at = 0;
    for (int i = 0; i < a.n; ++i) {
        a.req[i].first = at;
        at += tiles_of(i);
    }
    a.share = a.pool_share = 0;
    a.pool_height = height;
    a.items = a.pool_first = at;
    plan_runs(a, 0, a.n, [&](int i) {
        const int q = (a.row[i + 1] - a.row[i]) / (a.n_heads / a.n_kv_heads);
        return std::pair<int, double>(tiles_of(i), OWN + paged_len(a, i) - (a.causal ? std::min(q, a.req[i].own_len) / 2 : 0));
    });
    return height;
}

}  // namespace tts
