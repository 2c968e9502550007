// The HIP calls and launch wrappers of fake_operators.cpp, and those of a decoder block's own past: what a call would have launched is written down.
#include "fake_operators.cpp"

#include "../paper_2211_13939_amd/csrc/paged_plan.h"

namespace {
// What an attention's launches were, and the first thing about them that is not as it has to be.
std::string wrong;
int few = 0, many = 0, joins = 0, pools = 0, split = 0, last_height = 0;
long long rows_seen = 0;
bool parts_pending = false, pools_pending = false;
void expect(bool ok, const char* what)
{
    if (!ok && wrong.empty()) wrong = what;
}
// Every tile of a launch: entries' tiles follow each other, parts cover their sequence, and what is written apart fits in the arena.
void look_at(const tts::PagedArgs& a, int height, bool requests, bool prefixes)
{
    using namespace tts;
    const long long room = (long long)paged_room(a.n_kv_heads) * paged_part_floats(16, paged_width(a.head_dim));
    const int group = a.n_heads / a.n_kv_heads;
    long long at = 0;
    bool apart = false;
    expect(a.n >= 1 && a.n <= PAGED_BATCH && a.n_pools <= PAGED_POOLS && a.row[0] == 0, "numbers of the launch");
    for (int i = 0; requests && i < a.n; ++i) {
        const int rows = a.row[i + 1] - a.row[i], len = paged_len(a, a.req[i]), parts = paged_parts(len, a.share), g = prefix_of(a.req[i]);
        expect(rows > 0 && rows % group == 0 && (!a.each || rows == a.each), "rows of a request");
        expect(g < a.n_pools && (g < 0 || (a.pool[g].begin <= i && i < a.pool[g].end)), "a request's prefix");
        expect(a.req[i].first == at, "a request's first tile");
        expect(parts == 1 || ((long long)parts * a.share >= len && a.share % 32 == 0 && parts <= PAGED_MAX_SPLITS), "a request's parts");
        at += (long long)(rows + height - 1) / height * a.n_kv_heads * parts;
        apart |= parts > 1 || (a.pooled && g >= 0);
        split += parts > 1;
        rows_seen += rows;
    }
    if (!requests) at = a.pool_first;
    expect(at == a.pool_first && (!apart || at * (long long)paged_part_floats(height, paged_width(a.head_dim)) <= room), "room for requests' parts");
    if (prefixes)
        for (int g = 0; g < a.n_pools; ++g) {
            const PagedPool& o = a.pool[g];
            const int parts = paged_parts(o.len, a.pool_share);
            expect(o.first == at && o.begin < o.end && o.len > 0 && (parts == 1 || (long long)parts * a.pool_share >= o.len), "a prefix's tiles");
            expect(parts == 1 || a.pool_share % 32 == 0, "a prefix's parts");
            at += (long long)(a.row[o.end] - a.row[o.begin] + a.pool_height - 1) / a.pool_height * a.n_kv_heads * parts;
            split += parts > 1;
        }
    const long long pool_floats = (at - a.pool_first) * (long long)paged_part_floats(a.pool_height, paged_width(a.head_dim));
    expect(!prefixes || (a.pool_parts - a.parts >= a.pool_first * (long long)paged_part_floats(16, paged_width(a.head_dim)) && a.pool_parts - a.parts + pool_floats <= room), "room for prefixes' parts");
    expect(a.items == at, "tiles of the launch");
    pools += prefixes ? a.n_pools : 0;
    expect(!a.join || ((apart || prefixes) && (prefixes || !a.pooled || !a.n_pools) && (long long)a.rows * a.n_kv_heads <= 16LL * paged_room(a.n_kv_heads)), "parts that the last one joins");
    expect(a.rows == a.row[a.n] && (!requests || a.per == 0 || a.per * a.n == a.pool_first), "numbers of the launch");
    parts_pending |= (apart || prefixes) && !a.join;
    joins += a.join;
    pools_pending = requests && !prefixes && a.pooled && a.n_pools;
}
tts::RotaryArgs rotary;
tts::AppendArgs append;
int append_rows = 0;
}  // namespace

namespace tts {
hipError_t launch_rotary(RotaryArgs& a, bool, bool, int, hipStream_t)
{
    ++launches;
    rotary = a;
    devices_seen = current;
    return call("launch");
}
hipError_t launch_append(AppendArgs& a, bool, bool, int, hipStream_t)
{
    ++launches;
    append = a;
    append_rows += a.rows;
    last_n = a.n;
    requests_seen += a.n;
    return call("launch");
}
hipError_t allow_paged() { return call("allow"); }
hipError_t launch_paged_few(const PagedArgs& a, bool, int, hipStream_t)
{
    ++launches;
    ++few;
    requests_seen += a.n;
    expect(!parts_pending, "parts that were not joined");
    look_at(a, PAGED_FEW_ROWS, true, a.pooled && a.n_pools && a.items > a.pool_first);
    return call("launch");
}
hipError_t launch_paged_many(const PagedArgs& a, int height, hipStream_t)
{
    ++launches;
    ++many;
    last_height = height;
    if (a.pooled) {
        expect(pools_pending && a.pool_height == height, "prefixes behind their requests");
        look_at(a, height, false, true);
    } else {
        requests_seen += a.n;
        expect(!parts_pending, "parts that were not joined");
        look_at(a, height, true, false);
    }
    expect(a.start[0] == (a.pooled ? a.pool_first : 0) && a.start[8] == a.items, "shares of the XCDs");
    for (int i = 0; i < 8; ++i) expect(a.start[i] <= a.start[i + 1], "shares in order");
    return call("launch");
}
hipError_t launch_paged_join(const PagedArgs&, bool, hipStream_t)
{
    ++launches;
    ++joins;
    expect(!pools_pending, "prefixes that were not read");
    parts_pending = false;
    return call("launch");
}
}  // namespace tts

extern "C" {
void past_reset()
{
    fake_reset();
    append_rows = few = many = joins = pools = split = last_height = 0;
    rows_seen = 0;
    parts_pending = pools_pending = false;
    wrong.clear();
}
const char* past_wrong()
{
    expect(!parts_pending, "parts that were not joined at the end");
    return wrong.c_str();
}
int past_few() { return few; }
int past_many() { return many; }
int past_joins() { return joins; }
int past_pools() { return pools; }
int past_split() { return split; }
int past_height() { return last_height; }
long long past_rows() { return rows_seen; }
int past_append_rows() { return append_rows; }
long long past_append_k() { return (long long)(size_t)append.k; }
int past_append_first(int i) { return append.req[i].first; }
int past_append_position(int i) { return append.req[i].position; }
int past_rotary_first() { return rotary.first; }
}
