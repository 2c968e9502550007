// Attention of a dynamic batch to a paged cache: every query row of a request attends its prefix's rows and its own up to its place, o = softmax(scale * q k^T) v, several query heads to
// a head of k and v.  One pass over the keys with the softmax's running maximum and sum.  A prefix that several requests share is read once for all of them: their rows are rows of one
// product.  What of a row's keys was taken apart (prefix and own rows, parts of long sequences) meets by way of each part's maximum, sum and columns.
//
// Keys come 16 at a time: pages have whole 16s, so that 16 keys of a head lie back to back in one page, whose number is the wave's, not the lane's, to look up.
#include "past_kernels.h"
#include "attend.h"
#include "lds_loads.h"
#include "words.h"

#include <algorithm>
#include <type_traits>

namespace tts {

namespace {

constexpr int NO_LIMIT = 0x7FFFFFFF;

// The launch's requests: a lane has every 64th, so that one trip to the arguments finds what a tile or a row is of.
template <typename Args> struct Requests {
    static constexpr int N = (Args::BATCH + 63) / 64;
    PagedReq r[N];
    int row[N];
    __device__ __forceinline__ void load(const Args& p)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = min(64 * i + lane, p.n - 1);
            const uint4 x = *reinterpret_cast<const uint4*>(&p.req[at]);
            r[i] = PagedReq{x.x, (int)x.y, (int)x.z, (int)x.w};
            row[i] = p.row[at];
        }
    }
    // the last whose tiles begin at or ahead of `id`
    __device__ __forceinline__ int of_tile(const Args& p, int id) const
    {
        const int lane = threadIdx.x & 63;
        int before = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) before += __popcll(__ballot(64 * i + lane < p.n && r[i].first <= id));
        return __builtin_amdgcn_readfirstlane(before) - 1;
    }
    // the last whose rows begin at or ahead of the lane's `of`, by halves
    __device__ __forceinline__ int of_row(const Args& p, int of) const
    {
        int at = 0;
#pragma unroll
        for (int by = Args::BATCH / 2; by > 0; by /= 2) {
            const int first = pick(row, at + by);
            at = at + by < p.n && first <= of ? at + by : at;
        }
        return at;
    }
    // a number of the lane's request
    static __device__ __forceinline__ int pick(const int (&x)[N], int at)
    {
        int y = __shfl(x[0], at & 63, 64);
#pragma unroll
        for (int i = 1; i < N; ++i) {
            const int other = __shfl(x[i], at & 63, 64);
            y = at >= 64 * i ? other : y;
        }
        return y;
    }
    template <typename F> __device__ __forceinline__ int pick(F of, int at) const
    {
        int x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = of(r[i]);
        return pick(x, at);
    }
};

// Which keys a tile of rows goes over: rows of the table, how long, where the own ones begin.
struct Sequence {
    int pre_row, pre_len, own_row, own_len, own_at;
    __device__ __forceinline__ int end() const { return own_len ? own_at + own_len : pre_len; }
    // 16 keys from `key` on, a multiple of 16: how many there are, and where they lie in a head of the cache (elements; somewhere in it if there are none).  Where the sequence is not empty.
    __device__ __forceinline__ int look(const PagedCommon& p, int key, long long& at) const
    {
        const bool own = key >= own_at && own_len > 0;
        const int j = own ? key - own_at : key, len = own ? own_len : pre_len, row = own ? own_row : pre_row, there = min(j, len - 1) >> p.page_shift;
        // (numbers of pages do not change while a kernel runs: the scalar cache's loads, which wait for no others; without a branch, so that several go together)
        using Table = const __attribute__((address_space(4))) int*;
        const int page = ((Table)(uintptr_t)p.table)[(long long)row * p.table_cols + there];
        const int n = (unsigned)page < (unsigned)p.n_pages ? max(0, min(16, len - j)) : 0;
        at = n > 0 ? page * p.page_stride + (long long)(j & ((1 << p.page_shift) - 1)) * p.head_dim : 0;
        return n;
    }
};

// A number of rows (query, head of the group), or the rows ahead of one, as queries.
template <typename Args> __device__ __forceinline__ int rows_to_queries(const Args& p, int rows)
{
    return __builtin_expect(p.by_group == NOT_BY, 0) ? rows / (p.n_heads / p.n_kv_heads) : over(rows, p.by_group);
}

// What a tile of rows is of: rows first_row .. row_end - 1 of the launch, a head of k and v, keys begin .. end - 1 of a sequence.
struct Item {
    Sequence seq;
    int first_row, row_end, kv, begin, end;
    int part;                            // index of its part; -1: the rows are whole with it
    int request, request_row, queries;   // of one request: which, its first row, its queries; -1: a prefix's
    int pool;                            // its prefix, read apart, -1: none
    int slots;                           // 1, 2, 4, 8 or 16: rows of the tile at most
    // how many keys a row may see
    template <typename Args> __device__ __forceinline__ int limit_of(const Args& p, int row) const
    {
        return p.causal && request >= 0 ? seq.own_at + max(0, seq.own_len - queries + rows_to_queries(p, row - request_row) + 1) : NO_LIMIT;
    }
};
template <int HEIGHT, typename Args> __device__ __forceinline__ Item item_of(const Args& p, Requests<Args>& all, int id)
{
    Item t;
    const bool own = !p.pooled || id < p.pool_first;
    // (steps of one query each, say: nothing to look for)
    if (own ? !p.per || !p.each : !p.each || p.q_first < 0 || p.share) all.load(p);
    if (own) {
        PagedReq r;
        int i, rows;
        if (p.per && p.each) {
            i = over(id, p.by_per);
            r = p.req[i];
            t.request_row = i * p.each;
            rows = p.each;
        } else {
            i = all.of_tile(p, id);
            const int at = i & 63;
#pragma unroll
            for (int k = 0; k < Requests<Args>::N; ++k)
                if (i >> 6 == k) {
                    r = PagedReq{(unsigned)__builtin_amdgcn_readlane((int)all.r[k].len_prefix, at), __builtin_amdgcn_readlane(all.r[k].table_row, at), __builtin_amdgcn_readlane(all.r[k].q_row, at),
                                 __builtin_amdgcn_readlane(all.r[k].first, at)};
                    t.request_row = __builtin_amdgcn_readlane(all.row[k], at);
                }
            rows = p.row[i + 1] - t.request_row;
        }
        const int pool = prefix_of(r), len = paged_len(p, r), parts = paged_parts(len, p.share), tiles = (rows + HEIGHT - 1) / HEIGHT;
        int at = id - r.first, split = 0, tile = 0;
        if (HEIGHT == PAGED_FEW_ROWS) {
            if (parts > 1) {
                split = at % parts;
                at /= parts;
            }
            t.kv = at;
            if (tiles > 1) {
                tile = at % tiles;
                t.kv = at / tiles;
            }
        } else {
            // (the last tile first: it sees the most keys)
            tile = tiles - 1 - at % tiles;
            at /= tiles;
            split = at % parts;
            t.kv = at / parts;
        }
        t.seq.own_row = r.table_row;
        t.seq.own_len = own_len_of(r);
        const bool before = !p.pooled && pool >= 0;
        t.seq.pre_row = before ? p.pool[pool].table_row : 0;
        t.seq.pre_len = before ? p.pool[pool].len : 0;
        t.seq.own_at = (t.seq.pre_len + 15) / 16 * 16;
        t.first_row = t.request_row + tile * HEIGHT;
        t.row_end = t.request_row + rows;
        t.begin = split * p.share;
        t.end = parts == 1 ? t.seq.end() : min(t.seq.end(), t.begin + p.share);
        t.pool = p.pooled ? pool : -1;
        t.part = parts > 1 || t.pool >= 0 ? id : -1;
        t.request = i;
        t.queries = rows_to_queries(p, rows);
    } else {
        t.pool = 0;
        if (p.n_pools > 1) {
            const int lane = threadIdx.x & 63;
            t.pool = __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < p.n_pools && p.pool[min(lane, p.n_pools - 1)].first <= id))) - 1;
        }
        const PagedPool o = p.pool[t.pool];
        const int first_row = p.each ? o.begin * p.each : p.row[o.begin];
        t.row_end = p.each ? o.end * p.each : p.row[o.end];
        const int tiles = (t.row_end - first_row + HEIGHT - 1) / HEIGHT, parts = paged_parts(o.len, p.pool_share);
        int at = id - o.first, split = 0, tile;
        if (HEIGHT == PAGED_FEW_ROWS) {                  // (tiles over the same keys: an XCD's, where heads and parts are a multiple of eight)
            if (parts > 1) {
                split = at % parts;
                at /= parts;
            }
            t.kv = at % p.n_kv_heads;
            tile = at / p.n_kv_heads;
        } else {
            tile = at % tiles;
            at /= tiles;
            split = at % parts;
            t.kv = at / parts;
        }
        t.seq = {o.table_row, o.len, 0, 0, (o.len + 15) / 16 * 16};
        t.first_row = first_row + tile * HEIGHT;
        t.begin = split * p.pool_share;
        t.end = parts == 1 ? o.len : min(o.len, t.begin + p.pool_share);
        t.part = id - p.pool_first;
        t.request = t.queries = -1;
        t.request_row = 0;
    }
    const int left = t.row_end - t.first_row;
    t.slots = left > 8 ? 16 : left > 4 ? 8 : left > 2 ? 4 : left;
    return t;
}

// A lane's row of the launch: its query's row of q and out, its head, and how many of the sequence's keys it may see.
struct Row {
    long long q_row;
    int head, limit;
    int request;                         // of rows of a prefix that asked for it
    __device__ __forceinline__ Row() {}
    template <typename Args> __device__ __forceinline__ void of_request(const Args& p, const Item& t, int row)
    {
        const int group = p.n_heads / p.n_kv_heads, in = row - t.request_row, query = rows_to_queries(p, in);
        q_row = (long long)(p.q_first >= 0 ? p.q_first + rows_to_queries(p, t.request_row) : p.req[t.request].q_row) + query;
        head = t.kv * group + in - query * group;
    }
    template <typename Args> __device__ __forceinline__ Row(const Args& p, const Requests<Args>& all, const Item& t, int row)
    {
        row = min(row, t.row_end - 1);
        const int group = p.n_heads / p.n_kv_heads;
        limit = t.limit_of(p, row);
        request = t.request;
        if (t.request >= 0) of_request(p, t, row);
        else {
            request = p.each ? row / p.each : all.of_row(p, row);
            const int query = rows_to_queries(p, row);   // (rows of a request: a multiple of the group's heads)
            if (p.q_first >= 0) q_row = (long long)p.q_first + query;
            else {
                const int first = p.each ? request * p.each : Requests<Args>::pick(all.row, request);
                q_row = (long long)all.pick([](const PagedReq& r) { return r.q_row; }, request) + query - rows_to_queries(p, first);
            }
            head = t.kv * group + row - query * group;
        }
    }
};

__device__ __forceinline__ float log_sum(float m, float l)       // m in units of log2
{
    return l == 0.f ? -__builtin_inff() : ((m == -__builtin_inff() ? 0.f : m) + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// Keys that some of a tile's rows see and others do not (a request's last ones) may have an infinity or NaN for a value, which a weight of 0 would not keep from the latter.  Such values are
// taken out ahead of the product (`finite`) and, if there were any, added at the end to the rows that see them: their weight is some number above 0, and what comes of it is the value itself.
template <typename T> __device__ __forceinline__ bool not_finite_in(uint32_t w)
{
    if constexpr (sizeof(T) == 4) return (w & 0x7F800000u) == 0x7F800000u;
    else return (((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u) != 0;
}
template <typename T> __device__ __forceinline__ uint32_t finite(uint32_t w)
{
    if constexpr (sizeof(T) == 4) return not_finite_in<T>(w) ? 0 : w;
    else return w & ((w & 0x7F80u) == 0x7F80u ? 0xFFFF0000u : ~0u) & ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFFu : ~0u);
}
template <typename T> __device__ __forceinline__ float not_finite(T x)
{
    const float f = to_float(x);
    return not_finite_in<float>(__float_as_uint(f)) ? f : 0.f;
}

// Where a wave's step of 16 or 32 keys lies, and how many of each 16 there are.
template <int TILES> struct Place {
    long long at[TILES];
    int n[TILES];
    __device__ __forceinline__ void look(const PagedCommon& p, const Sequence& seq, int first)
    {
#pragma unroll
        for (int i = 0; i < TILES; ++i) n[i] = seq.look(p, first + 16 * i, at[i]);
    }
};

// A wave's rows over keys: the lane's part of a step's keys and values, its query row's running softmax (maximum of all keys so far, sum of the lane's own keys, the outputs' columns).
template <typename T, int D, bool FULL> struct PagedRunning : Operands<T, D> {
    using G = Geometry<T, D>;
    using Operands<T, D>::k;
    using Operands<T, D>::v;
    static constexpr int WORDS = G::NE * sizeof(T) / 4;
    uint4 q[G::NF];
    floatx4 o[G::NE] = {};
    float m = -__builtin_inff(), l = 0;
    bool odd = false;                    // whether a value was taken out
    __device__ __forceinline__ void load_keys(const char* kp, const Place<G::TILES>& place, int head_dim, int lane)
    {
        const int g = lane >> 4, c = lane & 15;
        const uint32_t k_at = c * head_dim * (uint32_t)sizeof(T) + 16 * g;
#pragma unroll
        for (int t = 0; t < G::TILES; ++t) {
            const char* from = kp + place.at[t] * (long long)sizeof(T);
#pragma unroll
            for (int f = 0; f < G::NF; ++f)
                k[t][f] = *reinterpret_cast<const uint4*>(from + (FULL || (4 * f + g) * G::EPL < head_dim ? k_at + 64 * f : 0));
        }
    }
    // Columns that narrower heads have not: zeros (here, where the loads are waited for)
    __device__ __forceinline__ void narrow(int head_dim, int lane)
    {
        if constexpr (!FULL)
#pragma unroll
            for (int f = 0; f < G::NF; ++f) {
                const bool in = (4 * f + (lane >> 4)) * G::EPL < head_dim;
#pragma unroll
                for (int t = 0; t < G::TILES; ++t) k[t][f] = in ? k[t][f] : make_uint4(0, 0, 0, 0);
            }
    }
    __device__ __forceinline__ void load_values(const char* vp, const Place<G::TILES>& place, int head_dim, int lane)
    {
        const int g = lane >> 4, c = lane & 15;
        const uint32_t v_column = G::NE * c < head_dim ? G::NE * c : 0;
#pragma unroll
        for (int i = 0; i < G::PER_LANE; ++i) {
            const char* from = vp + place.at[i / 4] * (long long)sizeof(T) + ((4 * g + (i & 3)) * head_dim + v_column) * (uint32_t)sizeof(T);
            if constexpr (G::NE * sizeof(T) == 8) *reinterpret_cast<uint2*>(v[i]) = *reinterpret_cast<const uint2*>(from);
            else
#pragma unroll
                for (size_t b = 0; b < G::NE * sizeof(T); b += 16) *reinterpret_cast<uint4*>(v[i] + b / 4) = *reinterpret_cast<const uint4*>(from + b);
        }
    }
    // Keys that there are not (n: how many there are of each 16), or not for this row (from `limit` on): no score.  `first`: the step's first
    static __device__ __forceinline__ void hide(float (&s)[G::PER_LANE], const int (&n)[G::TILES], int first, int limit, int g)
    {
#pragma unroll
        for (int i = 0; i < G::PER_LANE; ++i) s[i] = ((4 * g + (i & 3) < n[i / 4]) & (first + G::key(i, g) < limit)) ? s[i] : -__builtin_inff();
    }
    // Scores become weights.
    __device__ __forceinline__ void weigh(float (&s)[G::PER_LANE], float scale)
    {
        float top = s[0];
#pragma unroll
        for (int i = 1; i < G::PER_LANE; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(m, across_max(top) * scale);
        const float base = top == -__builtin_inff() ? 0.f : top, by = __builtin_amdgcn_exp2f(m - base);
        m = top;
        l *= by;
#pragma unroll
        for (int i = 0; i < G::PER_LANE; ++i) {
            s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale, -base));
            l += s[i];
        }
#pragma unroll
        for (int e = 0; e < G::NE; ++e) o[e] *= by;
    }
    // Keys that there are not, or not for any row (from `end` on): no value either (0 times an infinity would be NaN); of those from `clear` on, which not all rows see, no infinities and NaN.
    __device__ __forceinline__ void mend(const int (&n)[G::TILES], int first, int clear, int end, int g)
    {
#pragma unroll
        for (int i = 0; i < G::PER_LANE; ++i) {
            const uint32_t there = 4 * g + (i & 3) < min(n[i / 4], end - first - 16 * (i / 4)) ? ~0u : 0u;
#pragma unroll
            for (int e = 0; e < WORDS; ++e) v[i][e] &= there;
        }
        if (clear >= end || first + G::N <= clear) return;
        bool any = false;
#pragma unroll
        for (int i = 0; i < G::PER_LANE; ++i)
#pragma unroll
            for (int e = 0; e < WORDS; ++e) any |= not_finite_in<T>(v[i][e]);
        if (__builtin_expect(__any(any), 0)) {
            odd = true;
#pragma unroll
            for (int i = 0; i < G::PER_LANE; ++i)
#pragma unroll
                for (int e = 0; e < WORDS; ++e) v[i][e] = first + G::key(i, g) >= clear ? finite<T>(v[i][e]) : v[i][e];
        }
    }
    // ... which the rows that see them have here.
    __device__ __forceinline__ void add_odd(const PagedCommon& p, const Sequence& seq, const char* vp, int from, int to, int limit, int g)
    {
        for (int key = from; key < to; ++key) {
            long long at;
            if (key % 16 >= seq.look(p, key / 16 * 16, at)) continue;
            const T* value = reinterpret_cast<const T*>(vp) + at + key % 16 * p.head_dim;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < G::NE; ++e) {
                    const float x = not_finite(value[min(G::NE * (4 * g + j) + e, p.head_dim - 1)]);
                    o[e][j] += key < limit ? x : 0.f;
                }
        }
    }
};

// Floats that one XCD writes and another reads within a launch (sc1: stores go through to memory, loads look past the caches).
struct Shared {
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ __forceinline__ Shared(float* at, int floats) : rsrc(__builtin_amdgcn_make_buffer_rsrc(at, 0, 4 * floats, BUFFER_RSRC_RAW)) {}
    __device__ __forceinline__ void put(int at, float x) const { __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), rsrc, 4 * at, 0, AGENT); }
    __device__ __forceinline__ void put4(int at, const float* x) const
    {
        __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])}, rsrc, 4 * at, 0, AGENT);
    }
    __device__ __forceinline__ float get(int at) const { return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rsrc, 4 * at, 0, AGENT)); }
    __device__ __forceinline__ void get4(int at, float* x) const
    {
        const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(rsrc, 4 * at, 0, AGENT);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
    }
};

// The parts of a row that a tile has one of: tiles of its own keys' from `own` on and its row of them, its prefix's from `pre` on.
struct Parts {
    int own_parts = 1, own = 0, in_own = 0, pre_parts = 0, pre = 0, in_pre = 0;
    __device__ __forceinline__ int all() const { return own_parts + pre_parts; }
    template <typename Args> __device__ __forceinline__ void look(const Args& p, const Requests<Args>& requests, const Item& t, int row, int request)
    {
        row = min(row, t.row_end - 1);
        if (t.request >= 0) {
            own_parts = paged_parts(t.seq.own_at + t.seq.own_len, p.share);
            own = t.part - (p.share ? t.begin / p.share : 0);
            in_own = row - t.first_row;
            if (t.pool >= 0) {
                const PagedPool o = p.pool[t.pool];
                const int in = row - (p.each ? o.begin * p.each : p.row[o.begin]);
                pre_parts = paged_parts(o.len, p.pool_share);
                pre = o.first - p.pool_first + (in / 16 * p.n_kv_heads + t.kv) * pre_parts;
                in_pre = in % 16;
            }
        } else {
            pre_parts = paged_parts(t.seq.pre_len, p.pool_share);
            pre = t.part - (p.pool_share ? t.begin / p.pool_share : 0);
            in_pre = row - t.first_row;
            const int begin = p.each ? request * p.each : p.row[request], in = row - begin, rows = p.each ? p.each : p.row[request + 1] - begin;
            if (p.share) own_parts = paged_parts(requests.pick([](const PagedReq& r) { return own_len_of(r); }, request), p.share);
            own = (p.per ? request * p.per : p.req[request].first) + (t.kv * ((rows + 15) / 16) + in / 16) * own_parts;
            in_own = in % 16;
        }
    }
};

// A tile of 16 rows over a part of its sequence; the waves take steps of keys in turn, the next one's on its way, and meet in LDS.
//
// Bound by latency: from the launch to the first step's scores lie three dependent trips to memory (arguments, a page's number, keys), 3.2 us with the way out; then a step of 32 keys takes
// a wave what 16 KB take from wherever they are, and many of them the memory's rate (16 requests over 3000 to 9000 rows, 16 heads of 128 that share 4: 40 us, 4.0 TB/s; a short one by itself
// 7.2). One step's registers, whose keys and values are asked for again as they are used up, leave room for 3 or 4 workgroups a compute unit; two steps' in turn were 20 KB of code and
// slower (15.2 against 12.8 us over 30 drawn calls). A workgroup has eight waves while that leaves no compute unit without one: their steps in turn are a shorter way through a sequence.
template <typename T, int D, bool FULL, int WAVES, typename Args> __global__ __launch_bounds__(WAVES * 64, D == 128 ? (WAVES == 4 && sizeof(T) == 2 ? 3 : 2) : 4) void k_paged_few(Args p)
{
    using G = Geometry<T, D>;
    constexpr int NE = G::NE, PITCH = D + 4, STRIDE = WAVES * G::N;
    __shared__ __align__(16) float s_o[WAVES][16][PITCH];
    __shared__ float s_ml[WAVES][2][16];
    Requests<Args> all;
    const Item t = item_of<PAGED_FEW_ROWS>(p, all, blockIdx.x);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, g = lane >> 4;
    const Row mine(p, all, t, t.first_row + (lane & 15));
    const T* q_at = static_cast<const T*>(p.q) + mine.q_row * p.q_stride + mine.head * p.head_dim;
    PagedRunning<T, D, FULL> run;
#pragma unroll
    for (int f = 0; f < G::NF; ++f) {
        const int d = (4 * f + g) * G::EPL;
        const bool there = FULL || d < p.head_dim;
        const uint4 x = *reinterpret_cast<const uint4*>(q_at + (there ? d : 0));
        run.q[f] = there ? x : make_uint4(0, 0, 0, 0);
    }
    const size_t head_at = (size_t)t.kv * (p.head_dim << p.page_shift) * sizeof(T);
    const char *kp = static_cast<const char*>(p.k_pages) + head_at, *vp = static_cast<const char*>(p.v_pages) + head_at;
    // keys from `clear` on are not seen by all rows, from `end` on by none
    const int end = min(t.end, __builtin_amdgcn_readlane(mine.limit, 15)), clear = min(end, __builtin_amdgcn_readfirstlane(mine.limit)), limit = min(mine.limit, end);
    const int begin = t.begin + wave * G::N;
    if (begin < end) {
        // The next step's keys are asked for when this one's have been used, its values when this one's have: one step's registers, always one half of a step on its way.  (Of a step that
        // there is not some other keys are, and nobody takes them.)
        const int last = (end - 1) / 16 * 16;
        Place<G::TILES> now, next;
        now.look(p, t.seq, begin);
        run.load_keys(kp, now, p.head_dim, lane);
        run.load_values(vp, now, p.head_dim, lane);
        for (int first = begin; first < end; first += STRIDE) {
            next.look(p, t.seq, min(first + STRIDE, last));
            float s[G::PER_LANE];
            run.narrow(p.head_dim, lane);
            run.scores(run.q, s);
            __builtin_amdgcn_sched_barrier(0);
            run.load_keys(kp, next, p.head_dim, lane);
            __builtin_amdgcn_sched_barrier(0);
            bool whole = first + G::N <= clear;
#pragma unroll
            for (int i = 0; i < G::TILES; ++i) whole &= now.n[i] == 16;
            if (!whole) run.hide(s, now.n, first, limit, g);
            run.weigh(s, p.scale);
            if (!whole) run.mend(now.n, first, clear, end, g);
            run.add(s, run.o);
            __builtin_amdgcn_sched_barrier(0);
            run.load_values(vp, next, p.head_dim, lane);
            now = next;
        }
        if (__builtin_expect(run.odd, 0))
            for (int first = begin; first < end; first += STRIDE) run.add_odd(p, t.seq, vp, max(first, clear), min(first + G::N, end), mine.limit, g);
    }
    const float l = across_sum(run.l);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < NE; ++e) s_o[wave][lane & 15][NE * (4 * g + j) + e] = run.o[e][j];
    if (g == 0) {
        s_ml[wave][0][lane] = run.m;
        s_ml[wave][1][lane] = l;
    }
    __syncthreads();
    // a row's columns are 16 threads', of four waves; what its place is a lane of this wave has
    const int in_tile = threadIdx.x / 16 % 16, chunk = threadIdx.x & 15;
    const long long q_row = (long long)((unsigned long long)(unsigned)__shfl((int)(mine.q_row >> 32), in_tile, 64) << 32 | (unsigned)__shfl((int)mine.q_row, in_tile, 64));
    const int head = __shfl(mine.head, in_tile, 64);
    const bool works = WAVES == 4 || threadIdx.x < 256;
    float top = -__builtin_inff(), sum = 0, c[NE] = {};
    if (works) {
#pragma unroll
        for (int i = 0; i < WAVES; ++i) top = fmaxf(top, s_ml[i][0][in_tile]);
        const float base = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float by = __builtin_amdgcn_exp2f(s_ml[i][0][in_tile] - base);
            sum += by * s_ml[i][1][in_tile];
#pragma unroll
            for (int e = 0; e < NE; ++e) c[e] += by * s_o[i][in_tile][NE * chunk + e];
        }
    }
    bool there = works && t.first_row + in_tile < t.row_end;
    if (t.part >= 0) {
        // rows of columns, then the rows' maxima and sums, past the caches: whoever joins them may be on another XCD
        constexpr int FLOATS = (int)paged_part_floats(16, D);
        const Shared parts(p.parts, p.part_floats);
        const int pools_at = (int)(p.pool_parts - p.parts);
        if (works) {
            const int to = (t.request >= 0 ? 0 : pools_at) + t.part * FLOATS;
#pragma unroll
            for (int e = 0; e < NE; e += 4) parts.put4(to + in_tile * D + NE * chunk + e, c + e);
            if (chunk == 0) {
                parts.put(to + 16 * D + in_tile, top);
                parts.put(to + 16 * D + 16 + in_tile, sum);
            }
        }
        if (!p.join) return;
        // This part is there for everybody; then whoever counts the last of a row's joins it: which that is does not matter to the result, parts go four by four to p.subs sums in turn, and these
        // meet in LDS.  Rows are fewer than 16, often: then their sums go to different groups of 16 threads.
        const int row_in = in_tile % t.slots, sub = in_tile / t.slots, subs = 16 / t.slots;
        Parts at;
        at.look(p, all, t, t.first_row + row_in, __shfl(mine.request, row_in, 64));
        there = works && t.first_row + row_in < t.row_end;
        stores_done();
        __syncthreads();
        __shared__ int s_last[16];
        if (works && chunk == 0 && sub == 0) {
            int* count = p.arrived + (size_t)t.kv * p.rows + min(t.first_row + row_in, t.row_end - 1);
            const bool last = there && __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == at.all() - 1;
            if (last) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last[row_in] = last;
        }
        __syncthreads();
        there = there && s_last[row_in];
        constexpr int AT_ONCE = 4;
        for (int one = sub; one < p.subs; one += subs) {
            top = -__builtin_inff();
            sum = 0;
#pragma unroll
            for (int e = 0; e < NE; ++e) c[e] = 0;
            for (int n = AT_ONCE * one; there && n < at.all(); n += AT_ONCE * p.subs) {
                float m[AT_ONCE], l[AT_ONCE], x[AT_ONCE][NE];
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    const int i = min(n + k, at.all() - 1);
                    const bool of_own = i < at.own_parts;
                    const int from = of_own ? (at.own + i) * FLOATS : pools_at + (at.pre + i - at.own_parts) * FLOATS, r = of_own ? at.in_own : at.in_pre;
                    m[k] = parts.get(from + 16 * D + r);
                    l[k] = parts.get(from + 16 * D + 16 + r);
#pragma unroll
                    for (int e = 0; e < NE; e += 4) parts.get4(from + r * D + NE * chunk + e, x[k] + e);
                }
                float most = top;
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) most = n + k < at.all() ? fmaxf(most, m[k]) : most;
                const float base = most == -__builtin_inff() ? 0.f : most, by = __builtin_amdgcn_exp2f(top - base);
                top = most;
                sum *= by;
#pragma unroll
                for (int e = 0; e < NE; ++e) c[e] *= by;
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    if (n + k >= at.all()) continue;
                    const float w = __builtin_amdgcn_exp2f(m[k] - base);
                    sum += w * l[k];
#pragma unroll
                    for (int e = 0; e < NE; ++e) c[e] += w * x[k][e];
                }
            }
            if (p.subs > 1 && works) {   // (s_o and s_ml have been read by everybody)
                s_ml[one][0][row_in] = top;
                s_ml[one][1][row_in] = sum;
#pragma unroll
                for (int e = 0; e < NE; ++e) s_o[one][row_in][NE * chunk + e] = c[e];
            }
        }
        there = there && sub == 0;
        if (p.subs > 1) {
            __syncthreads();
            if (there) {
                top = -__builtin_inff();
                for (int n = 0; n < p.subs; ++n) top = fmaxf(top, s_ml[n][0][row_in]);
                const float base = top == -__builtin_inff() ? 0.f : top;
                sum = 0;
#pragma unroll
                for (int e = 0; e < NE; ++e) c[e] = 0;
                for (int n = 0; n < p.subs; ++n) {
                    const float by = __builtin_amdgcn_exp2f(s_ml[n][0][row_in] - base);
                    sum += by * s_ml[n][1][row_in];
#pragma unroll
                    for (int e = 0; e < NE; ++e) c[e] += by * s_o[n][row_in][NE * chunk + e];
                }
            }
        }
    }
    if (!there) return;
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int e = 0; e < NE; ++e) c[e] *= inv;
    if (NE * chunk < p.head_dim) store_columns<T, NE>(static_cast<T*>(p.out) + q_row * p.out_stride + head * p.head_dim + NE * chunk, c);
    if (p.lse && chunk == 0) p.lse[q_row * p.n_heads + head] = log_sum(top, sum);
}

// Many rows, two bytes: 32 * NW rows, 32 a wave, over the keys in tiles of 64 that all waves read from LDS while the next R - 1 are on their way there, 16 bytes a lane straight from
// memory; one barrier a tile.  Where 64 tiles' keys lie, and which there are, is looked up at once and kept in LDS.
//
// Bound by the matrix pipe's and the softmax's turns, one behind the other in a wave: a tile's 64 keys take a workgroup of 128 rows by itself 1.25 us (columns 128; 64: 0.9), two of them a
// compute unit 0.97 each (three of 64: 0.69), 1.1 PFLOP/s of the pipe's 2.5 (8 prompts of 1500 to 4000 behind a prefix of 500, 16 heads of 128 that share 4: 478 us, 0.88 over the scores
// that count). A second workgroup a compute unit is worth more than taller tiles (2 slots of 32 KB and 232 registers leave room for it): 256 rows, three slots, took 289 us for 2 requests of
// 4096 where 128 take 294, but 72 against 56 for one of 512 over 2560. All waves take all of the workgroup's tiles: where they skipped
// those that their rows do not see, the compiler kept every sum twice and copied all of them each tile, with registers in scratch memory besides (the prompts 588 us).  Two such forms gave wrong results
// now and then with two workgroups a compute unit, and why is not known: by its code the copies stood as far behind the matrix instructions as they have to (48 more wait states there changed nothing), no scalar
// register was read too early, and barriers and waits are the ones below.  The build ends if this kernel spills again.
template <int D, int NW, int R> struct PagedMany {
    static constexpr int ROW = 2 * D, PART = KEYS * ROW, SLOT = 2 * PART, LOADS = PART / 1024 / NW, AHEAD = 64, SIXTEENS = 2 * AHEAD * KEYS / 16;
    static constexpr int LDS = R * SLOT + SIXTEENS * 10 + 16;            // 8 bytes for where 16 keys lie, 2 for which of them there are; whether a value was taken out
    static_assert(LOADS * 1024 * NW == PART, "shares of the waves");
};

template <int D, int NW, int R, bool FULL, typename Args> __global__ __launch_bounds__(64 * NW, D == 128 ? 2 : 3) void k_paged_many(Args p)
{
    using M = PagedMany<D, NW, R>;
    constexpr int ROW = M::ROW, NK = D / 16, HEIGHT = 32 * NW;
    extern __shared__ __align__(16) char lds[];
    long long* where = reinterpret_cast<long long*>(lds + R * M::SLOT);
    uint16_t* which = reinterpret_cast<uint16_t*>(where + M::SIXTEENS);
    int* odd = reinterpret_cast<int*>(which + M::SIXTEENS);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
    const int xcd = blockIdx.x & 7, id = p.start[xcd] + (blockIdx.x >> 3);
    if (id >= p.start[xcd + 1]) return;
    Requests<Args> all;
    const Item t = item_of<HEIGHT>(p, all, id);
    // keys that the workgroup's last row sees, that all of its rows do; that the wave's last does, that all of the wave's do
    const int end = min(t.end, t.limit_of(p, min(t.row_end, t.first_row + HEIGHT) - 1)), all_clear = min(end, t.limit_of(p, t.first_row));
    const int wave_end = min(end, t.limit_of(p, min(t.row_end - 1, t.first_row + 32 * wave + 31))), clear = min(end, t.limit_of(p, min(t.row_end - 1, t.first_row + 32 * wave)));
    const int first_tile = t.begin / KEYS, n_tiles = (end + KEYS - 1) / KEYS;
    auto look = [&](int first) {         // 64 tiles from `first` on
        for (int i = threadIdx.x; i < M::AHEAD * KEYS / 16; i += 64 * NW) {
            const int key = first * KEYS + 16 * i;
            if (key - 16 * i % KEYS >= end) break;       // (whole tiles)
            long long at = 0;
            const int n = key < end ? t.seq.look(p, key, at) : 0;
            where[(first * (KEYS / 16) + i) % M::SIXTEENS] = 2 * at;
            which[(first * (KEYS / 16) + i) % M::SIXTEENS] = (uint16_t)((1u << n) - 1);
        }
    };
    look(first_tile);
    const int row = t.first_row + 32 * wave + c;
    const int limit = t.limit_of(p, min(row, t.row_end - 1));
    ManyRunning<D> run;
    {
        const Row mine(p, all, t, row);
        const bf16_t* from = static_cast<const bf16_t*>(p.q) + mine.q_row * p.q_stride + mine.head * p.head_dim;
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            const int d = 16 * k + 8 * h;
            const uint4 x = *reinterpret_cast<const uint4*>(from + (FULL || d < p.head_dim ? d : 0));
            run.q[k] = FULL || d < p.head_dim ? x : make_uint4(0, 0, 0, 0);
        }
    }
    // this wave's share of a tile: the row and piece that lie where the lane's 16 bytes go
    int from_row[M::LOADS];
    uint32_t k_offset[M::LOADS], v_offset[M::LOADS];
    bool k_there[M::LOADS], v_there[M::LOADS];
#pragma unroll
    for (int i = 0; i < M::LOADS; ++i) {
        const int at = (wave + i * NW) * 1024 + lane * 16, at_row = at / ROW, piece = at % ROW / 16, k_piece = key_piece<D>(at_row, piece), v_piece = value_piece<D>(at_row, piece);
        from_row[i] = at_row;
        k_there[i] = FULL || 8 * k_piece < p.head_dim;
        v_there[i] = FULL || 8 * v_piece < p.head_dim;
        k_offset[i] = 2 * (at_row % 16 * p.head_dim + 8 * k_piece);
        v_offset[i] = 2 * (at_row % 16 * p.head_dim + 8 * v_piece);
    }
    const uint32_t lds_at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)lds;
    const size_t head_at = (size_t)t.kv * (p.head_dim << p.page_shift) * 2;
    const char *kp = static_cast<const char*>(p.k_pages) + head_at, *vp = static_cast<const char*>(p.v_pages) + head_at;
    auto same = [](uint64_t x) -> uint64_t {             // of a value that all lanes have
        const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)x), high = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
        return (uint64_t)high << 32 | low;
    };
    auto ask_which = [&](int tile) { return *reinterpret_cast<const uint64_t*>(which + tile * (KEYS / 16) % M::SIXTEENS); };
    auto bring = [&](int tile, int slot) {
        uint64_t from[M::LOADS];
#pragma unroll
        for (int i = 0; i < M::LOADS; ++i) from[i] = same((uint64_t)where[(tile * (KEYS / 16) + (wave + i * NW) * 1024 / ROW / 16) % M::SIXTEENS]);
#pragma unroll
        for (int i = 0; i < M::LOADS; ++i) {
            const uint32_t to = lds_at + slot * M::SLOT + (wave + i * NW) * 1024;
            if (k_there[i]) to_lds_from<16>(kp + from[i], k_offset[i], to);
            if (v_there[i]) to_lds_from<16>(vp + from[i], v_offset[i], to + M::PART);
        }
    };
    if (!FULL)                           // (columns that there are not: zeros, which nothing is loaded over)
        for (int i = threadIdx.x; i < R * M::SLOT / 16; i += 64 * NW) reinterpret_cast<uint4*>(lds)[i] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x == 0) *odd = 0;
    __syncthreads();
    for (int i = 0; i < R - 1 && first_tile + i < n_tiles; ++i) bring(first_tile + i, i);
    uint64_t next_which = ask_which(first_tile);
    // The queries are here, with the first tile: waited for in the loop, they would be together with the tiles that are on their way.
#pragma unroll
    for (int k = 0; k < NK; ++k) asm volatile("" : "+v"(run.q[k].x), "+v"(run.q[k].y), "+v"(run.q[k].z), "+v"(run.q[k].w));
    for (int tile = first_tile, slot = 0, free = R - 1; tile < n_tiles; ++tile) {
        // (the tiles behind this one that are on their way: R - 2 but at the end)
        if (tile + R - 2 < n_tiles) arrived<(R - 2) * 2 * M::LOADS>();
        else arrived<0>();
        if ((tile - first_tile) % M::AHEAD == M::AHEAD / 2 && tile + M::AHEAD / 2 < n_tiles) {
            look(tile + M::AHEAD / 2);
            __syncthreads();
        }
        if (tile + R - 1 < n_tiles) bring(tile + R - 1, free);
        const uint64_t mask = same(next_which);
        next_which = ask_which(tile + 1);
        const char* keys = lds + slot * M::SLOT;
        char* values = lds + slot * M::SLOT + M::PART;
        const int key = tile * KEYS;
        if (mask != ~0ull || key + KEYS > all_clear) {
            // values of keys that there are not: zeros (0 times an infinity would be NaN); infinities and NaN of those that not all rows see are taken out
            bool bad = false;
#pragma unroll
            for (int i = 0; i < M::LOADS; ++i) {
                uint4* at = reinterpret_cast<uint4*>(values + (wave + i * NW) * 1024 + lane * 16);
                if (!(mask >> from_row[i] & 1)) *at = make_uint4(0, 0, 0, 0);
                else if (key + from_row[i] >= all_clear) {
                    const uint4 x = *at;
                    const bool here = not_finite_in<bf16_t>(x.x) || not_finite_in<bf16_t>(x.y) || not_finite_in<bf16_t>(x.z) || not_finite_in<bf16_t>(x.w);
                    if (here) *at = make_uint4(finite<bf16_t>(x.x), finite<bf16_t>(x.y), finite<bf16_t>(x.z), finite<bf16_t>(x.w));
                    bad |= here;
                }
            }
            if (bad) *odd = 1;
            lds_barrier();
        }
        // (by all waves, also those whose rows end before: the tile's barrier waits for the others, and a branch here had the compiler copy all sums from turn to turn)
        const int seen = min(limit, end) - key;
        const uint64_t own = key + KEYS <= clear ? mask : mask & (seen >= KEYS ? ~0ull : seen <= 0 ? 0ull : (1ull << seen) - 1);
        run.template take<2>(keys, values, mask != ~0ull || key + KEYS > clear, own, p.scale, lane);
        free = slot;                                     // (the slot that the tile before this one was in)
        slot = slot + 1 == R ? 0 : slot + 1;
    }
    lds_barrier();
    if (*odd)
        for (int key = all_clear; key < wave_end; ++key) {
            long long at;
            if (key % 16 >= t.seq.look(p, key / 16 * 16, at) || key < t.begin) continue;
            const bf16_t* value = reinterpret_cast<const bf16_t*>(vp) + at + key % 16 * p.head_dim;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int column = 32 * d + 8 * (i / 4) + 4 * h + (i & 3);
                    const float x = not_finite(value[min(column, p.head_dim - 1)]);
                    run.o[d][i] += key < limit ? x : 0.f;
                }
        }
    const float l = run.sum(), m = run.m;
    if (t.part >= 0) {
        float* part = (t.request >= 0 ? p.parts : p.pool_parts) + t.part * paged_part_floats(HEIGHT, D);
        const int in_tile = 32 * wave + c;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(part + in_tile * D + 32 * d + 2 * i + 4 * h) = make_float4(run.o[d][i], run.o[d][i + 1], run.o[d][i + 2], run.o[d][i + 3]);
        if (h == 0) {
            part[HEIGHT * D + in_tile] = m;
            part[HEIGHT * D + HEIGHT + in_tile] = l;
        }
        return;
    }
    // (looked up again: its registers are the loop's)
    int again = min(row, t.row_end - 1);
    asm volatile("" : "+v"(again));
    Row mine;
    mine.of_request(p, t, again);
    run.store(static_cast<bf16_t*>(p.out) + mine.q_row * p.out_stride + mine.head * p.head_dim, l == 0.f ? 0.f : 1.0f / l, row < t.row_end, p.head_dim, lane);
    if (p.lse && row < t.row_end && h == 0) p.lse[mine.q_row * p.n_heads + mine.head] = log_sum(m, l);
}

// A row from its parts, its own keys' and its prefix's: their maxima give each a weight, then the row's waves take parts in turn, a column or two a lane, and meet in LDS.
// Bound by latency: 4096 rows of 17 parts, 36 MB, take 12.0 us by a wave a row, eight parts a turn of the loop (four: 13.1; all eight asked for ahead of the first's use: 13.1); by four waves a row
// 3 more, which fewer rows fill the card with.
constexpr int JOIN_WAVES = 4;
template <typename T, int D, int ACROSS, typename Args> __global__ __launch_bounds__(JOIN_WAVES * 64) void k_paged_join(Args p)
{
    constexpr int PER = D / 64, AT_ONCE = JOIN_WAVES / ACROSS;           // columns of a lane, rows of a workgroup
    __shared__ float s_m[JOIN_WAVES], s_l[JOIN_WAVES], s_o[JOIN_WAVES][D];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, of_row = wave % ACROSS;
    const int rows = p.rows, id = blockIdx.x * AT_ONCE + wave / ACROSS;
    const bool in = id < rows * p.n_kv_heads;
    const int row = in ? id % rows : 0, kv = in ? id / rows : 0;
    int i;
    if (p.each) i = row / p.each;
    else {
        Requests<Args> all;
        all.load(p);
        i = __builtin_amdgcn_readfirstlane(all.of_row(p, row));
    }
    const PagedReq r = p.req[i];
    const int pool = prefix_of(r), own_parts = paged_parts(paged_len(p, r), p.share), in_request = row - p.row[i];
    // (tiles in the order of item_of: of 16 rows a tile's parts one behind the other; of more a part's tiles, the last one first)
    const bool low = p.height == PAGED_FEW_ROWS;
    const int own_tiles = (p.row[i + 1] - p.row[i] + p.height - 1) / p.height, own_tile = in_request / p.height, own_step = low ? 1 : own_tiles;
    const int own_at = r.first + (low ? (kv * own_tiles + own_tile) * own_parts : kv * own_parts * own_tiles + own_tiles - 1 - own_tile);
    int pool_parts = 0, pool_at = 0, pool_step = 0, pool_row = 0;
    if (p.pooled && pool >= 0) {
        const PagedPool o = p.pool[pool];
        const int height = p.pool_height, in_pool = row - p.row[o.begin], tiles = (p.row[o.end] - p.row[o.begin] + height - 1) / height, tile = in_pool / height;
        pool_parts = paged_parts(o.len, p.pool_share);
        pool_row = in_pool % height;
        const bool few = height == PAGED_FEW_ROWS;
        pool_at = o.first - p.pool_first + (few ? (tile * p.n_kv_heads + kv) * pool_parts : kv * pool_parts * tiles + tile);
        pool_step = few ? 1 : tiles;
    }
    const int parts = own_parts + pool_parts;
    const bool todo = in && parts > 1;                   // (whole rows are there already)
    const float* own = p.parts + own_at * paged_part_floats(p.height, D);
    const float* pre = p.pool_parts + pool_at * paged_part_floats(p.pool_height, D);
    auto part_at = [&](int n, int& height, int& in_tile) -> const float* {
        const bool mine = n < own_parts;
        height = mine ? p.height : p.pool_height;
        in_tile = mine ? in_request % p.height : pool_row;
        return mine ? own + (size_t)n * own_step * paged_part_floats(p.height, D) : pre + (size_t)(n - own_parts) * pool_step * paged_part_floats(p.pool_height, D);
    };
    float m = -__builtin_inff(), l = 0, o[PER] = {};
    if (todo) {
#pragma unroll 8
        for (int n = of_row; n < parts; n += ACROSS) {
            int height, in_tile;
            const float* part = part_at(n, height, in_tile);
            const float m_here = part[height * D + in_tile], l_here = part[height * D + height + in_tile];
            float x[PER];
            if constexpr (PER == 2) *reinterpret_cast<float2*>(x) = *reinterpret_cast<const float2*>(part + in_tile * D + 2 * lane);
            else x[0] = part[in_tile * D + lane];
            const float top = fmaxf(m, m_here), base = top == -__builtin_inff() ? 0.f : top;
            const float by = __builtin_amdgcn_exp2f(m - base), w = __builtin_amdgcn_exp2f(m_here - base);
            l = by * l + w * l_here;
#pragma unroll
            for (int e = 0; e < PER; ++e) o[e] = by * o[e] + w * x[e];
            m = top;
        }
    }
    if constexpr (ACROSS > 1) {
#pragma unroll
        for (int e = 0; e < PER; ++e) s_o[wave][PER * lane + e] = o[e];
        if (lane == 0) {
            s_m[wave] = m;
            s_l[wave] = l;
        }
        __syncthreads();
        if (of_row != 0) return;
        float top = m;
#pragma unroll
        for (int n = 1; n < ACROSS; ++n) top = fmaxf(top, s_m[wave + n]);
        const float base = top == -__builtin_inff() ? 0.f : top;
        l = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] = 0;
#pragma unroll
        for (int n = 0; n < ACROSS; ++n) {
            const float by = __builtin_amdgcn_exp2f(s_m[wave + n] - base);
            l += by * s_l[wave + n];
#pragma unroll
            for (int e = 0; e < PER; ++e) o[e] += by * s_o[wave + n][PER * lane + e];
        }
        m = top;
    }
    if (!todo) return;
    const int group = p.n_heads / p.n_kv_heads, head = kv * group + in_request % group;
    const long long q_row = (long long)r.q_row + in_request / group;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    T* out = static_cast<T*>(p.out) + q_row * p.out_stride + head * p.head_dim + PER * lane;
    if (PER * lane < p.head_dim) {
        if constexpr (PER == 2 && sizeof(T) == 4) *reinterpret_cast<float2*>(out) = make_float2(o[0] * inv, o[1] * inv);
        else if constexpr (PER == 2) *reinterpret_cast<uint32_t*>(out) = pack_bf16x2(o[0] * inv, o[1] * inv);
        else *out = from_float<T>(o[0] * inv);
    }
    if (p.lse && lane == 0) p.lse[q_row * p.n_heads + head] = log_sum(m, l);
}

// Calls f with the launch's arguments, small ones where they do.
template <typename F> hipError_t with_args(const PagedArgs& a, F f)
{
    if (a.n > PAGED_SMALL || a.n_pools > PAGED_SMALL) return f(a);
    PagedArgsOf<PAGED_SMALL> small;
    static_cast<PagedCommon&>(small) = a;
    std::copy_n(a.req, a.n, small.req);
    std::copy_n(a.pool, a.n_pools, small.pool);
    std::copy_n(a.row, a.n + 1, small.row);
    return f(small);
}

template <typename T, int D, bool FULL> hipError_t go_few(const PagedArgs& a, int n_cu, hipStream_t s)
{
    return with_args(a, [&](const auto& args) {
        using Args = std::decay_t<decltype(args)>;
        if (a.items <= n_cu) hipLaunchKernelGGL((k_paged_few<T, D, FULL, 8, Args>), dim3(a.items), dim3(512), 0, s, args);
        else hipLaunchKernelGGL((k_paged_few<T, D, FULL, 4, Args>), dim3(a.items), dim3(256), 0, s, args);
        return hipGetLastError();
    });
}

template <int D, int NW, int R> hipError_t go_many(const PagedArgs& a, hipStream_t s)
{
    int most = 0;
    for (int i = 0; i < 8; ++i) most = std::max(most, a.start[i + 1] - a.start[i]);
    return with_args(a, [&](const auto& args) {
        using Args = std::decay_t<decltype(args)>;
        if (a.head_dim == D) hipLaunchKernelGGL((k_paged_many<D, NW, R, true, Args>), dim3(8 * most), dim3(64 * NW), (PagedMany<D, NW, R>::LDS), s, args);
        else hipLaunchKernelGGL((k_paged_many<D, NW, R, false, Args>), dim3(8 * most), dim3(64 * NW), (PagedMany<D, NW, R>::LDS), s, args);
        return hipGetLastError();
    });
}
template <int D, int NW, int R, bool FULL, int BATCH> hipError_t allow_one()
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_paged_many<D, NW, R, FULL, PagedArgsOf<BATCH>>), hipFuncAttributeMaxDynamicSharedMemorySize, PagedMany<D, NW, R>::LDS);
}
template <int D, int NW, int R> hipError_t allow()
{
    hipError_t e = allow_one<D, NW, R, true, PAGED_BATCH>();
    if (e == hipSuccess) e = allow_one<D, NW, R, false, PAGED_BATCH>();
    if (e == hipSuccess) e = allow_one<D, NW, R, true, PAGED_SMALL>();
    if (e == hipSuccess) e = allow_one<D, NW, R, false, PAGED_SMALL>();
    return e;
}

template <typename T, int D> hipError_t go_join(const PagedArgs& a, hipStream_t s)
{
    return with_args(a, [&](const auto& args) {
        using Args = std::decay_t<decltype(args)>;
        const long long rows = (long long)a.rows * a.n_kv_heads;
        if (rows >= 2048) hipLaunchKernelGGL((k_paged_join<T, D, 1, Args>), dim3((unsigned)((rows + JOIN_WAVES - 1) / JOIN_WAVES)), dim3(JOIN_WAVES * 64), 0, s, args);
        else hipLaunchKernelGGL((k_paged_join<T, D, JOIN_WAVES, Args>), dim3((unsigned)rows), dim3(JOIN_WAVES * 64), 0, s, args);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t allow_paged()
{
    hipError_t e = allow<64, 2, 3>();
    if (e == hipSuccess) e = allow<64, 4, 3>();
    if (e == hipSuccess) e = allow<128, 2, 2>();
    if (e == hipSuccess) e = allow<128, 4, 2>();
    return e;
}

hipError_t launch_paged_few(const PagedArgs& a, bool bf16, int n_cu, hipStream_t s)
{
    const bool wide = a.head_dim > 64, full = a.head_dim % 64 == 0;
    if (bf16 && wide) return full ? go_few<bf16_t, 128, true>(a, n_cu, s) : go_few<bf16_t, 128, false>(a, n_cu, s);
    if (bf16) return full ? go_few<bf16_t, 64, true>(a, n_cu, s) : go_few<bf16_t, 64, false>(a, n_cu, s);
    if (wide) return full ? go_few<float, 128, true>(a, n_cu, s) : go_few<float, 128, false>(a, n_cu, s);
    return full ? go_few<float, 64, true>(a, n_cu, s) : go_few<float, 64, false>(a, n_cu, s);
}

hipError_t launch_paged_many(const PagedArgs& a, int height, hipStream_t s)
{
    if (a.head_dim > 64) return height == 128 ? go_many<128, 4, 2>(a, s) : go_many<128, 2, 2>(a, s);
    return height == 128 ? go_many<64, 4, 3>(a, s) : go_many<64, 2, 3>(a, s);
}

hipError_t launch_paged_join(const PagedArgs& a, bool bf16, hipStream_t s)
{
    if (a.head_dim > 64) return bf16 ? go_join<bf16_t, 128>(a, s) : go_join<float, 128>(a, s);
    return bf16 ? go_join<bf16_t, 64>(a, s) : go_join<float, 64>(a, s);
}

}  // namespace tts
