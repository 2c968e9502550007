// Attention of a dynamic batch to a paged cache: every query row of a request attends its prefix's rows and its own up to its place, o = softmax(scale * q k^T) v, several query heads to
// a head of k and v.  One pass over the keys with the softmax's running maximum and sum.  A prefix that several requests share is read once for all of them: their rows are rows of one
// product.  What of a row's keys was taken apart (prefix and own rows, parts of long sequences) meets by way of each part's maximum, sum and columns.
//
// Keys come 16 at a time: pages have whole 16s, so that 16 keys of a head lie back to back in one page, whose number is the wave's, not the lane's, to look up.
#include "past_kernels.h"
#include "attend.h"

#include <algorithm>
#include <type_traits>

namespace tts {

namespace {

constexpr int FEW_WAVES = 4, NO_LIMIT = 0x7FFFFFFF;

// The entry (request or prefix) that tile `id` of a launch is of: the last whose tiles begin at or ahead of it.
template <typename Args> __device__ __forceinline__ int request_of_tile(const Args& p, int id)
{
    const int lane = threadIdx.x & 63;
    int before = 0;
#pragma unroll
    for (int i = 0; i < Args::BATCH; i += 64) before += __popcll(__ballot(i + lane < p.n && p.req[min(i + lane, p.n - 1)].first <= id));
    return __builtin_amdgcn_readfirstlane(before) - 1;
}
template <typename Args> __device__ __forceinline__ int pool_of_tile(const Args& p, int id)
{
    const int lane = threadIdx.x & 63;
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < p.n_pools && p.pool[min(lane, p.n_pools - 1)].first <= id))) - 1;
}
// The request of each lane's row of the launch (all lanes ask).
template <typename Args> __device__ __forceinline__ int request_of_row(const Args& p, int row)
{
    if (p.each) return row / p.each;
    const int lane = threadIdx.x & 63;
    int firsts[(Args::BATCH + 63) / 64], at = 0;
#pragma unroll
    for (int i = 0; i < Args::BATCH; i += 64) firsts[i / 64] = i + lane < p.n ? p.row[min(i + lane, p.n)] : NO_LIMIT;
    // the last whose first row is at or ahead of it, by halves
#pragma unroll
    for (int by = Args::BATCH / 2; by > 0; by /= 2) {
        const int ask = at + by;
        int first = __shfl(firsts[0], ask & 63, 64);
#pragma unroll
        for (int i = 64; i < Args::BATCH; i += 64) {
            const int other = __shfl(firsts[i / 64], ask & 63, 64);
            first = ask >= i ? other : first;
        }
        at = first <= row ? ask : at;
    }
    return at;
}

// Which keys a tile of rows goes over: rows of the table, how long, where the own ones begin.
struct Sequence {
    int pre_row, pre_len, own_row, own_len, own_at;
    __device__ __forceinline__ int end() const { return own_len ? own_at + own_len : pre_len; }
    // 16 keys from `key` on, a multiple of 16: how many there are, and where they lie in a head of the cache (elements; somewhere in it if there are none)
    __device__ __forceinline__ int look(const PagedCommon& p, int key, long long& at) const
    {
        const bool own = key >= own_at;
        const int j = own ? key - own_at : key, len = own ? own_len : pre_len, row = own ? own_row : pre_row;
        int n = max(0, min(16, len - j));
        int page = -1;
        // (numbers of pages do not change while a kernel runs: the scalar cache's loads, which wait for no others)
        using Table = const __attribute__((address_space(4))) int*;
        if (n > 0) page = ((Table)(uintptr_t)p.table)[(long long)row * p.table_cols + (j >> p.page_shift)];
        if ((unsigned)page >= (unsigned)p.n_pages) n = 0;
        at = n > 0 ? page * p.page_stride + (long long)(j & ((1 << p.page_shift) - 1)) * p.head_dim : 0;
        return n;
    }
};

// What a tile of rows is of: rows first_row .. row_end - 1 of the launch, a head of k and v, keys begin .. end - 1 of a sequence.
struct Item {
    Sequence seq;
    int first_row, row_end, kv, begin, end, part;        // part: index of its part; -1: the rows are whole with it
    int request;                                         // -1: of a prefix
};
template <int HEIGHT, typename Args> __device__ __forceinline__ Item item_of(const Args& p, int id)
{
    Item t;
    if (!p.pooled || id < p.pool_first) {
        const int i = request_of_tile(p, id);
        const PagedReq r = p.req[i];
        const int pool = p.pool_of[i], len = paged_len(p, i), parts = paged_parts(len, p.share);
        const int rows = p.row[i + 1] - p.row[i], tiles = (rows + HEIGHT - 1) / HEIGHT;
        int at = id - r.first, split, tile;
        if (HEIGHT == PAGED_FEW_ROWS) {
            split = at % parts;
            at /= parts;
            tile = at % tiles;
            t.kv = at / tiles;
        } else {
            // (the last tile first: it sees the most keys)
            tile = tiles - 1 - at % tiles;
            at /= tiles;
            split = at % parts;
            t.kv = at / parts;
        }
        t.seq.own_row = r.table_row;
        t.seq.own_len = r.own_len;
        const bool before = !p.pooled && pool >= 0;
        t.seq.pre_row = before ? p.pool[pool].table_row : 0;
        t.seq.pre_len = before ? p.pool[pool].len : 0;
        t.seq.own_at = (t.seq.pre_len + 15) / 16 * 16;
        t.first_row = p.row[i] + tile * HEIGHT;
        t.row_end = p.row[i + 1];
        t.begin = split * p.share;
        t.end = parts == 1 ? t.seq.end() : min(t.seq.end(), t.begin + p.share);
        t.part = parts > 1 || (p.pooled && pool >= 0) ? id : -1;
        t.request = i;
    } else {
        const PagedPool o = p.pool[pool_of_tile(p, id)];
        const int rows = p.row[o.end] - p.row[o.begin], tiles = (rows + HEIGHT - 1) / HEIGHT, parts = paged_parts(o.len, p.pool_share);
        int at = id - o.first, split, tile;
        if (HEIGHT == PAGED_FEW_ROWS) {                  // (tiles over the same keys: an XCD's, where heads and parts are a multiple of eight)
            split = at % parts;
            at /= parts;
            t.kv = at % p.n_kv_heads;
            tile = at / p.n_kv_heads;
        } else {
            tile = at % tiles;
            at /= tiles;
            split = at % parts;
            t.kv = at / parts;
        }
        t.seq = {o.table_row, o.len, 0, 0, (o.len + 15) / 16 * 16};
        t.first_row = p.row[o.begin] + tile * HEIGHT;
        t.row_end = p.row[o.end];
        t.begin = split * p.pool_share;
        t.end = parts == 1 ? o.len : min(o.len, t.begin + p.pool_share);
        t.part = id - p.pool_first;
        t.request = -1;
    }
    return t;
}

// A lane's row of the launch: its query's row of q and out, its head, and how many of the sequence's keys it may see.
struct Row {
    long long q_row;
    int head, limit;
    template <typename Args> __device__ __forceinline__ Row(const Args& p, const Item& t, int row)
    {
        row = min(row, t.row_end - 1);
        const int group = p.n_heads / p.n_kv_heads, i = t.request >= 0 ? t.request : request_of_row(p, row);
        const int in = row - p.row[i], query = in / group;
        q_row = (long long)p.req[i].q_row + query;
        head = t.kv * group + in % group;
        limit = NO_LIMIT;
        if (p.causal && t.request >= 0) limit = t.seq.own_at + max(0, t.seq.own_len - (p.row[i + 1] - p.row[i]) / group + query + 1);
    }
};

__device__ __forceinline__ float log_sum(float m, float l)       // m in units of log2
{
    return l == 0.f ? -__builtin_inff() : ((m == -__builtin_inff() ? 0.f : m) + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// Keys that some of a tile's rows see and others do not (a request's last ones) may have an infinity or NaN for a value, which a weight of 0 would not keep from the latter.  Such values are
// taken out ahead of the product (`finite`) and, if there were any, added at the end to the rows that see them: their weight is some number above 0, and what comes of it is the value itself.
template <typename T> __device__ __forceinline__ uint32_t finite(uint32_t w, bool& odd)
{
    if constexpr (sizeof(T) == 4) {
        const bool bad = (w & 0x7F800000u) == 0x7F800000u;
        odd |= bad;
        return bad ? 0 : w;
    } else {
        const bool low = (w & 0x7F80u) == 0x7F80u, high = (w & 0x7F800000u) == 0x7F800000u;
        odd |= low | high;
        return w & (low ? 0xFFFF0000u : ~0u) & (high ? 0xFFFFu : ~0u);
    }
}
template <typename T> __device__ __forceinline__ float not_finite(T x)
{
    const float f = to_float(x);
    return (__float_as_uint(f) & 0x7F800000u) == 0x7F800000u ? f : 0.f;
}

// A step of a wave: 16 or 32 keys.  Where they lie and how many of each 16 there are; the lane's part of them.
template <typename T, int D, bool FULL> struct PagedKeys : Operands<T, D> {
    using G = Geometry<T, D>;
    using Operands<T, D>::k;
    using Operands<T, D>::v;
    int n[G::TILES];
    __device__ __forceinline__ void load(const char* kp, const char* vp, const long long (&at)[G::TILES], const int (&there)[G::TILES], int head_dim, int lane)
    {
        const int g = lane >> 4, c = lane & 15;
        const uint32_t k_at = c * head_dim * (uint32_t)sizeof(T) + 16 * g, v_column = G::NE * c < head_dim ? G::NE * c : 0;
#pragma unroll
        for (int t = 0; t < G::TILES; ++t) {
            n[t] = there[t];
            const char* from = kp + at[t] * (long long)sizeof(T);
#pragma unroll
            for (int f = 0; f < G::NF; ++f) {
                if constexpr (FULL) k[t][f] = *reinterpret_cast<const uint4*>(from + (k_at + 64 * f));
                else {
                    const bool in = (4 * f + g) * G::EPL < head_dim;
                    const uint4 x = *reinterpret_cast<const uint4*>(from + (in ? k_at + 64 * f : 0));
                    k[t][f] = in ? x : make_uint4(0, 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < G::PER_LANE; ++i) {
            const char* from = vp + at[i / 4] * (long long)sizeof(T) + ((4 * g + (i & 3)) * head_dim + v_column) * (uint32_t)sizeof(T);
            if constexpr (G::NE * sizeof(T) == 8) *reinterpret_cast<uint2*>(v[i]) = *reinterpret_cast<const uint2*>(from);
            else
#pragma unroll
                for (size_t b = 0; b < G::NE * sizeof(T); b += 16) *reinterpret_cast<uint4*>(v[i] + b / 4) = *reinterpret_cast<const uint4*>(from + b);
        }
    }
};

// The running softmax of a lane's query row: maximum (of all keys so far), sum (of the lane's own keys), the outputs' columns.
template <typename T, int D, bool FULL> struct PagedRunning {
    using G = Geometry<T, D>;
    floatx4 o[G::NE] = {};
    float m = -__builtin_inff(), l = 0;
    bool odd = false;                    // whether a value was taken out
    // first: the step's first key; keys from `limit` on the lane's row does not see, ahead of `clear` every row sees all
    __device__ __forceinline__ void step(PagedKeys<T, D, FULL>& now, const uint4 (&q)[G::NF], float scale, int first, int limit, int clear, int g)
    {
        float s[G::PER_LANE];
        now.scores(q, s);
        bool whole = first + G::N <= clear;
#pragma unroll
        for (int t = 0; t < G::TILES; ++t) whole &= now.n[t] == 16;
        if (!whole) {
            // keys that there are not, or not for this row: no score; of the former no value either (0 times an infinity would be NaN)
#pragma unroll
            for (int i = 0; i < G::PER_LANE; ++i) {
                const int key = first + G::key(i, g);
                const bool there = 4 * g + (i & 3) < now.n[i / 4];
                s[i] = (there & (key < limit)) ? s[i] : -__builtin_inff();
#pragma unroll
                for (size_t e = 0; e < G::NE * sizeof(T) / 4; ++e) {
                    bool bad = false;
                    const uint32_t left = finite<T>(now.v[i][e], bad);
                    now.v[i][e] = there ? key < clear ? now.v[i][e] : left : 0;
                    odd |= there & (key >= clear) & bad;
                }
            }
        }
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
        now.add(s, o);
    }
};

// A tile of 16 rows over a part of its sequence; the waves take steps of keys in turn, the next one's on its way, and meet in LDS.
template <typename T, int D, bool FULL, typename Args> __global__ __launch_bounds__(FEW_WAVES * 64) void k_paged_few(Args p)
{
    using G = Geometry<T, D>;
    constexpr int NE = G::NE, PITCH = D + 4, STRIDE = FEW_WAVES * G::N;
    __shared__ __align__(16) float s_o[FEW_WAVES][16][PITCH];
    __shared__ float s_ml[FEW_WAVES][2][16];
    const Item t = item_of<PAGED_FEW_ROWS>(p, blockIdx.x);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, g = lane >> 4;
    const Row mine(p, t, t.first_row + (lane & 15));
    const T* q_at = static_cast<const T*>(p.q) + mine.q_row * p.q_stride + mine.head * p.head_dim;
    uint4 q[G::NF];
#pragma unroll
    for (int f = 0; f < G::NF; ++f) {
        const int d = (4 * f + g) * G::EPL;
        const bool there = FULL || d < p.head_dim;
        const uint4 x = *reinterpret_cast<const uint4*>(q_at + (there ? d : 0));
        q[f] = there ? x : make_uint4(0, 0, 0, 0);
    }
    const size_t head_at = (size_t)t.kv * (p.head_dim << p.page_shift) * sizeof(T);
    const char *kp = static_cast<const char*>(p.k_pages) + head_at, *vp = static_cast<const char*>(p.v_pages) + head_at;
    const int clear = __builtin_amdgcn_readfirstlane(mine.limit), end = min(t.end, __builtin_amdgcn_readlane(mine.limit, 15));
    PagedRunning<T, D, FULL> run;
    PagedKeys<T, D, FULL> a, b;
    auto load = [&](PagedKeys<T, D, FULL>& to, int first) {
        long long at[G::TILES];
        int n[G::TILES];
#pragma unroll
        for (int i = 0; i < G::TILES; ++i) n[i] = t.seq.look(p, first + 16 * i, at[i]);
        to.load(kp, vp, at, n, p.head_dim, lane);
    };
    auto step = [&](PagedKeys<T, D, FULL>& now, int first) { run.step(now, q, p.scale, first, min(mine.limit, end), min(clear, end), g); };
    int first = t.begin + wave * G::N;
    if (first < end) {
        load(a, first);
        for (; first + STRIDE < end; first += 2 * STRIDE) {
            load(b, first + STRIDE);
            step(a, first);
            load(a, min(first + 2 * STRIDE, (end - 1) / 16 * 16));       // (a step that there is not: some keys, and nobody takes them)
            step(b, first + STRIDE);
        }
        if (first < end) step(a, first);
    }
    if (__any(run.odd))
        for (first = t.begin + wave * G::N; first < end; first += STRIDE)
            for (int key = max(first, clear); key < min(first + G::N, end); ++key) {
                long long at;
                if (key % 16 >= t.seq.look(p, key / 16 * 16, at)) continue;
                const T* value = reinterpret_cast<const T*>(vp) + at + key % 16 * p.head_dim;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < NE; ++e) {
                        const int column = NE * (4 * g + j) + e;
                        const float x = not_finite(value[FULL || column < p.head_dim ? column : 0]);
                        run.o[e][j] += key < mine.limit ? x : 0.f;
                    }
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
    const int in_tile = threadIdx.x / 16, chunk = threadIdx.x & 15;
    float top = -__builtin_inff(), sum = 0, c[NE] = {};
#pragma unroll
    for (int i = 0; i < FEW_WAVES; ++i) top = fmaxf(top, s_ml[i][0][in_tile]);
    const float base = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
    for (int i = 0; i < FEW_WAVES; ++i) {
        const float by = __builtin_amdgcn_exp2f(s_ml[i][0][in_tile] - base);
        sum += by * s_ml[i][1][in_tile];
#pragma unroll
        for (int e = 0; e < NE; ++e) c[e] += by * s_o[i][in_tile][NE * chunk + e];
    }
    if (t.part >= 0) {                   // rows of columns, then the rows' maxima and sums
        float* part = (t.request >= 0 ? p.parts : p.pool_parts) + t.part * paged_part_floats(16, D);
        store_columns<float, NE>(part + in_tile * D + NE * chunk, c);
        if (chunk == 0) {
            part[16 * D + in_tile] = top;
            part[16 * D + 16 + in_tile] = sum;
        }
        return;
    }
    const Row row(p, t, t.first_row + in_tile);
    if (t.first_row + in_tile >= t.row_end) return;
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int e = 0; e < NE; ++e) c[e] *= inv;
    if (NE * chunk < p.head_dim) store_columns<T, NE>(static_cast<T*>(p.out) + row.q_row * p.out_stride + row.head * p.head_dim + NE * chunk, c);
    if (p.lse && chunk == 0) p.lse[row.q_row * p.n_heads + row.head] = log_sum(top, sum);
}

// Many rows, two bytes: 32 * NW rows, 32 a wave, over the keys in tiles of 64 that all waves read from LDS while the next R - 1 are on their way there, 16 bytes a lane straight from
// memory; one barrier a tile.  Where 64 tiles' keys lie, and which there are, is looked up at once and kept in LDS.
template <int D, int NW, int R> struct PagedMany {
    static constexpr int ROW = 2 * D, PART = KEYS * ROW, SLOT = 2 * PART, LOADS = PART / 1024 / NW, AHEAD = 64, SIXTEENS = 2 * AHEAD * KEYS / 16;
    static constexpr int LDS = R * SLOT + SIXTEENS * 10 + 16;            // 8 bytes for where 16 keys lie, 2 for which of them there are; whether a value was taken out
    static_assert(LOADS * 1024 * NW == PART, "shares of the waves");
};
// 16 bytes a lane to LDS, from a wave's address and a lane's offset
__device__ __forceinline__ void to_lds_from(const char* base, uint32_t offset, uint32_t to)
{
    uint32_t m0;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" : "={m0}"(m0) : "s"(to), "v"(offset), "s"(base) : "memory");
}

template <int D, int NW, int R> __global__ __launch_bounds__(64 * NW, D == 128 ? 2 : NW == 8 ? 4 : 3) void k_paged_many(PagedArgs p)
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
    const Item t = item_of<HEIGHT>(p, id);
    const int row = t.first_row + 32 * wave + c;
    const Row mine(p, t, row);
    ManyRunning<D> run;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
        const int d = 16 * k + 8 * h;
        const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(p.q) + mine.q_row * p.q_stride + mine.head * p.head_dim + (d < p.head_dim ? d : 0));
        run.q[k] = d < p.head_dim ? x : make_uint4(0, 0, 0, 0);
    }
    // keys that the workgroup's last row sees, that the wave's last does, that all of the wave's rows do, and all of the workgroup's
    const Row last(p, t, t.row_end - 1 < t.first_row + HEIGHT - 1 ? t.row_end - 1 : t.first_row + HEIGHT - 1);
    const int end = min(t.end, __builtin_amdgcn_readfirstlane(last.limit)), wave_end = min(end, __builtin_amdgcn_readlane(mine.limit, 31)), clear = min(end, __builtin_amdgcn_readfirstlane(mine.limit));
    const Row top(p, t, t.first_row);
    const int all_clear = min(end, __builtin_amdgcn_readfirstlane(top.limit));
    const int first_tile = t.begin / KEYS, n_tiles = (end + KEYS - 1) / KEYS;
    // this wave's share of a tile: the row and piece that lie where the lane's 16 bytes go
    int from_row[M::LOADS];
    uint32_t k_offset[M::LOADS], v_offset[M::LOADS];
    bool k_there[M::LOADS], v_there[M::LOADS];
#pragma unroll
    for (int i = 0; i < M::LOADS; ++i) {
        const int at = (wave + i * NW) * 1024 + lane * 16, at_row = at / ROW, piece = at % ROW / 16, k_piece = key_piece<D>(at_row, piece), v_piece = value_piece<D>(at_row, piece);
        from_row[i] = at_row;
        k_there[i] = 8 * k_piece < p.head_dim;
        v_there[i] = 8 * v_piece < p.head_dim;
        k_offset[i] = 2 * (at_row % 16 * p.head_dim + 8 * k_piece);
        v_offset[i] = 2 * (at_row % 16 * p.head_dim + 8 * v_piece);
    }
    const uint32_t lds_at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)lds;
    const size_t head_at = (size_t)t.kv * (p.head_dim << p.page_shift) * 2;
    const char *kp = static_cast<const char*>(p.k_pages) + head_at, *vp = static_cast<const char*>(p.v_pages) + head_at;
    auto look = [&](int first) {         // 64 tiles from `first` on
        for (int i = threadIdx.x; i < M::AHEAD * KEYS / 16; i += 64 * NW) {
            const int key = first * KEYS + 16 * i;
            long long at;
            const int n = key < end ? t.seq.look(p, key, at) : 0;
            where[(first * (KEYS / 16) + i) % M::SIXTEENS] = n ? 2 * at : 0;
            which[(first * (KEYS / 16) + i) % M::SIXTEENS] = (uint16_t)((1u << n) - 1);
        }
    };
    auto same = [](uint64_t x) -> uint64_t {             // of a value that all lanes have
        const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)x), high = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
        return (uint64_t)high << 32 | low;
    };
    auto there = [&](int tile) { return same(*reinterpret_cast<const uint64_t*>(which + tile * (KEYS / 16) % M::SIXTEENS)); };
    auto bring = [&](int tile, int slot) {
#pragma unroll
        for (int i = 0; i < M::LOADS; ++i) {
            const long long from = (long long)same((uint64_t)where[(tile * (KEYS / 16) + (wave + i * NW) * 1024 / ROW / 16) % M::SIXTEENS]);
            const uint32_t to = lds_at + slot * M::SLOT + (wave + i * NW) * 1024;
            if (k_there[i]) to_lds_from(kp + from, k_offset[i], to);
            if (v_there[i]) to_lds_from(vp + from, v_offset[i], to + M::PART);
        }
    };
    if (p.head_dim < D)                  // (columns that there are not: zeros, which nothing is loaded over)
        for (int i = threadIdx.x; i < R * M::SLOT / 16; i += 64 * NW) reinterpret_cast<uint4*>(lds)[i] = make_uint4(0, 0, 0, 0);
    look(first_tile);
    if (threadIdx.x == 0) *odd = 0;
    __syncthreads();
    for (int i = 0; i < R - 1 && first_tile + i < n_tiles; ++i) bring(first_tile + i, i);
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
        const uint64_t mask = there(tile);
        const char* keys = lds + slot * M::SLOT;
        char* values = lds + slot * M::SLOT + M::PART;
        const int key = tile * KEYS;
        if (mask != 0 && (mask != ~0ull || key + KEYS > all_clear)) {
            // values of keys that there are not: zeros (0 times an infinity would be NaN); infinities and NaN of those that not all rows see are taken out
            bool bad = false;
#pragma unroll
            for (int i = 0; i < M::LOADS; ++i) {
                uint4* at = reinterpret_cast<uint4*>(values + (wave + i * NW) * 1024 + lane * 16);
                if (!(mask >> from_row[i] & 1)) *at = make_uint4(0, 0, 0, 0);
                else if (key + from_row[i] >= all_clear) {
                    const uint4 x = *at;
                    *at = make_uint4(finite<bf16_t>(x.x, bad), finite<bf16_t>(x.y, bad), finite<bf16_t>(x.z, bad), finite<bf16_t>(x.w, bad));
                }
            }
            if (bad) *odd = 1;
            lds_barrier();
        }
        if (mask != 0 && key < wave_end) {
            const int seen = min(mine.limit, end) - key;
            const uint64_t own = key + KEYS <= clear ? mask : mask & (seen >= KEYS ? ~0ull : seen <= 0 ? 0ull : (1ull << seen) - 1);
            run.template take<2>(keys, values, mask != ~0ull || key + KEYS > clear, own, p.scale, lane);
        }
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
                    run.o[d][i] += key < mine.limit ? x : 0.f;
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
    run.store(static_cast<bf16_t*>(p.out) + mine.q_row * p.out_stride + mine.head * p.head_dim, l == 0.f ? 0.f : 1.0f / l, row < t.row_end, p.head_dim, lane);
    if (p.lse && row < t.row_end && h == 0) p.lse[mine.q_row * p.n_heads + mine.head] = log_sum(m, l);
}

// A row from its parts, its own keys' and its prefix's: their maxima give each a weight, then the row's waves take parts in turn, a column or two a lane, and meet in LDS.
constexpr int JOIN_WAVES = 4;
template <typename T, int D, int ACROSS, typename Args> __global__ __launch_bounds__(JOIN_WAVES * 64) void k_paged_join(Args p)
{
    constexpr int PER = D / 64, AT_ONCE = JOIN_WAVES / ACROSS;           // columns of a lane, rows of a workgroup
    __shared__ float s_m[JOIN_WAVES], s_l[JOIN_WAVES], s_o[JOIN_WAVES][D];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, of_row = wave % ACROSS;
    const int rows = p.row[p.n], id = blockIdx.x * AT_ONCE + wave / ACROSS;
    const bool in = id < rows * p.n_kv_heads;
    const int row = in ? id % rows : 0, kv = in ? id / rows : 0, i = __builtin_amdgcn_readfirstlane(request_of_row(p, row)), pool = p.pool_of[i];
    const int own_parts = paged_parts(paged_len(p, i), p.share), in_request = row - p.row[i], own_tiles = (p.row[i + 1] - p.row[i] + 15) / 16;
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
    const float* own = p.parts + (p.req[i].first + (kv * own_tiles + in_request / 16) * own_parts) * paged_part_floats(16, D);
    const float* pre = p.pool_parts + pool_at * paged_part_floats(p.pool_height, D);
    auto part_at = [&](int n, int& height, int& in_tile) -> const float* {
        const bool mine = n < own_parts;
        height = mine ? 16 : p.pool_height;
        in_tile = mine ? in_request % 16 : pool_row;
        return mine ? own + n * paged_part_floats(16, D) : pre + (size_t)(n - own_parts) * pool_step * paged_part_floats(p.pool_height, D);
    };
    float m = -__builtin_inff(), l = 0, o[PER] = {};
    if (todo) {
#pragma unroll 4
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
    const long long q_row = (long long)p.req[i].q_row + in_request / group;
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
    std::copy_n(a.pool_of, a.n, small.pool_of);
    return f(small);
}

template <typename T, int D, bool FULL> hipError_t go_few(const PagedArgs& a, hipStream_t s)
{
    return with_args(a, [&](const auto& args) {
        hipLaunchKernelGGL((k_paged_few<T, D, FULL, std::decay_t<decltype(args)>>), dim3(a.items), dim3(FEW_WAVES * 64), 0, s, args);
        return hipGetLastError();
    });
}

template <int D, int NW, int R> hipError_t go_many(const PagedArgs& a, hipStream_t s)
{
    int most = 0;
    for (int i = 0; i < 8; ++i) most = std::max(most, a.start[i + 1] - a.start[i]);
    hipLaunchKernelGGL((k_paged_many<D, NW, R>), dim3(8 * most), dim3(64 * NW), (PagedMany<D, NW, R>::LDS), s, a);
    return hipGetLastError();
}
template <int D, int NW, int R> hipError_t allow()
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_paged_many<D, NW, R>), hipFuncAttributeMaxDynamicSharedMemorySize, PagedMany<D, NW, R>::LDS);
}

template <typename T, int D> hipError_t go_join(const PagedArgs& a, hipStream_t s)
{
    return with_args(a, [&](const auto& args) {
        using Args = std::decay_t<decltype(args)>;
        const long long rows = (long long)a.row[a.n] * a.n_kv_heads;
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
    if (e == hipSuccess) e = allow<64, 8, 3>();
    if (e == hipSuccess) e = allow<128, 2, 2>();
    if (e == hipSuccess) e = allow<128, 4, 2>();
    if (e == hipSuccess) e = allow<128, 8, 3>();
    return e;
}

hipError_t launch_paged_few(const PagedArgs& a, bool bf16, hipStream_t s)
{
    const bool wide = a.head_dim > 64, full = a.head_dim % 64 == 0;
    if (bf16 && wide) return full ? go_few<bf16_t, 128, true>(a, s) : go_few<bf16_t, 128, false>(a, s);
    if (bf16) return full ? go_few<bf16_t, 64, true>(a, s) : go_few<bf16_t, 64, false>(a, s);
    if (wide) return full ? go_few<float, 128, true>(a, s) : go_few<float, 128, false>(a, s);
    return full ? go_few<float, 64, true>(a, s) : go_few<float, 64, false>(a, s);
}

hipError_t launch_paged_many(const PagedArgs& a, int height, hipStream_t s)
{
    if (a.head_dim > 64) return height == 256 ? go_many<128, 8, 3>(a, s) : height == 128 ? go_many<128, 4, 2>(a, s) : go_many<128, 2, 2>(a, s);
    return height == 256 ? go_many<64, 8, 3>(a, s) : height == 128 ? go_many<64, 4, 3>(a, s) : go_many<64, 2, 3>(a, s);
}

hipError_t launch_paged_join(const PagedArgs& a, bool bf16, hipStream_t s)
{
    if (a.head_dim > 64) return bf16 ? go_join<bf16_t, 128>(a, s) : go_join<float, 128>(a, s);
    return bf16 ? go_join<bf16_t, 64>(a, s) : go_join<float, 64>(a, s);
}

}  // namespace tts
