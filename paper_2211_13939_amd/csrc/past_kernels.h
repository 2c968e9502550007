// Host-visible launch wrappers of the kernels of a decoder block's own past (rotary.hip, paged.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tts {

// x / y by 2^32 / y rounded up; y = 1: by 0.  Exact while x * y <= 2^32, for powers of two always.
constexpr unsigned by_of(unsigned y) { return y <= 1 ? 0 : (unsigned)(((1ull << 32) + y - 1) / y); }
constexpr unsigned NOT_BY = ~0u;         // (of no y)
__host__ __device__ inline int over(int x, unsigned by)
{
    return by ? (int)(((unsigned long long)(unsigned)x * by) >> 32) : x;
}

// How heads are dealt to a wave's lanes: a unit is what a lane has of a head, two chunks of `width` columns.  Halves: chunks that lie rot_dim / 2 apart, then what does not turn in
// neighbouring ones, the last of either so far back that it ends with them (what two lanes have they write alike); pairs: neighbouring chunks of 4.  Heads of `units` units lie `side` to a
// wave; of more than 64, in `blocks` of 64, and then no two have the same of what turns: a call in place would turn it twice.
struct TurnShape {
    int width, units, side, blocks;
};
inline TurnShape turn_shape(int head_dim, int rot_dim, bool pairs)
{
    TurnShape s;
    const int half = rot_dim / 2, rest = head_dim - rot_dim;
    for (s.width = pairs ? 4 : 8;; s.width /= 2) {
        s.units = pairs ? (head_dim + 7) / 8 : (half + s.width - 1) / s.width + (rest + 2 * s.width - 1) / (2 * s.width);
        if (pairs || s.width == 1 || ((!half || half >= s.width) && (!rest || rest >= s.width) && (half % s.width == 0 || s.units <= 64))) break;
    }
    s.side = s.units < 64 ? 64 / s.units : 1;
    s.blocks = (s.units + 63) / 64;
    return s;
}

struct TurnAngles {
    const uint64_t* freqs;               // turns a position, times 2^64
    float magnitude;
    int half, width, units, side, blocks;    // half: rot_dim / 2
    unsigned by_units;                   // for over()
    bool pairs;
};
struct RotaryArgs {
    const void* x;
    void* y;
    const int* positions;                // null: row r is at first + r
    long long x_stride, y_stride;        // elements
    TurnAngles turn;
    int rows, first, heads, head_dim;
    bool back;
    int per, jobs;                       // of a row: head steps of a wave, waves
    unsigned by_jobs;                    // for over(), where that is exact
};
hipError_t launch_rotary(RotaryArgs& a, bool x_bf16, bool y_bf16, int n_cu, hipStream_t s);

constexpr int APPEND_BATCH = 128, APPEND_SMALL = 16;     // requests of a launch
struct AppendReq {
    int first;                           // of its rows, in the launch
    int row, table_row, position;
};
struct AppendCommon {
    const void *k, *v, *q;               // the launch's first rows; q: null if there are none
    void *k_pages, *v_pages, *q_out;
    const int* table;
    long long k_stride, v_stride, q_stride, q_out_stride, page_stride;   // elements
    TurnAngles turn;
    int rows, n, heads, kv_heads, head_dim, n_pages, table_cols, page_shift;
    int per, k_jobs, v_jobs, q_jobs;     // of a row: head steps of a wave, waves
    int each;                            // rows of every request, 0: they differ
    unsigned by_each, by_jobs, by_v;     // for over() (by_jobs: where that is exact); v: lanes that a head takes
};
template <int N> struct AppendArgsOf : AppendCommon {
    static constexpr int BATCH = N;
    AppendReq req[N];
};
using AppendArgs = AppendArgsOf<APPEND_BATCH>;
hipError_t launch_append(AppendArgs& a, bool x_bf16, bool bf16, int n_cu, hipStream_t s);

// Attention to a paged cache.  What a launch's rows are: of the rows (query, head of a group) of its requests, as many for each head of k and v, `row` counts on from request to request.
// Requests of one prefix lie side by side.  A sequence of keys is a prefix's rows and a request's own behind them, which begin at a whole 16 (the keys between do not exist).
constexpr int PAGED_BATCH = 128, PAGED_SMALL = 16, PAGED_POOLS = 32;     // requests of a launch, prefixes
struct PagedReq {
    unsigned len_prefix;                 // rows of its own, and above 25 bits of them 1 + its prefix, 0: none
    int table_row, q_row;
    int first;                           // of its tiles (of all key heads and parts), in the launch
};
__host__ __device__ inline int own_len_of(const PagedReq& r) { return (int)(r.len_prefix & 0x1FFFFFFu); }
__host__ __device__ inline int prefix_of(const PagedReq& r) { return (int)(r.len_prefix >> 25) - 1; }
struct PagedPool {
    int table_row, len;
    int begin, end;                      // its requests in the launch
    int first;
};
struct PagedCommon {
    const void *q, *k_pages, *v_pages;
    const int* table;
    void* out;
    float *lse, *parts, *pool_parts;     // parts of requests' tiles; of prefixes'
    int part_floats;                     // room for parts, in floats
    int* arrived;                        // how many of a row's parts are there: [key heads][rows], zeros between launches
    long long q_stride, out_stride, page_stride;               // elements
    float scale;                         // times log2(e)
    int n_heads, n_kv_heads, head_dim, n_pages, table_cols, page_shift;
    int n, n_pools, rows;                // rows of all requests (of one key head)
    int each;                            // rows of every request, 0: they differ
    int per;                             // tiles of every request, 0: they differ
    unsigned by_per, by_group;           // 2^32 / per, 2^32 / group, rounded up (group: of query heads to a key head), for over(); by_group NOT_BY where that is not exact
    int q_first;                         // query row of the launch's first query, where they lie back to back; -1: they do not
    int items;                           // tiles of the launch
    int share, pool_share;               // length of a part of a request's keys, of a prefix's, 0: they have none
    int pool_first;                      // first tile that is a prefix's
    int height, pool_height;             // rows of a request's tile, of a prefix's
    bool causal;
    bool pooled;                         // prefixes have tiles of their own, over all their requests' rows; otherwise a request's keys begin with its prefix's
    bool join;                           // a row's last part to arrive joins them, in so many sums
    int subs;
    int start[9];                        // many rows: first of the tiles that each XCD takes
};
template <int N> struct PagedArgsOf : PagedCommon {
    static constexpr int BATCH = N, POOLS = N < PAGED_POOLS ? N : PAGED_POOLS;
    PagedReq req[N];
    PagedPool pool[POOLS];
    int row[N + 1];
};
using PagedArgs = PagedArgsOf<PAGED_BATCH>;
// Length of a request's keys, with its prefix's if that is not read apart; parts of a length (one without keys, too, where there are none)
template <typename Args> __host__ __device__ inline int paged_len(const Args& a, const PagedReq& r)
{
    const int g = prefix_of(r);
    return own_len_of(r) + (a.pooled || g < 0 ? 0 : (a.pool[g].len + 15) / 16 * 16);
}
__host__ __device__ inline int paged_parts(int len, int share) { return share == 0 || len <= share ? 1 : (len - 1) / share + 1; }
inline int log2_of(int n) { return 31 - __builtin_clz((unsigned)n); }
constexpr int up16(int n) { return (n + 15) / 16 * 16; }
constexpr int PAGED_FEW_ROWS = 16;       // of a tile
constexpr size_t paged_part_floats(int rows, int d) { return (size_t)rows * (d + 2); }
constexpr int paged_width(int head_dim) { return head_dim > 64 ? 128 : 64; }
hipError_t allow_paged();                // once on each device, before the first launch there
hipError_t launch_paged_few(const PagedArgs& a, bool bf16, int n_cu, hipStream_t s);     // tiles of 16 rows
hipError_t launch_paged_many(const PagedArgs& a, int height, hipStream_t s);    // of 64 or 128, two bytes
hipError_t launch_paged_join(const PagedArgs& a, bool bf16, hipStream_t s);     // rows of requests that have a prefix apart or parts, where their last part does not join them

}  // namespace tts
