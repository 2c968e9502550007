// Host-visible launch wrappers of the operators' kernels (norm.hip, linear8.hip, cross.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tts {

constexpr int E8_BLOCK = 128;            // columns of an 8-bit row under one scale
constexpr int width8(int dim) { return (dim + E8_BLOCK - 1) / E8_BLOCK * E8_BLOCK; }
constexpr int scale_columns(int dim) { return (width8(dim) / E8_BLOCK + 3) / 4 * 4; }

struct NormArgs {
    const void *x, *res;                 // res: null if there is none
    void *total, *y;                     // null: not wanted
    uint8_t *y8, *scales;                // null: not wanted
    const float* gain;                   // null: no norm
    long long x_stride, res_stride, total_stride, y_stride;    // elements
    int rows, dim;
    float eps;
    bool y_bf16;
};
hipError_t launch_norm(const NormArgs& a, bool x_bf16, bool res_bf16, int n_cu, hipStream_t s);

// Channels lie in pairs of units of 32: row 8 a + 4 h + j of the t-th is channel 32 h + 16 t + 4 a + j of the 64.
constexpr int channel_units(int channels) { return (channels + 63) / 64 * 2; }
constexpr int channel_unit(int n) { return n / 64 * 2 + n / 16 % 2; }
constexpr int channel_row(int n) { return n / 4 % 4 * 8 + n / 32 % 2 * 4 + n % 4; }
struct Linear8Args {
    const uint8_t *x8, *sx;              // [rows][width8], [rows][scale_columns]
    const uint4* w;                      // [units][halves of blocks][2][64 lanes] 16 bytes: the c-th of lane l holds row l % 32 of the unit, columns 32 * (l / 32) + 16 * c ..
    const uint32_t* sw;                  // [units][words of scales][32 rows]
    const float* bias;                   // [32 * units], zeros where there is none
    void* y;
    long long y_stride;
    int rows, out_dim, blocks;           // blocks: of 128 columns
};
hipError_t allow_linear8();              // once on each device, before the first launch there
hipError_t launch_linear8(const Linear8Args& a, bool y_bf16, int n_cu, hipStream_t s);

constexpr int CROSS_BATCH = 128;         // requests of a launch
struct CrossReq {
    long long mem_row;
    int mem_len, q_row, q_len;
    int first;                           // of its row tiles, of all key heads and as often as its memory has parts, in the launch
};
struct CrossCommon {
    const void *q, *k, *v;
    void* out;
    const uint8_t* keep;
    const void* zeros;                   // 16 bytes and more
    float *lse, *parts;
    long long q_stride, k_stride, v_stride, out_stride;        // elements
    float scale;                         // times log2(e)
    int n_heads, n_kv_heads, head_dim;
    int n;
    bool single, runs;                   // few rows: every request has one row tile, and no parts; an XCD takes a run of the tiles
    int items, share;                    // few rows: tiles, and the length of a part, 0: there are none
    int start[9];                        // many rows: first of the row tiles that each XCD takes
};
template <int N> struct CrossArgsOf : CrossCommon {
    static constexpr int BATCH = N;
    CrossReq req[N];
    int row[N];                          // few rows: first of each request's rows (query, head) in the launch, where there are parts
};
using CrossArgs = CrossArgsOf<CROSS_BATCH>;
// Small batches of few rows take small arguments: what a launch carries costs the host (a request's step from Python 6.8 us with 3.7 KB, 5.6 with 0.6).
constexpr int CROSS_SMALL = 16;
size_t cross_parts_bytes();
hipError_t allow_cross();                // once on each device, before the first launch there
// `few`: 16 rows a workgroup, both types; `many`: 128 or 256, two bytes alone.  They fill in what the launch's tiles are.
hipError_t launch_cross_few(CrossArgs& a, bool bf16, int n_cu, hipStream_t s);
hipError_t launch_cross_many(CrossArgs& a, int n_cu, hipStream_t s);
// A request is the latter's from two of the former's row tiles up, if the call has two and a half of those for every compute unit.  us, few / many: 16
// requests, 8 heads of 64, 135 keys: 64 queries each (512 tiles) 5.4 / 6.5, 96 (768) 6.9 / 7.0, 192 (1536) 11.7 / 7.4; one of 1000 over 1000 keys (504) 20.7 /
// 19.4, with 16 heads of 128 that share 4 (1000) 41 / 24; 32 requests of 40 queries over 300, 8 heads that share one (640) 9.2 / 8.8.
constexpr int CROSS_MANY_ROWS = 33;
constexpr int CROSS_MAX_TILES = 1 << 23;     // a grid has fewer than 2^32 threads, and XCDs' shares of the tiles may be of different heights
inline bool cross_many(long long few_tiles, int n_cu) { return 2 * few_tiles >= 5LL * n_cu; }

}  // namespace tts
