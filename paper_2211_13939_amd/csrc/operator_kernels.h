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
// A launch of `tiles` workgroups, which eight XCDs are dealt in turn: an XCD takes a run of tiles.  A side of a grid has fewer than 2^32 threads, so that large calls' lie on two, rows of
// them a multiple of eight wide.  (Some workgroups are left over: linear8_tile is `tiles` or more for them.)
struct Linear8Grid { int across, down; };
inline Linear8Grid linear8_grid(int tiles)
{
    const int wgs = (tiles + 7) / 8 * 8, down = (wgs - 1) / (1 << 20) + 1;
    return {((wgs + down - 1) / down + 7) / 8 * 8, down};
}
__host__ __device__ inline int linear8_tile(int wg, int tiles)
{
    const int per = (tiles + 7) / 8, at = wg >> 3;
    return at < per ? (wg & 7) * per + at : tiles;
}

struct Linear8Args {
    const uint8_t *x8, *sx;              // [rows][width8], [rows][scale_columns]
    const uint4* w;                      // [units][halves of blocks][2][64 lanes] 16 bytes: the c-th of lane l holds row l % 32 of the unit, columns 32 * (l / 32) + 16 * c ..
    const uint32_t* sw;                  // [units][words of scales][32 rows]
    const float* bias;                   // [32 * units], zeros where there is none
    void* y;
    long long y_stride;
    int rows, out_dim, blocks;           // blocks: of 128 columns
};
// The kernel that a call takes; tiles: channels x rows of a workgroup.
enum class Linear8Form { FEW, SPLIT, TILE_64_64, TILE_64_128, TILE_128_128, TILE_256_128 };
inline Linear8Form linear8_form(int rows, int out_dim, int blocks, bool two_bytes, int n_cu)
{
    const int units = channel_units(out_dim);
    // A few rows: memory's rate is what counts (8192 x 8192 weights 11.6 us, 5.8 TB/s).  Up to 16 of them the plain loads of x still cost less than
    // a ring, unless the weights are many (16 rows, k_linear8_few / k_linear8_split: 1024 x 1024 2.8 / 3.2 us, 4096 x 4096 5.7 / 5.2, 8192 x 8192 15.7 /
    // 12.3; 8 rows of 4096 x 4096 4.5 / 5.0).
    if (rows <= 8 || (rows <= 16 && units * blocks <= 2048)) return Linear8Form::FEW;
    // Otherwise tiles: a larger one asks for fewer bytes, a smaller one has its latencies spread over more workgroups.  us, two-byte results, 32 x 32 split / 64 x 64 / 64
    // channels x 128 rows / 128 x 128 / 256 x 128: 200 x 2048 x 2048 5.7 / 6.6 / 8.3 / 12.3 / 20.6; 512 x 2048 x 2048 10.0 / 6.9 / 8.4 / 12.5 / 20.7; 1024 x 2048 x 2048 17.0 / 8.4 /
    // 9.2 / 12.5 / 20.9; 1542 x 2048 x 2048 - / 15.6 / 11.5 / 13.6 / 21.2; 3500 x 2048 x 2048 - / 25.7 / 25.6 / 19.5 / 22.9; 8000 x 1024 x 1024 - / 16.3 / 15.1 / 13.1 / 16.0; 16384 x
    // 1024 x 1024 - / 33.0 / 27.1 / 27.4 / 24.9; 16384 x 4096 x 4096 - / 427 / 358 / 278 / 251.  (Measured up to 4096 channels and columns; wider calls follow the same counts of tiles.)
    auto tiles = [&](int n, int m) { return (long long)((units + n - 1) / n) * ((rows + 32 * m - 1) / (32 * m)); };
    const int two = 2 * n_cu;
    if (tiles(1, 1) <= two) return Linear8Form::SPLIT;
    // (few columns: a workgroup is its first loads and its results, of which more, smaller ones have more at once.  64 x 128 rows against the largest: 16384 x 512 x 2048 32.0 /
    // 35.5 us, 4096 x 256 x 1024 5.2 / 6.5; 16384 x 640 x 2048 38.6 / 34.9.)
    if (blocks <= 4 && tiles(2, 4) >= two) return Linear8Form::TILE_64_128;
    if (two_bytes) {
        // The smallest that goes round once with two workgroups a compute unit: what comes in a second round costs a whole one.
        if (tiles(2, 2) <= two) return Linear8Form::TILE_64_64;
        if (tiles(2, 4) <= two) return Linear8Form::TILE_64_128;
        if (tiles(4, 4) <= two) return Linear8Form::TILE_128_128;
        return Linear8Form::TILE_256_128;
    }
    // Operands' way to bf16 keeps the vector pipes busy, and several workgroups a compute unit even out.  The largest that leaves two of them: us, 64 x 64 / 64 x 128 / 128 x
    // 128 / 256 x 128: 1280 x 2048 x 2048 17.5 / 18.6 / 19.9 / 33.7, 3000 x 2048 x 2048 32.9 / 30.5 / 31.9 / 35.4, 3000 x 4096 x 4096 115 / 102 / 94 / 102, 16384 x 4096 x
    // 4096 657 / 550 / - / 460.  (64 x 64 with two steps in LDS, four workgroups a compute unit: 1542 x 2048 x 2048 23.8 -> 21.7.)
    if (tiles(8, 4) >= two) return Linear8Form::TILE_256_128;
    if (tiles(4, 4) >= two) return Linear8Form::TILE_128_128;
    if (tiles(2, 4) >= two) return Linear8Form::TILE_64_128;
    return Linear8Form::TILE_64_64;
}
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
// 256 rows a workgroup where memories are long and it leaves some for most compute units, 128 otherwise.  us, 128 / 256: 8 requests of 3000 queries over
// 3000 keys, 16 heads of 64 356 / 325, 16 of 128 that share 4 620 / 560; one of 4000 over 4000 (252 workgroups) 143 / 134, of 1000 over 1000 24 / 31;
// 64 of 600 over 135 33 / 35.
inline bool cross_many_large(const CrossReq* req, int n, int group, int n_kv_heads, int n_cu)
{
    long long large = 0;
    int longest = 0;
    for (int i = 0; i < n; ++i) {
        large += ((long long)req[i].q_len * group + 255) / 256 * n_kv_heads;
        longest = req[i].mem_len > longest ? req[i].mem_len : longest;
    }
    return longest >= 1024 && large >= n_cu - n_cu / 4;
}

}  // namespace tts
