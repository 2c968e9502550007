// Host-visible launch wrappers of the kernels of a decoder block's own past (rotary.hip, paged.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tts {

// How heads are dealt to a wave's lanes: a unit is what a lane has of a head, two chunks of `width` columns.  Halves: chunks that lie rot_dim / 2 apart, then what does not turn in
// neighbouring ones; pairs: neighbouring chunks of 4.  Heads of `units` units lie `side` to a wave; of more than 64, in `blocks` of 64.
struct TurnShape {
    int width, units, side, blocks;
};
inline TurnShape turn_shape(int head_dim, int rot_dim, bool pairs)
{
    TurnShape s;
    if (pairs || rot_dim == 0) {
        s.width = pairs ? 4 : 8;
        s.units = (head_dim + 2 * s.width - 1) / (2 * s.width);
    } else {
        s.width = rot_dim / 2 % 8 == 0 ? 8 : rot_dim / 2 % 4 == 0 ? 4 : rot_dim / 2 % 2 == 0 ? 2 : 1;
        s.units = rot_dim / 2 / s.width + (head_dim - rot_dim + 2 * s.width - 1) / (2 * s.width);
    }
    s.side = s.units < 64 ? 64 / s.units : 1;
    s.blocks = (s.units + 63) / 64;
    return s;
}

struct TurnAngles {
    const uint64_t* freqs;               // turns a position, times 2^64
    float magnitude;
    int half, width, units, side, blocks;    // half: rot_dim / 2
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
};
template <int N> struct AppendArgsOf : AppendCommon {
    static constexpr int BATCH = N;
    AppendReq req[N];
};
using AppendArgs = AppendArgsOf<APPEND_BATCH>;
hipError_t launch_append(AppendArgs& a, bool x_bf16, bool bf16, int n_cu, hipStream_t s);

}  // namespace tts
