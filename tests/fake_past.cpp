// The HIP calls and launch wrappers of fake_operators.cpp, and those of a decoder block's own past: what a call would have launched is written down.
#include "fake_operators.cpp"

#include "../paper_2211_13939_amd/csrc/past_kernels.h"

namespace {
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
}  // namespace tts

extern "C" {
void past_reset() { fake_reset(); append_rows = 0; }
int past_append_rows() { return append_rows; }
long long past_append_k() { return (long long)(size_t)append.k; }
int past_append_first(int i) { return append.req[i].first; }
int past_append_position(int i) { return append.req[i].position; }
int past_rotary_first() { return rotary.first; }
}
