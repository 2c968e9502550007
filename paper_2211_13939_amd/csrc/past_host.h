// What the host code of a decoder block's own past (rotary.cpp, cache.cpp, paged.cpp) has in common: angles, and the checks of strides and of a cache.
#pragma once
#include <cmath>
#include <vector>

#include "../../include/tts_rotary.h"
#include "operator_host.h"
#include "past_kernels.h"

namespace tts {

inline int check_angles(const tts_rotary_angles& a, int head_dim)
{
    if (a.rot_dim < 2 || a.rot_dim > head_dim || a.rot_dim % 2) return fail(TTS_E_INVAL, "rot_dim must be even, in 2..head_dim");
    if (a.layout != TTS_ROTARY_HALF && a.layout != TTS_ROTARY_PAIRS) return fail(TTS_E_INVAL, "layout must be 0 (halves) or 1 (pairs)");
    if (a.scaling < TTS_ROTARY_PLAIN || a.scaling > TTS_ROTARY_PARTS) return fail(TTS_E_INVAL, "scaling must be in 0..3");
    if (!(a.base >= 1 && a.base <= 0x1p60)) return fail(TTS_E_INVAL, "base must be in 1..2^60");
    if (!(a.magnitude >= 0x1p-60 && a.magnitude <= 0x1p60)) return fail(TTS_E_INVAL, "magnitude must be in 2^-60..2^60");
    if (a.scaling != TTS_ROTARY_PLAIN && !(a.factor >= 1 && a.factor <= 0x1p30)) return fail(TTS_E_INVAL, "factor must be in 1..2^30");
    if (a.scaling == TTS_ROTARY_BASE && a.rot_dim < 4) return fail(TTS_E_INVAL, "a base can be scaled for rot_dim from 4 on");
    if (a.scaling == TTS_ROTARY_PARTS && !(a.trained_len >= 1 && a.low >= 0 && a.low < a.high && a.high <= 0x1p30))
        return fail(TTS_E_INVAL, "parts: trained_len from 1 on and 0 <= low < high <= 2^30 are wanted");
    return TTS_OK;
}

// Turns a position of each pair, times 2^64 (a frequency is 1 radian at most).
inline std::vector<uint64_t> turn_freqs(const tts_rotary_angles& a)
{
    constexpr long double TWO_PI = 6.283185307179586476925286766559L;
    std::vector<uint64_t> v(a.rot_dim / 2);
    long double base = a.base;
    if (a.scaling == TTS_ROTARY_BASE) base *= powl(a.factor, (long double)a.rot_dim / (a.rot_dim - 2));
    for (size_t i = 0; i < v.size(); ++i) {
        long double f = powl(base, -2.0L * (long double)i / a.rot_dim);
        if (a.scaling == TTS_ROTARY_LINEAR) f /= a.factor;
        if (a.scaling == TTS_ROTARY_PARTS) {
            long double g = (a.trained_len * f / TWO_PI - a.low) / ((long double)a.high - a.low);
            g = g < 0 ? 0 : g > 1 ? 1 : g;
            f *= g + (1 - g) / a.factor;
        }
        v[i] = (uint64_t)(f / TWO_PI * 0x1p64L + 0.5L);
    }
    return v;
}

inline TurnAngles turn_angles(const tts_rotary_angles& a, int head_dim, const uint64_t* freqs)
{
    const bool pairs = a.rot_dim && a.layout == TTS_ROTARY_PAIRS;
    const TurnShape s = turn_shape(head_dim, a.rot_dim, pairs);
    return {freqs, (float)a.magnitude, a.rot_dim / 2, s.width, s.units, s.side, s.blocks, by_of((unsigned)s.units), pairs};
}

// Rows of `width` elements, `stride` apart (0: back to back).
inline int check_rows(const char* name, const void* at, long long width, long long& stride)
{
    if (!stride) stride = width;
    if (stride < width || stride > (1LL << 40) || stride % 8) return fail(TTS_E_INVAL, "%s: a stride of %lld for %lld columns", name, stride, width);
    if (!aligned(at, 16)) return fail(TTS_E_INVAL, "%s must be 16-byte aligned", name);
    return TTS_OK;
}

inline bool is_page_rows(int n, int least, int most) { return n >= least && n <= most && (n & (n - 1)) == 0; }

}  // namespace tts
