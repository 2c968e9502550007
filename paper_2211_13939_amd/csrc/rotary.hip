// Rotary positions, alone and on the way into a paged cache: pairs of a head's columns turn by their row's position.
//
// Bound by memory: every element is read and written once.  A lane has the angles of its columns and takes them through several heads of its row, so that forming them costs
// little: an angle is position * frequency in turns, as 64-bit fixed point, of which the product's low bits are what is left of whole turns, exact
// for every position; of that the nearest quarter of a turn is a change of signs and places, and the rest, 1/8 of a turn at most, goes into the series of sine and cosine.
#include "past_kernels.h"
#include "mfma.h"

#include <algorithm>
#include <type_traits>

namespace tts {

namespace {

constexpr int WAVES = 4, AHEAD = 4;      // of a workgroup; heads whose loads are on their way together

template <typename T, int V> struct Words {
    static constexpr int BYTES = V * (int)sizeof(T), N = BYTES < 4 ? 1 : BYTES / 4;
    uint32_t w[N];
    __device__ __forceinline__ void load(const T* at)
    {
        if constexpr (BYTES == 2) w[0] = reinterpret_cast<const uint16_t*>(at)[0];
        else if constexpr (BYTES == 4) w[0] = reinterpret_cast<const uint32_t*>(at)[0];
        else if constexpr (BYTES == 8) *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(at);
        else
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) *reinterpret_cast<uint4*>(w + 4 * i) = reinterpret_cast<const uint4*>(at)[i];
    }
    __device__ __forceinline__ void store(T* at) const
    {
        if constexpr (BYTES == 2) reinterpret_cast<uint16_t*>(at)[0] = (uint16_t)w[0];
        else if constexpr (BYTES == 4) reinterpret_cast<uint32_t*>(at)[0] = w[0];
        else if constexpr (BYTES == 8) *reinterpret_cast<uint2*>(at) = *reinterpret_cast<const uint2*>(w);
        else
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) reinterpret_cast<uint4*>(at)[i] = *reinterpret_cast<const uint4*>(w + 4 * i);
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
    }
    __device__ __forceinline__ void set(const float* f)
    {
        if constexpr (sizeof(T) == 4)
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] = __float_as_uint(f[i]);
        else if constexpr (V == 1) w[0] = f2bf_bits(f[0]);
        else
#pragma unroll
            for (int i = 0; i < V; i += 2) w[i / 2] = pack_bf16x2(f[i], f[i + 1]);
    }
};

// Sine and cosine of `position` times a frequency (turns a position, times 2^64).
__device__ __forceinline__ void sine_cosine(int position, uint64_t freq, float& s, float& c)
{
    const uint32_t low = (uint32_t)freq, high = (uint32_t)(freq >> 32), p = (uint32_t)position;
    const uint32_t turns = __umulhi(p, low) + p * high - (position < 0 ? low : 0);       // times 2^32
    const uint32_t quarter = (turns + 0x20000000u) >> 30;
    const float a = (float)(int)(turns - (quarter << 30)) * 1.4629180792671596e-9f;      // 2 pi / 2^32; at most pi / 4
    const float q = a * a;
    // their series, whose first term left out is below 2^-28 here
    const float sn = __builtin_fmaf(a * q, __builtin_fmaf(q, __builtin_fmaf(q, __builtin_fmaf(q, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), a);
    const float cs = __builtin_fmaf(q, __builtin_fmaf(q, __builtin_fmaf(q, __builtin_fmaf(q, __builtin_fmaf(q, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const float x = quarter & 1 ? sn : cs, y = quarter & 1 ? cs : sn;
    c = __uint_as_float(__float_as_uint(x) ^ (quarter + 1 & 2) << 30);
    s = __uint_as_float(__float_as_uint(y) ^ (quarter & 2) << 30);
}

// A lane's unit of a head: its columns and their angles.  V: columns of a chunk.
template <int V, bool PAIRS> struct Unit {
    static constexpr int PAIRS_OF = V;
    int a, b;                            // first columns of the two chunks
    bool on[PAIRS ? V : 1];              // whether they turn
    float c[V], s[V];
    __device__ __forceinline__ Unit(const TurnAngles& t, int unit, int position, bool back, int head_dim)
    {
        const int turning = t.half / V;
        int first;                       // of the lane's pairs
        if constexpr (PAIRS) {
            a = 2 * V * unit;
            b = a + V;
            first = V * unit;
#pragma unroll
            for (int i = 0; i < V; ++i) on[i] = first + i < t.half;
        } else {
            on[0] = unit < turning;
            const int rest = 2 * t.half + 2 * V * (unit - turning);
            a = on[0] ? V * unit : rest;
            b = on[0] ? t.half + V * unit : rest + V < head_dim ? rest + V : rest;     // (a chunk that there is not: the first again)
            first = V * unit;
        }
        const float sign = back ? -t.magnitude : t.magnitude;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            sine_cosine(position, t.half ? t.freqs[min(first + i, t.half - 1)] : 0, s[i], c[i]);
            c[i] *= t.magnitude;
            s[i] *= sign;
        }
    }
    template <typename TX, typename TY> __device__ __forceinline__ void turn(const Words<TX, V>& xa, const Words<TX, V>& xb, Words<TY, V>& ya, Words<TY, V>& yb) const
    {
        float u[V], w[V];
        if constexpr (PAIRS) {
            float f[2 * V];
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = xa.get(i), f[V + i] = xb.get(i);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float p = f[2 * i], r = f[2 * i + 1];
                f[2 * i] = on[i] ? __builtin_fmaf(p, c[i], -(r * s[i])) : p;
                f[2 * i + 1] = on[i] ? __builtin_fmaf(r, c[i], p * s[i]) : r;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] = f[i], w[i] = f[V + i];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float p = xa.get(i), r = xb.get(i);
                u[i] = on[0] ? __builtin_fmaf(p, c[i], -(r * s[i])) : p;
                w[i] = on[0] ? __builtin_fmaf(r, c[i], p * s[i]) : r;
            }
        }
        ya.set(u);
        yb.set(w);
    }
};

// Head steps from .. to of a wave: `side` heads each, a lane's unit of one of them.
template <typename TX, typename TY, int V, bool PAIRS>
__device__ __forceinline__ void turn_heads(const TurnAngles& t, const TX* x, TY* y, int x_apart, int y_apart, int heads, int from, int to, int block, int position, bool back, int head_dim)
{
    const int lane = threadIdx.x & 63, in_side = t.units < 64 ? lane / t.units : 0, unit = t.units < 64 ? lane % t.units : 64 * block + lane;
    if (in_side >= t.side || unit >= t.units) return;
    const Unit<V, PAIRS> u(t, unit, position, back, head_dim);
    for (int at = from; at < to; at += AHEAD) {
        Words<TX, V> xa[AHEAD], xb[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const TX* from_head = x + (long long)min((at + i) * t.side + in_side, heads - 1) * x_apart;
            xa[i].load(from_head + u.a);
            xb[i].load(from_head + u.b);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int head = (at + i) * t.side + in_side;
            if (at + i >= to || head >= heads) break;
            Words<TY, V> ya, yb;
            u.turn(xa[i], xb[i], ya, yb);
            ya.store(y + (long long)head * y_apart + u.a);
            yb.store(y + (long long)head * y_apart + u.b);
        }
    }
}

template <typename TX, typename TY>
__device__ __forceinline__ void copy_heads(const TX* x, TY* y, int x_apart, int y_apart, int heads, int from, int to, int head_dim)
{
    const int lane = threadIdx.x & 63, units = head_dim / 8, side = 64 / units, in_side = lane / units, column = lane % units * 8;
    if (in_side >= side) return;
    for (int at = from; at < to; at += AHEAD) {
        Words<TX, 8> in[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) in[i].load(x + (long long)min((at + i) * side + in_side, heads - 1) * x_apart + column);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int head = (at + i) * side + in_side;
            if (at + i >= to || head >= heads) break;
            Words<TY, 8> out;
            if constexpr (std::is_same<TX, TY>::value) out = in[i];
            else {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = in[i].get(j);
                out.set(f);
            }
            out.store(y + (long long)head * y_apart + column);
        }
    }
}

template <typename TX, typename TY, int V, bool PAIRS> __global__ __launch_bounds__(64 * WAVES) void k_rotary(RotaryArgs p)
{
    const long long all = (long long)p.rows * p.jobs, waves = (long long)gridDim.x * WAVES;
    for (long long at = (long long)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); at < all; at += waves) {
        const int row = (int)(at / p.jobs), job = (int)(at - (long long)row * p.jobs), block = job % p.turn.blocks, from = job / p.turn.blocks * p.per;
        const int steps = (p.heads + p.turn.side - 1) / p.turn.side;
        const int position = p.positions ? p.positions[row] : p.first + row;
        turn_heads<TX, TY, V, PAIRS>(p.turn, static_cast<const TX*>(p.x) + row * p.x_stride, static_cast<TY*>(p.y) + row * p.y_stride, p.head_dim, p.head_dim, p.heads, from, min(from + p.per, steps),
                                     block, position, p.back, p.head_dim);
    }
}

// The request that row `row` of a launch is of.
template <typename Args> __device__ __forceinline__ int request_of_row(const Args& p, int row)
{
    const int lane = threadIdx.x & 63;
    int before = 0;
#pragma unroll
    for (int i = 0; i < Args::BATCH; i += 64) before += __popcll(__ballot(i + lane < p.n && p.req[min(i + lane, p.n - 1)].first <= row));
    return __builtin_amdgcn_readfirstlane(before) - 1;
}

template <typename TX, typename TY, int V, bool PAIRS, typename Args> __global__ __launch_bounds__(64 * WAVES) void k_append(Args p)
{
    const int jobs = p.k_jobs + p.v_jobs + p.q_jobs;
    const long long all = (long long)p.rows * jobs, waves = (long long)gridDim.x * WAVES;
    for (long long at = (long long)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); at < all; at += waves) {
        const int row = (int)(at / jobs);
        int job = (int)(at - (long long)row * jobs);
        const AppendReq r = p.req[request_of_row(p, row)];
        const int cache_row = r.row + (row - r.first), position = r.position + (row - r.first);
        if (job >= p.k_jobs + p.v_jobs) {
            job -= p.k_jobs + p.v_jobs;
            const int from = job / p.turn.blocks * p.per, steps = (p.heads + p.turn.side - 1) / p.turn.side;
            turn_heads<TX, TY, V, PAIRS>(p.turn, static_cast<const TX*>(p.q) + row * p.q_stride, static_cast<TY*>(p.q_out) + row * p.q_out_stride, p.head_dim, p.head_dim, p.heads, from,
                                         min(from + p.per, steps), job % p.turn.blocks, position, false, p.head_dim);
            continue;
        }
        const int page = p.table[(long long)r.table_row * p.table_cols + (cache_row >> p.page_shift)];
        if ((unsigned)page >= (unsigned)p.n_pages) continue;                                // (no page: the row is not kept)
        const int apart = p.head_dim << p.page_shift;
        const long long to = page * p.page_stride + (long long)(cache_row & ((1 << p.page_shift) - 1)) * p.head_dim;
        if (job < p.k_jobs) {
            const int from = job / p.turn.blocks * p.per, steps = (p.kv_heads + p.turn.side - 1) / p.turn.side;
            turn_heads<TX, TY, V, PAIRS>(p.turn, static_cast<const TX*>(p.k) + row * p.k_stride, static_cast<TY*>(p.k_pages) + to, p.head_dim, apart, p.kv_heads, from, min(from + p.per, steps),
                                         job % p.turn.blocks, position, false, p.head_dim);
        } else {
            const int from = (job - p.k_jobs) * p.per, side = 64 / (p.head_dim / 8), steps = (p.kv_heads + side - 1) / side;
            copy_heads(static_cast<const TX*>(p.v) + row * p.v_stride, static_cast<TY*>(p.v_pages) + to, p.head_dim, apart, p.kv_heads, from, min(from + p.per, steps), p.head_dim);
        }
    }
}

// Calls f with the types and the unit's form.
template <typename F> hipError_t with_types(bool x_bf16, bool y_bf16, F f)
{
    if (x_bf16) return y_bf16 ? f(bf16_t(), bf16_t()) : f(bf16_t(), float());
    return y_bf16 ? f(float(), bf16_t()) : f(float(), float());
}
template <typename F> hipError_t with_unit(const TurnAngles& t, F f)
{
    if (t.pairs) return f(std::integral_constant<int, 4>(), std::true_type());
    switch (t.width) {
    case 8: return f(std::integral_constant<int, 8>(), std::false_type());
    case 4: return f(std::integral_constant<int, 4>(), std::false_type());
    case 2: return f(std::integral_constant<int, 2>(), std::false_type());
    default: return f(std::integral_constant<int, 1>(), std::false_type());
    }
}

int steps_of(int heads, int side) { return (heads + side - 1) / side; }
unsigned grid_of(long long waves) { return (unsigned)std::min<long long>((waves + WAVES - 1) / WAVES, 1 << 20); }

}  // namespace

hipError_t launch_rotary(RotaryArgs& a, bool x_bf16, bool y_bf16, int n_cu, hipStream_t s)
{
    const int steps = steps_of(a.heads, a.turn.side);
    a.per = (long long)a.rows * steps * a.turn.blocks <= 16 * n_cu ? 1 : steps;
    a.jobs = (steps + a.per - 1) / a.per * a.turn.blocks;
    return with_types(x_bf16, y_bf16, [&](auto x, auto y) {
        return with_unit(a.turn, [&](auto width, auto pairs) {
            hipLaunchKernelGGL((k_rotary<decltype(x), decltype(y), decltype(width)::value, decltype(pairs)::value>), dim3(grid_of((long long)a.rows * a.jobs)), dim3(64 * WAVES), 0, s, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_append(AppendArgs& a, bool x_bf16, bool bf16, int n_cu, hipStream_t s)
{
    const int k_steps = steps_of(a.kv_heads, a.turn.side), q_steps = a.q ? steps_of(a.heads, a.turn.side) : 0, v_steps = steps_of(a.kv_heads, 64 / (a.head_dim / 8));
    a.per = (long long)a.rows * ((k_steps + q_steps) * a.turn.blocks + v_steps) <= 16 * n_cu ? 1 : AHEAD;
    a.k_jobs = (k_steps + a.per - 1) / a.per * a.turn.blocks;
    a.q_jobs = (q_steps + a.per - 1) / a.per * a.turn.blocks;
    a.v_jobs = (v_steps + a.per - 1) / a.per;
    const unsigned grid = grid_of((long long)a.rows * (a.k_jobs + a.q_jobs + a.v_jobs));
    return with_types(x_bf16, bf16, [&](auto x, auto y) {
        return with_unit(a.turn, [&](auto width, auto pairs) {
            auto launch = [&](const auto& args) {
                using Args = std::decay_t<decltype(args)>;
                hipLaunchKernelGGL((k_append<decltype(x), decltype(y), decltype(width)::value, decltype(pairs)::value, Args>), dim3(grid), dim3(64 * WAVES), 0, s, args);
                return hipGetLastError();
            };
            if (a.n > APPEND_SMALL) return launch(a);
            AppendArgsOf<APPEND_SMALL> small;
            static_cast<AppendCommon&>(small) = a;
            std::copy_n(a.req, a.n, small.req);
            return launch(small);
        });
    });
}

}  // namespace tts
