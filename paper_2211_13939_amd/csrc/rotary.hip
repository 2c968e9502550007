// Rotary positions, alone and on the way into a paged cache: pairs of a head's columns turn by their row's position.
//
// Bound by memory: every element is read and written once.  A lane has the angles of its columns and takes them through several heads of its row, so that forming them costs
// little: an angle is position * frequency in turns, as 64-bit fixed point, of which the product's low bits are what is left of whole turns, exact
// for every position; of that the nearest quarter of a turn is a change of signs and places, and the rest, 1/8 of a turn at most, goes into the series of sine and cosine.
//
// Measured: 16384 rows of 40 heads of 128 in bf16 take what memory does (64 us, 5.3 TB/s), 16000 rows on their way into a cache with their queries 86 us (5.0 TB/s); small calls a launch and the trips that
// depend on each other (one row 2.7 us; 64 requests' rows 3.8: arguments, table, store, with rows and angles asked for meanwhile).  What a lane takes through registers are vectors: pieces copied as structs went
// through scratch memory, or were copied when they were stored (64 rows 8.0 us, 16000 101).  A head whose turning columns are no multiple of 16 has its last pieces overlap (of 26 columns of 96: single
// columns took 20 us for 2778 rows of 4 heads, pieces of 8 columns 12.7).  Far from memory's rate: few heads of few columns, where a wave's lanes are not all used (one head of k and v: 10 of 64).
#include "past_kernels.h"
#include "mfma.h"

#include <algorithm>
#include <type_traits>

namespace tts {

namespace {

constexpr int WAVES = 4, AHEAD = 4;      // of a workgroup; heads whose loads are on their way together

// V columns of a head from any on: an address is aligned to an element (the hardware takes wide accesses at any).
template <typename T, int V> struct Words {
    static constexpr int BYTES = V * (int)sizeof(T), N = BYTES < 4 ? 1 : BYTES / 4, PIECE = BYTES < 16 ? N : 4;
    typedef uint32_t Piece __attribute__((ext_vector_type(PIECE)));
    typedef Piece Anywhere __attribute__((aligned(sizeof(T))));
    uint32_t w[N];
    __device__ __forceinline__ void load(const T* at)
    {
        if constexpr (BYTES == 2) w[0] = reinterpret_cast<const uint16_t*>(at)[0];
        else
#pragma unroll
            for (int i = 0; i < N / PIECE; ++i) {
                const Piece x = reinterpret_cast<const Anywhere*>(at)[i];
#pragma unroll
                for (int j = 0; j < PIECE; ++j) w[PIECE * i + j] = x[j];
            }
    }
    __device__ __forceinline__ void store(T* at) const
    {
        if constexpr (BYTES == 2) reinterpret_cast<uint16_t*>(at)[0] = (uint16_t)w[0];
        else
#pragma unroll
            for (int i = 0; i < N / PIECE; ++i) {
                Piece x;
#pragma unroll
                for (int j = 0; j < PIECE; ++j) x[j] = w[PIECE * i + j];
                reinterpret_cast<Anywhere*>(at)[i] = x;
            }
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
    int a, b, first;                     // first columns of the two chunks; the first of the lane's pairs
    bool on[PAIRS ? V : 1];              // whether they turn
    float c[V], s[V];
    __device__ __forceinline__ Unit(const TurnAngles& t, int unit, int head_dim)
    {
        const int turning = (t.half + V - 1) / V;
        if constexpr (PAIRS) {
            a = 2 * V * unit;
            b = a + V;
            first = V * unit;
#pragma unroll
            for (int i = 0; i < V; ++i) on[i] = first + i < t.half;
        } else {
            on[0] = unit < turning;
            first = min(V * unit, t.half - V);
            const int rest = 2 * t.half + 2 * V * (unit - turning);
            a = on[0] ? first : min(rest, head_dim - V);
            b = on[0] ? t.half + first : min(rest + V, head_dim - V);
        }
    }
    __device__ __forceinline__ void angles(const TurnAngles& t, int position, bool back)
    {
        const float sign = back ? -t.magnitude : t.magnitude;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            sine_cosine(position, t.half ? t.freqs[max(0, min(first + i, t.half - 1))] : 0, s[i], c[i]);
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

// Where a wave's rows go, and at which position they are; y null: nowhere.
template <typename TY> struct To { TY* y; int position; };
// Head steps from .. to of a wave: `side` heads each, a lane's unit of one of them.  `where` says where they go, when the first are on their way: a new row's page takes two trips to memory.
template <typename TX, typename TY, int V, bool PAIRS, typename Where>
__device__ __forceinline__ void turn_heads(const TurnAngles& t, const TX* x, int x_apart, int y_apart, int heads, int from, int to, int block, bool back, int head_dim, Where where)
{
    const int lane = threadIdx.x & 63, in_side = over(lane, t.by_units), unit = t.units < 64 ? lane - in_side * t.units : 64 * block + lane;
    if (in_side >= t.side || unit >= t.units) return;
    Unit<V, PAIRS> u(t, unit, head_dim);
    TY* y = nullptr;
    for (int at = from; at < to; at += AHEAD) {
        Words<TX, V> xa[AHEAD], xb[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const TX* from_head = x + (long long)min((at + i) * t.side + in_side, heads - 1) * x_apart;
            xa[i].load(from_head + u.a);
            xb[i].load(from_head + u.b);
        }
        if (at == from) {
            const To<TY> place = where();
            if (!place.y) return;
            y = place.y;
            u.angles(t, place.position, back);
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

template <typename TX, typename TY, typename Where>
__device__ __forceinline__ void copy_heads(const TX* x, int x_apart, int y_apart, int heads, int from, int to, int head_dim, unsigned by_units, Where where)
{
    const int lane = threadIdx.x & 63, units = head_dim / 8, in_side = over(lane, by_units), column = (lane - in_side * units) * 8, side = over(64, by_units);
    if (in_side >= side) return;
    TY* y = nullptr;
    for (int at = from; at < to; at += AHEAD) {
        Words<TX, 8> in[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) in[i].load(x + (long long)min((at + i) * side + in_side, heads - 1) * x_apart + column);
        if (at == from) {
            y = where().y;
            if (!y) return;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int head = (at + i) * side + in_side;
            if (at + i >= to || head >= heads) break;
            if constexpr (std::is_same<TX, TY>::value) in[i].store(y + (long long)head * y_apart + column);
            else {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = in[i].get(j);
                Words<TY, 8> out;
                out.set(f);
                out.store(y + (long long)head * y_apart + column);
            }
        }
    }
}

// (a row's waves, `blocks` of them over the same heads)
__device__ __forceinline__ int row_of(long long at, int jobs, unsigned by) { return by != NOT_BY ? over((int)at, by) : (int)(at / jobs); }
__device__ __forceinline__ int from_of(int job, int blocks) { return blocks == 1 ? job : job / blocks; }

template <typename TX, typename TY, int V, bool PAIRS> __global__ __launch_bounds__(64 * WAVES) void k_rotary(RotaryArgs p)
{
    const long long all = (long long)p.rows * p.jobs, waves = (long long)gridDim.x * WAVES;
    for (long long at = (long long)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); at < all; at += waves) {
        const int row = row_of(at, p.jobs, p.by_jobs), job = (int)(at - (long long)row * p.jobs), step = from_of(job, p.turn.blocks), from = step * p.per;
        const int steps = (p.heads + p.turn.side - 1) / p.turn.side;
        turn_heads<TX, TY, V, PAIRS>(p.turn, static_cast<const TX*>(p.x) + row * p.x_stride, p.head_dim, p.head_dim, p.heads, from, min(from + p.per, steps), job - step * p.turn.blocks, p.back,
                                     p.head_dim, [&] { return To<TY>{static_cast<TY*>(p.y) + row * p.y_stride, p.positions ? p.positions[row] : p.first + row}; });
    }
}

// The request that row `row` of a launch is of.  (One trip to the arguments, which are far.)
template <typename Args> __device__ __forceinline__ AppendReq request_of_row(const Args& p, int row)
{
    if (p.each) return p.req[over(row, p.by_each)];
    const int lane = threadIdx.x & 63;
    AppendReq mine[(Args::BATCH + 63) / 64];
    int before = 0;
#pragma unroll
    for (int i = 0; i < Args::BATCH; i += 64) mine[i / 64] = p.req[min(i + lane, p.n - 1)];
#pragma unroll
    for (int i = 0; i < Args::BATCH; i += 64) before += __popcll(__ballot(i + lane < p.n && mine[i / 64].first <= row));
    const int at = __builtin_amdgcn_readfirstlane(before) - 1;
    AppendReq r = {};
#pragma unroll
    for (int i = 0; i < Args::BATCH; i += 64)
        if (at >> 6 == i / 64) {
            const AppendReq& m = mine[i / 64];
            r = {__builtin_amdgcn_readlane(m.first, at & 63), __builtin_amdgcn_readlane(m.row, at & 63), __builtin_amdgcn_readlane(m.table_row, at & 63), __builtin_amdgcn_readlane(m.position, at & 63)};
        }
    return r;
}

template <typename TX, typename TY, int V, bool PAIRS, typename Args> __global__ __launch_bounds__(64 * WAVES) void k_append(Args p)
{
    const int jobs = p.k_jobs + p.v_jobs + p.q_jobs;
    const long long all = (long long)p.rows * jobs, waves = (long long)gridDim.x * WAVES;
    for (long long at = (long long)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); at < all; at += waves) {
        const int row = row_of(at, jobs, p.by_jobs);
        int job = (int)(at - (long long)row * jobs);
        const AppendReq r = request_of_row(p, row);
        const int position = r.position + (row - r.first), apart = p.head_dim << p.page_shift;
        auto in_page = [&](void* pages) {
            const int cache_row = r.row + (row - r.first), page = p.table[(long long)r.table_row * p.table_cols + (cache_row >> p.page_shift)];
            // (no page: the row is not kept)
            TY* y = (unsigned)page < (unsigned)p.n_pages ? static_cast<TY*>(pages) + page * p.page_stride + (long long)(cache_row & ((1 << p.page_shift) - 1)) * p.head_dim : nullptr;
            return To<TY>{y, position};
        };
        if (job < p.k_jobs) {
            const int step = from_of(job, p.turn.blocks), from = step * p.per, steps = (p.kv_heads + p.turn.side - 1) / p.turn.side;
            turn_heads<TX, TY, V, PAIRS>(p.turn, static_cast<const TX*>(p.k) + row * p.k_stride, p.head_dim, apart, p.kv_heads, from, min(from + p.per, steps), job - step * p.turn.blocks, false,
                                         p.head_dim, [&] { return in_page(p.k_pages); });
            continue;
        }
        job -= p.k_jobs;
        if (job < p.v_jobs) {
            const int from = job * p.per, side = over(64, p.by_v), steps = (p.kv_heads + side - 1) / side;
            copy_heads<TX, TY>(static_cast<const TX*>(p.v) + row * p.v_stride, p.head_dim, apart, p.kv_heads, from, min(from + p.per, steps), p.head_dim, p.by_v, [&] { return in_page(p.v_pages); });
            continue;
        }
        job -= p.v_jobs;
        const int step = from_of(job, p.turn.blocks), from = step * p.per, steps = (p.heads + p.turn.side - 1) / p.turn.side;
        turn_heads<TX, TY, V, PAIRS>(p.turn, static_cast<const TX*>(p.q) + row * p.q_stride, p.head_dim, p.head_dim, p.heads, from, min(from + p.per, steps), job - step * p.turn.blocks, false,
                                     p.head_dim, [&] { return To<TY>{static_cast<TY*>(p.q_out) + row * p.q_out_stride, position}; });
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

unsigned by_jobs_of(long long rows, int jobs) { return rows * jobs * jobs <= 1LL << 32 ? by_of((unsigned)jobs) : NOT_BY; }
int steps_of(int heads, int side) { return (heads + side - 1) / side; }
unsigned grid_of(long long waves) { return (unsigned)std::min<long long>((waves + WAVES - 1) / WAVES, 1 << 20); }

}  // namespace

hipError_t launch_rotary(RotaryArgs& a, bool x_bf16, bool y_bf16, int n_cu, hipStream_t s)
{
    const int steps = steps_of(a.heads, a.turn.side);
    a.per = (long long)a.rows * steps * a.turn.blocks <= 16 * n_cu ? 1 : steps;
    a.jobs = (steps + a.per - 1) / a.per * a.turn.blocks;
    a.by_jobs = by_jobs_of(a.rows, a.jobs);
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
    a.by_v = by_of((unsigned)a.head_dim / 8);
    a.by_jobs = by_jobs_of(a.rows, a.k_jobs + a.q_jobs + a.v_jobs);
    a.each = a.n > 1 ? a.req[1].first : a.rows;
    for (int i = 0; i < a.n; ++i)
        if (a.each && (a.req[i].first != (long long)i * a.each || a.rows != (long long)a.n * a.each)) a.each = 0;
    if ((long long)a.rows * a.each > 1LL << 32) a.each = 0;
    a.by_each = by_of((unsigned)a.each);
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
