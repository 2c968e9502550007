// Cross attention: every query row of a request attends the request's memory, o = softmax(scale * q k^T) v, several query heads to a head of
// k and v.  One pass over the memory with the softmax's running maximum and sum; rows of a request and a key head are its
// (query, head of the group) pairs, 16 to a tile, so that heads which share keys share their loads too.
//
// Scores are formed transposed, keys as the matrix instruction's rows: a lane then holds four neighbouring keys of ONE query row, and so
// do its exponentials, which are the second product's operand (values as rows, query rows as columns) without leaving their registers.  The second product
// sums over keys in whatever order both operands share.
#include "operator_kernels.h"
#include "mfma.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace tts {

namespace {

constexpr int FEW_WAVES = 4;
constexpr int MAX_PARTS = 2048, MAX_SPLITS = 256;    // parts of one launch, of one row tile
constexpr int part_floats(int d) { return 16 * (d + 2); }

// of the four lanes that share l % 16
__device__ __forceinline__ float across_max(float x)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float across_sum(float x)
{
    x += __shfl_xor(x, 16, 64);
    return x + __shfl_xor(x, 32, 64);
}

// A step's keys of a wave.  Lane l, group g = l / 16.  First operand: rows of keys, the lane's is key l % 16 of each 16; second: of the keys that
// the lane holds scores of, 4 g .. 4 g + 3 of each 16, the D / 16 columns from (D / 16) * (l % 16) on.  Row i of the second product's tile
// e is then column (D / 16) * i + e of the head.
// FULL: heads are D wide.  Of narrower ones the first operand's missing columns are zeros; the second's are any (nobody stores what comes of them).
template <typename T, int D> struct Geometry {
    static constexpr int PER_LANE = sizeof(T) == 2 ? 8 : 4, N = 4 * PER_LANE, TILES = N / 16;       // scores of a lane, keys of a step
    static constexpr int EPL = 16 / sizeof(T), NF = D / (4 * EPL), NE = D / 16;                      // elements of 16 bytes, loads of a key, columns of a lane
    static __device__ __forceinline__ int key(int i, int g) { return 16 * (i / 4) + 4 * g + (i & 3); }      // of the lane's i-th score
};

// Where a lane's parts of a step lie, in bytes from the step's first key
template <typename T, int D> struct Places {
    using G = Geometry<T, D>;
    uint32_t k[G::TILES], v[G::PER_LANE], k_column, v_column;
    __device__ __forceinline__ Places(long long ks, long long vs, int head_dim, int lane)
    {
        const int g = lane >> 4, c = lane & 15;
        k_column = 16 * g;
        v_column = G::NE * c < head_dim ? (uint32_t)sizeof(T) * G::NE * c : 0;
#pragma unroll
        for (int t = 0; t < G::TILES; ++t) k[t] = (16 * t + c) * (uint32_t)ks * (uint32_t)sizeof(T) + k_column;
#pragma unroll
        for (int i = 0; i < G::PER_LANE; ++i) v[i] = G::key(i, g) * (uint32_t)vs * (uint32_t)sizeof(T) + v_column;
    }
};

template <typename T, int D, bool FULL, bool MASK> struct Keys {
    using G = Geometry<T, D>;
    uint8_t seen[G::PER_LANE];
    uint4 k[G::TILES][G::NF];
    uint32_t v[G::PER_LANE][G::NE * sizeof(T) / 4];
    // kp, vp, keep: the step's first key; last: the last of its keys that there is, counted from 0, k_last, v_last: where that lies (keys behind it are
    // loaded from there)
    __device__ __forceinline__ void load(const char* kp, const char* vp, const uint8_t* keep, const Places<T, D>& at, int last, uint32_t k_last, uint32_t v_last, int head_dim, int lane)
    {
        if constexpr (MASK)
#pragma unroll
            for (int i = 0; i < G::PER_LANE; ++i) seen[i] = keep[(uint32_t)min(G::key(i, lane >> 4), last)];
        k_last += at.k_column;
        v_last += at.v_column;
#pragma unroll
        for (int t = 0; t < G::TILES; ++t) {
            const uint32_t from = min(at.k[t], k_last);
#pragma unroll
            for (int f = 0; f < G::NF; ++f) {
                if constexpr (FULL) k[t][f] = *reinterpret_cast<const uint4*>(kp + from + 64 * f);
                else {
                    const bool there = (4 * f + (lane >> 4)) * G::EPL < head_dim;
                    const uint4 x = *reinterpret_cast<const uint4*>(kp + (there ? from + 64 * f : from - at.k_column));
                    k[t][f] = there ? x : make_uint4(0, 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < G::PER_LANE; ++i) {
            const uint32_t from = min(at.v[i], v_last);
            if constexpr (G::NE * sizeof(T) == 8) *reinterpret_cast<uint2*>(v[i]) = *reinterpret_cast<const uint2*>(vp + from);
            else
#pragma unroll
                for (size_t b = 0; b < G::NE * sizeof(T); b += 16) *reinterpret_cast<uint4*>(v[i] + b / 4) = *reinterpret_cast<const uint4*>(vp + from + b);
        }
        // (left alone, the compiler puts them in front of their use: 26 requests of 2185 .. 2925 keys, 8 fp32 heads of 128, 171 in place of 101 us)
        if constexpr (MASK) __builtin_amdgcn_sched_barrier(0);
    }
    __device__ __forceinline__ void scores(const uint4 (&q)[G::NF], float* s) const
    {
#pragma unroll
        for (int t = 0; t < G::TILES; ++t) {
            floatx4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int f = 0; f < G::NF; ++f) a = mfma_frag<T>(k[t][f], q[f], a);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[4 * t + j] = a[j];
        }
    }
    __device__ __forceinline__ void add(const float* w, floatx4* o) const
    {
        if constexpr (sizeof(T) == 2) {
            // (weights to bf16, the values' type: each off by up to 2^-8 of itself, so that the result is by no more than that before its own rounding, which is as large; two
            // products, of their upper and lower halves, would keep them at twice the matrix instructions)
            const uint4 b = make_uint4(pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7]));
#pragma unroll
            for (int e = 0; e < G::NE; ++e) {
                const uint32_t half = e & 1 ? 0x07060302u : 0x05040100u;     // the upper or lower halves of two words
                uint32_t a[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(v[2 * i + 1][e / 2], v[2 * i][e / 2], half);
                o[e] = mfma_frag<bf16_t>(make_uint4(a[0], a[1], a[2], a[3]), b, o[e]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < G::PER_LANE; ++i)
#pragma unroll
                for (int e = 0; e < G::NE; ++e) o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][e]), w[i], o[e], 0, 0, 0);
        }
    }
};

// The running softmax of a lane's query row: maximum (of all keys so far), sum (of the lane's own keys), the outputs' columns.
template <typename T, int D, bool FULL, bool MASK> struct Running {
    using G = Geometry<T, D>;
    floatx4 o[G::NE] = {};
    float m = -__builtin_inff(), l = 0;
    // `last`: of the step's keys, counted from 0
    __device__ __forceinline__ void step(Keys<T, D, FULL, MASK>& now, const uint4 (&q)[G::NF], float scale, int last, int g)
    {
        float s[G::PER_LANE];
        now.scores(q, s);
        if (MASK || last < G::N - 1) {
            // hidden keys: no score, and no value either (0 times an infinity would be NaN)
#pragma unroll
            for (int i = 0; i < G::PER_LANE; ++i) {
                const bool there = (G::key(i, g) <= last) & (!MASK || now.seen[i] != 0);
                s[i] = there ? s[i] : -__builtin_inff();
#pragma unroll
                for (size_t e = 0; e < G::NE * sizeof(T) / 4; ++e) now.v[i][e] = there ? now.v[i][e] : 0;
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

// The request that tile (row) `id` of a launch is of: the last whose tiles (rows) begin at or ahead of it.
template <bool ROWS = false, typename Args> __device__ __forceinline__ int request_of(const Args& p, int id)
{
    const int lane = threadIdx.x & 63;
    int before = 0;
#pragma unroll
    for (int i = 0; i < Args::BATCH; i += 64) {
        const int at = min(i + lane, p.n - 1);
        before += __popcll(__ballot(i + lane < p.n && (ROWS ? p.row[at] : p.req[at].first) <= id));
    }
    return __builtin_amdgcn_readfirstlane(before) - 1;
}

// (one without keys, too, where there are none)
__host__ __device__ __forceinline__ int parts_of(const CrossReq& r, int share) { return r.mem_len <= share ? 1 : (r.mem_len - 1) / share + 1; }

// D / 16 neighbouring columns of a row
template <typename T, int NE> __device__ __forceinline__ void store_columns(T* at, const float* v)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < NE; e += 4) *reinterpret_cast<float4*>(at + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    } else {
#pragma unroll
        for (int e = 0; e < NE; e += 4) *reinterpret_cast<uint2*>(at + e) = make_uint2(pack_bf16x2(v[e], v[e + 1]), pack_bf16x2(v[e + 2], v[e + 3]));
    }
}

// The rows of a tile from the parts of its memory: maximum and sum, then columns.  `m` in units of log2; at(part) gives a part's maximum, sum and columns.
template <typename T, int D, typename At>
__device__ __forceinline__ void finish_row(const CrossCommon& p, const CrossReq& r, int kv, int row, int chunk, int n_parts, At at)
{
    constexpr int NE = D / 16;
    const int group = p.n_heads / p.n_kv_heads;
    if (row >= r.q_len * group) return;
    float m = -__builtin_inff(), l = 0, o[NE] = {};
    for (int i = 0; i < n_parts; ++i) m = fmaxf(m, *at(i, 0));
    const float base = m == -__builtin_inff() ? 0.f : m;
    for (int i = 0; i < n_parts; ++i) {
        const float by = __builtin_amdgcn_exp2f(*at(i, 0) - base);
        l += by * *at(i, 1);
        const float* from = at(i, 2);
#pragma unroll
        for (int e = 0; e < NE; ++e) o[e] += by * from[e];
    }
    const long long q_row = (long long)r.q_row + row / group;
    const int head = kv * group + row % group;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < NE; ++e) o[e] *= inv;
    if (NE * chunk < p.head_dim) store_columns<T, NE>(static_cast<T*>(p.out) + q_row * p.out_stride + head * p.head_dim + NE * chunk, o);
    if (p.lse && chunk == 0) p.lse[q_row * p.n_heads + head] = l == 0.f ? -__builtin_inff() : (base + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// A tile of 16 rows over a part of its request's memory; the waves take steps of keys in turn, the next one's on its way, and meet in LDS.
template <typename T, int D, bool FULL, bool MASK, typename Args> __global__ __launch_bounds__(FEW_WAVES * 64) void k_cross_few(Args p)
{
    using G = Geometry<T, D>;
    constexpr int NE = G::NE, PITCH = D + 4, STRIDE = FEW_WAVES * G::N;
    __shared__ __align__(16) float s_o[FEW_WAVES][16][PITCH];
    __shared__ float s_ml[FEW_WAVES][2][16];
    const int id = p.runs ? (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3) : blockIdx.x, group = p.n_heads / p.n_kv_heads;
    if (id >= p.items) return;
    const CrossReq r = p.req[p.single ? id / p.n_kv_heads : request_of(p, id)];
    int at_tile = id - r.first, split = 0;
    if (p.share) {
        const int parts = parts_of(r, p.share);
        split = at_tile % parts;
        at_tile /= parts;
    }
    const int rows = r.q_len * group, tiles = (rows + 15) / 16, kv = at_tile / tiles, tile = at_tile % tiles;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, g = lane >> 4;
    const int begin = split * p.share, end = p.share ? min(r.mem_len, begin + p.share) : r.mem_len;
    const int row = 16 * tile + (lane & 15);
    const T* q_at = static_cast<const T*>(p.q) + ((long long)r.q_row + min(row, rows - 1) / group) * p.q_stride + (kv * group + min(row, rows - 1) % group) * p.head_dim;
    uint4 q[G::NF];
#pragma unroll
    for (int f = 0; f < G::NF; ++f) {
        const int d = (4 * f + g) * G::EPL;
        const bool there = FULL || d < p.head_dim;
        const uint4 x = *reinterpret_cast<const uint4*>(q_at + (there ? d : 0));
        q[f] = there ? x : make_uint4(0, 0, 0, 0);
    }
    const Places<T, D> at(p.k_stride, p.v_stride, p.head_dim, lane);
    const long long k_row = p.k_stride * (long long)sizeof(T), v_row = p.v_stride * (long long)sizeof(T);
    const char* kp = static_cast<const char*>(p.k) + r.mem_row * k_row + (size_t)kv * p.head_dim * sizeof(T);
    const char* vp = static_cast<const char*>(p.v) + r.mem_row * v_row + (size_t)kv * p.head_dim * sizeof(T);
    const uint8_t* keep = p.keep + r.mem_row;
    Running<T, D, FULL, MASK> run;
    Keys<T, D, FULL, MASK> a, b;
    auto load = [&](Keys<T, D, FULL, MASK>& to, int first) {
        first = min(first, end - 1);                     // (a step that there is not: the last key, and nobody takes it)
        const uint32_t last = min(end - 1 - first, G::N - 1);
        to.load(kp + first * k_row, vp + first * v_row, keep + first, at, last, last * (uint32_t)k_row, last * (uint32_t)v_row, p.head_dim, lane);
    };
    auto step = [&](Keys<T, D, FULL, MASK>& now, int first) { run.step(now, q, p.scale, min(end - 1 - first, G::N - 1), g); };
    int first = begin + wave * G::N;
    if (first < end) {
        load(a, first);
        for (; first + STRIDE < end; first += 2 * STRIDE) {
            load(b, first + STRIDE);
            step(a, first);
            load(a, first + 2 * STRIDE);
            step(b, first + STRIDE);
        }
        if (first < end) step(a, first);
    }
    float m = run.m, l = run.l;
    l = across_sum(l);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < NE; ++e) s_o[wave][lane & 15][NE * (4 * g + j) + e] = run.o[e][j];
    if (g == 0) {
        s_ml[wave][0][lane] = m;
        s_ml[wave][1][lane] = l;
    }
    __syncthreads();
    const int in_tile = threadIdx.x / 16, chunk = threadIdx.x & 15;
    if (!p.share) {
        finish_row<T, D>(p, r, kv, 16 * tile + in_tile, chunk, FEW_WAVES,
                         [&](int i, int what) -> const float* { return what < 2 ? &s_ml[i][what][in_tile] : &s_o[i][in_tile][NE * chunk]; });
        return;
    }
    // a part: rows of columns, then the rows' maxima and sums
    float* part = p.parts + (size_t)id * part_floats(D);
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
    store_columns<float, NE>(part + in_tile * D + NE * chunk, c);
    if (chunk == 0) {
        part[16 * D + in_tile] = top;
        part[16 * D + 16 + in_tile] = sum;
    }
}

// A row from its parts: their maxima give each a weight, then groups of D / 4 threads take parts in turn, four columns a thread, and meet in LDS.
constexpr int JOIN = 256;
static_assert(MAX_SPLITS <= JOIN, "a thread for every part");
template <typename T, int D, typename Args> __global__ __launch_bounds__(JOIN) void k_cross_join(Args p)
{
    constexpr int ACROSS = D / 4, GROUPS = JOIN / ACROSS;
    __shared__ float s_w[JOIN], s_top[JOIN / 64], s_sum[JOIN / 64];
    __shared__ float4 s_o[GROUPS][ACROSS];
    const int group = p.n_heads / p.n_kv_heads, id = blockIdx.x;
    const int at = request_of<true>(p, id), in_request = id - p.row[at];
    const CrossReq r = p.req[at];
    const int rows = r.q_len * group, tiles = (rows + 15) / 16, kv = in_request / rows, row = in_request % rows, in_tile = row % 16;
    const int n_parts = parts_of(r, p.share), wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const float* parts = p.parts + (size_t)(r.first + (kv * tiles + row / 16) * n_parts) * part_floats(D);
    const bool mine = (int)threadIdx.x < n_parts;
    const float* ml = parts + (size_t)(mine ? threadIdx.x : 0) * part_floats(D) + 16 * D + in_tile;
    const float m = mine ? ml[0] : -__builtin_inff(), l = mine ? ml[16] : 0.f;
    const float top_here = wave_max(m);
    if (lane == 0) s_top[wave] = top_here;
    __syncthreads();
    const float top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3])), base = top == -__builtin_inff() ? 0.f : top;
    const float by = __builtin_amdgcn_exp2f(m - base), sum_here = wave_sum(by * l);
    s_w[threadIdx.x] = by;
    if (lane == 0) s_sum[wave] = sum_here;
    __syncthreads();
    const float sum = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
    const int column = threadIdx.x % ACROSS;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* from = parts + in_tile * D + 4 * column;
#pragma unroll 4
    for (int i = threadIdx.x / ACROSS; i < n_parts; i += GROUPS) {
        const float4 x = *reinterpret_cast<const float4*>(from + (size_t)i * part_floats(D));
        const float w = s_w[i];
        o.x += w * x.x;
        o.y += w * x.y;
        o.z += w * x.z;
        o.w += w * x.w;
    }
    s_o[threadIdx.x / ACROSS][column] = o;
    __syncthreads();
    if (threadIdx.x >= ACROSS) return;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) {
        const float4 x = s_o[i][column];
        o.x += x.x;
        o.y += x.y;
        o.z += x.z;
        o.w += x.w;
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    const float v[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
    const long long q_row = (long long)r.q_row + row / group;
    const int head = kv * group + row % group;
    if (4 * column < p.head_dim) store_columns<T, 4>(static_cast<T*>(p.out) + q_row * p.out_stride + head * p.head_dim + 4 * column, v);
    if (p.lse && threadIdx.x == 0) p.lse[q_row * p.n_heads + head] = sum == 0.f ? -__builtin_inff() : (base + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// Many rows, two bytes: 32 * NW rows of a request and a key head, 32 a wave, over the memory in tiles of 64 keys that all waves read from LDS while
// the next R - 1 are on their way there, 16 bytes a lane straight from memory; one barrier a tile.
//
// Scores are transposed as above, of 32 keys and 32 rows an instruction: lane l holds row l % 32 and of each 16 keys 4 h .. 4 h + 3 and 8 + 4 h .. + 3
// (h = l / 32), which are eight of the second product's operand.  Its other operand, values with the keys along a lane, comes by LDS's transposing
// reads.  Keys' 16-byte pieces and values' 64-byte ones change places from row to row, so that reads down a column find all banks.
// Positions that are hidden or not there are loaded from zeros.  The sums are rescaled when a row's maximum has grown by more than 2^8: weights are at most
// that large until then, and their quotient is the same.
constexpr int KEYS = 64;
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
template <int D, int NW, int R> struct ManyRows {
    static constexpr int ROW = 2 * D, PART = KEYS * ROW, SLOT = 2 * PART, LOADS = PART / 1024 / NW, LDS = R * SLOT + 2 * KEYS * 8;
    static_assert(LOADS * 1024 * NW == PART, "shares of the waves");
};
// All but the last N loads of every wave are there, and all waves have read what they needed.
template <int N> __device__ __forceinline__ void arrived()
{
    static_assert(N < 64, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
// (written out as in linear8.hip: no registers to come back to)
__device__ __forceinline__ void to_lds(const char* from, uint32_t to)
{
    uint32_t m0;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off" : "={m0}"(m0) : "s"(to), "v"(from) : "memory");
}

// (128 registers where heads are narrow and tiles large: with 135 of them 3 waves in place of 4 share a SIMD, and 16 heads of 3000 x 3000 x 64 in eight requests
// take 366 in place of 328 us)
template <int D, int NW, int R, bool MASK> __global__ __launch_bounds__(64 * NW, D == 128 ? 2 : NW == 8 ? 4 : 3) void k_cross_many(CrossArgs p)
{
    using M = ManyRows<D, NW, R>;
    constexpr int ROW = M::ROW, ND = D / 32, NK = D / 16;
    extern __shared__ __align__(16) char lds[];
    uint64_t* masks = reinterpret_cast<uint64_t*>(lds + R * M::SLOT);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
    // Which tile: an XCD has a run of them, so that its L2 holds the memory that they share
    const int xcd = blockIdx.x & 7, id = p.start[xcd] + (blockIdx.x >> 3);
    if (id >= p.start[xcd + 1]) return;
    const CrossReq r = p.req[request_of(p, id)];
    const int group = p.n_heads / p.n_kv_heads, rows = r.q_len * group, tiles = (rows + 32 * NW - 1) / (32 * NW);
    const int kv = (id - r.first) / tiles, row = ((id - r.first) % tiles * NW + wave) * 32 + c, row_there = min(row, rows - 1);
    const long long q_row = (long long)r.q_row + row_there / group;
    const int head = kv * group + row_there % group;
    uint4 q[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) {
        const int d = 16 * k + 8 * h;
        const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(p.q) + q_row * p.q_stride + head * p.head_dim + (d < p.head_dim ? d : 0));
        q[k] = d < p.head_dim ? x : make_uint4(0, 0, 0, 0);
    }
    const int n_tiles = (r.mem_len + KEYS - 1) / KEYS;
    const long long k_row = 2 * p.k_stride, v_row = 2 * p.v_stride;
    // this wave's share of a tile: the row and piece that lie where the lane's 16 bytes go
    const char *k_from[M::LOADS], *v_from[M::LOADS];
    int from_row[M::LOADS];
    bool k_there[M::LOADS], v_there[M::LOADS];
#pragma unroll
    for (int i = 0; i < M::LOADS; ++i) {
        const int at = (wave + i * NW) * 1024 + lane * 16, at_row = at / ROW, piece = at % ROW / 16;
        const int k_piece = piece ^ (at_row & (D / 8 - 1)), v_piece = piece ^ (D == 128 ? at_row & 3 : at_row >> 1 & 1) << 2;
        from_row[i] = at_row;
        k_there[i] = 8 * k_piece < p.head_dim;
        v_there[i] = 8 * v_piece < p.head_dim;
        k_from[i] = static_cast<const char*>(p.k) + (r.mem_row + at_row) * k_row + 2 * kv * p.head_dim + 16 * k_piece;
        v_from[i] = static_cast<const char*>(p.v) + (r.mem_row + at_row) * v_row + 2 * kv * p.head_dim + 16 * v_piece;
    }
    const uint32_t lds_at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)lds;
    // which of a tile's keys there are; with a mask, of 64 tiles at a time
    auto there = [&](int tile) -> uint64_t {
        if constexpr (MASK) {
            const uint64_t m = masks[tile % (2 * KEYS)];
            const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)m), high = __builtin_amdgcn_readfirstlane((uint32_t)(m >> 32));
            return (uint64_t)high << 32 | low;
        }
        const int left = r.mem_len - tile * KEYS;
        return left >= KEYS ? ~0ull : (1ull << left) - 1;
    };
    auto look = [&](int first) {
        if constexpr (MASK)
            for (int t = first + wave; t < first + KEYS && t < n_tiles; t += NW) {
                const int key = t * KEYS + lane;
                const uint64_t m = __ballot(key < r.mem_len && p.keep[r.mem_row + min(key, r.mem_len - 1)] != 0);
                if (lane == 0) masks[t % (2 * KEYS)] = m;
            }
    };
    // (keys that are hidden may hold anything, their scores are not looked at; values count even with weight 0)
    auto bring_keys = [&](int tile, int slot) {
#pragma unroll
        for (int i = 0; i < M::LOADS; ++i) {
            const bool in = tile * KEYS + from_row[i] < r.mem_len;
            to_lds(in && k_there[i] ? k_from[i] + tile * (KEYS * k_row) : static_cast<const char*>(p.zeros), lds_at + slot * M::SLOT + (wave + i * NW) * 1024);
        }
    };
    auto bring_values = [&](int tile, int slot) {
        const uint64_t m = there(tile);
#pragma unroll
        for (int i = 0; i < M::LOADS; ++i) {
            const bool in = m >> from_row[i] & 1;
            to_lds(in && v_there[i] ? v_from[i] + tile * (KEYS * v_row) : static_cast<const char*>(p.zeros), lds_at + slot * M::SLOT + M::PART + (wave + i * NW) * 1024);
        }
    };
    auto bring = [&](int tile, int slot) {
        bring_keys(tile, slot);
        bring_values(tile, slot);
    };
    floatx16 o[ND] = {};
    float m = -__builtin_inff(), l = 0;
    // a tile, or its first 32 keys where there are no others
    auto take = [&](int slot, uint64_t mask, auto halves) {
        constexpr int N = decltype(halves)::value;
        const char* kt = lds + slot * M::SLOT + c * ROW;
        floatx16 s[N] = {};
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            const char* at = kt + 16 * ((2 * k + h) ^ (c & (D / 8 - 1)));
            const bf16x8 b = __builtin_bit_cast(bf16x8, q[k]);
#pragma unroll
            for (int t = 0; t < N; ++t) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(at + t * 32 * ROW), b, s[t], 0, 0, 0);
        }
        // reads two steps ahead of their products (left alone, the compiler puts each in front of its use)
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * N, 0);
#pragma unroll
        for (int k = 0; k < NK - 2; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, N, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, N, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 2 * N, 0);
        if (mask != (N == 2 ? ~0ull : 0xFFFFFFFFull)) {
#pragma unroll
            for (int t = 0; t < N; ++t) {
                const uint32_t bits = (uint32_t)(mask >> (32 * t)) >> (4 * h);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t in = __builtin_amdgcn_sbfe((int)bits, 8 * (i / 4) + (i & 3), 1);        // all bits or none
                    s[t][i] = __uint_as_float((__float_as_uint(s[t][i]) & in) | (0xFF800000u & ~in));
                }
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int i = 1; i < 16 * N; ++i) top = fmaxf(top, s[i / 16][i % 16]);
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * p.scale;
        if (__any(top > m + 8.f)) {
            top = fmaxf(m, top);
            const float by = __builtin_amdgcn_exp2f(m - (top == -__builtin_inff() ? 0.f : top));
            m = top;
            l *= by;
#pragma unroll
            for (int d = 0; d < ND; ++d) o[d] *= by;
        }
        const float base = m == -__builtin_inff() ? 0.f : m;
#pragma unroll
        for (int i = 0; i < 16 * N; ++i) {
            s[i / 16][i % 16] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 16][i % 16], p.scale, -base));
            l += s[i / 16][i % 16];
        }
        const char* vt = lds + slot * M::SLOT + M::PART + (4 * h + (lane >> 2 & 3)) * ROW + 32 * (lane >> 4 & 1) + 8 * (lane & 3);
        const int turn = D == 128 ? lane >> 2 & 3 : lane >> 3 & 1;
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) {
            uint4 w;                                     // (rounded to bf16, as in Keys::add)
            const int i = 8 * (k & 1);
            w.x = pack_bf16x2(s[k / 2][i], s[k / 2][i + 1]);
            w.y = pack_bf16x2(s[k / 2][i + 2], s[k / 2][i + 3]);
            w.z = pack_bf16x2(s[k / 2][i + 4], s[k / 2][i + 5]);
            w.w = pack_bf16x2(s[k / 2][i + 6], s[k / 2][i + 7]);
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                using Four = __attribute__((address_space(3))) shortx4*;
                const char* at = vt + 16 * k * ROW + 64 * (d ^ turn);
                const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)(at + 8 * ROW));
                const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, w), o[d], 0, 0, 0);
            }
        }
    };
    if (n_tiles) bring_keys(0, 0);
    if (MASK) {
        look(0);
        __syncthreads();
    }
    if (n_tiles) bring_values(0, 0);
    // The queries are here, with the first tile: waited for in the loop, they would be together with the tiles that are on their way.
#pragma unroll
    for (int k = 0; k < NK; ++k) asm volatile("" : "+v"(q[k].x), "+v"(q[k].y), "+v"(q[k].z), "+v"(q[k].w));
    for (int i = 1; i < R - 1 && i < n_tiles; ++i) bring(i, i);
    for (int tile = 0, slot = 0, free = R - 1; tile < n_tiles; ++tile) {
        // (the tiles behind this one that are on their way: R - 2 but at the end)
        if (tile + R - 2 < n_tiles) arrived<(R - 2) * 2 * M::LOADS>();
        else arrived<0>();
        if (MASK && tile % KEYS == 0 && tile + KEYS < n_tiles) {
            look(tile + KEYS);
            __syncthreads();
        }
        if (tile + R - 1 < n_tiles) bring(tile + R - 1, free);
        const uint64_t mask = there(tile);
        // (a form of its own for half a tile costs registers: only where they are to spare, and memories short)
        if (mask >> 32 != 0 || (mask != 0 && !(D == 64 && NW == 4))) take(slot, mask, std::integral_constant<int, 2>());
        else if (D == 64 && NW == 4 && mask != 0) take(slot, mask, std::integral_constant<int, 1>());
        free = slot;                                     // (the slot that the tile before this one was in)
        slot = slot + 1 == R ? 0 : slot + 1;
    }
    const auto sums = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(sums[0]) + __uint_as_float(sums[1]);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    bf16_t* out = static_cast<bf16_t*>(p.out) + q_row * p.out_stride + head * p.head_dim;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
            // columns 8 h' .. + 7 of each 16: the lanes that share a row exchange halves
            const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[d][i] * inv, o[d][i + 1] * inv), pack_bf16x2(o[d][i + 4] * inv, o[d][i + 5] * inv), false, false);
            const auto y = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[d][i + 2] * inv, o[d][i + 3] * inv), pack_bf16x2(o[d][i + 6] * inv, o[d][i + 7] * inv), false, false);
            const int column = 32 * d + 2 * i + 8 * h;
            if (row < rows && column < p.head_dim) *reinterpret_cast<uint4*>(out + column) = make_uint4(x[0], y[0], x[1], y[1]);
        }
    if (p.lse && row < rows && h == 0)
        p.lse[q_row * p.n_heads + head] = l == 0.f ? -__builtin_inff() : ((m == -__builtin_inff() ? 0.f : m) + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <int D, int NW, int R> hipError_t allow()
{
    const auto a = k_cross_many<D, NW, R, false>, b = k_cross_many<D, NW, R, true>;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(a), hipFuncAttributeMaxDynamicSharedMemorySize, ManyRows<D, NW, R>::LDS);
    return e == hipSuccess ? hipFuncSetAttribute(reinterpret_cast<const void*>(b), hipFuncAttributeMaxDynamicSharedMemorySize, ManyRows<D, NW, R>::LDS) : e;
}

template <int D, int NW, int R> hipError_t go_many(CrossArgs& a, hipStream_t s)
{
    // shares of the XCDs: equal in keys that their tiles go over, and a tile's own cost, some 160 keys' (16 requests of 600 queries, 8 heads of 64, over 64 keys 7.5
    // us, over 250 12.8, of which 2 are the launch's)
    constexpr int OWN = 160;
    const int group = a.n_heads / a.n_kv_heads;
    auto tiles_of = [&](const CrossReq& r) { return ((long long)r.q_len * group + 32 * NW - 1) / (32 * NW) * a.n_kv_heads; };
    double work = 0, done = 0;
    long long all = 0;
    int tiles = 0, most = 0;
    for (int i = 0; i < a.n; ++i) {
        work += (double)tiles_of(a.req[i]) * (a.req[i].mem_len + OWN);
        all += tiles_of(a.req[i]);
    }
    if (all > 0x7FFFFFFF / 8) return hipErrorInvalidValue;
    int x = 1;
    a.start[0] = 0;
    for (int i = 0; i < a.n; ++i) {
        a.req[i].first = tiles;
        const int mine = (int)tiles_of(a.req[i]), each = a.req[i].mem_len + OWN;
        for (; x < 8 && done + (double)mine * each >= work * x / 8; ++x) a.start[x] = std::min(tiles + mine, std::max(a.start[x - 1], tiles + (int)((work * x / 8 - done) / each + 0.5)));
        tiles += mine;
        done += (double)mine * each;
    }
    for (; x <= 8; ++x) a.start[x] = tiles;
    for (int i = 0; i < 8; ++i) most = std::max(most, a.start[i + 1] - a.start[i]);
    const auto kernel = a.keep ? k_cross_many<D, NW, R, true> : k_cross_many<D, NW, R, false>;
    constexpr int LDS = ManyRows<D, NW, R>::LDS;
    hipLaunchKernelGGL(kernel, dim3(8 * most), dim3(64 * NW), LDS, s, a);
    return hipGetLastError();
}

template <typename T, int D, bool FULL> hipError_t go_few(CrossArgs& a, int n_cu, hipStream_t s)
{
    int longest = 0;
    long long wgs = 0, rows = 0;                         // row tiles (or their parts), rows
    double keys = 0;                                     // that all row tiles go over
    const int group = a.n_heads / a.n_kv_heads;
    a.single = true;
    for (int i = 0; i < a.n; ++i) {
        const long long tiles = ((long long)a.req[i].q_len * group + 15) / 16;
        a.single &= tiles == 1;
        a.req[i].first = (int)wgs;
        wgs += tiles * a.n_kv_heads;
        keys += (double)tiles * a.n_kv_heads * a.req[i].mem_len;
        longest = std::max(longest, a.req[i].mem_len);
    }
    const bool step = a.single;
    a.share = 0;
    // Long memories are split, into parts of one length for all requests, where few workgroups or a few long ones would leave compute units idle.  What a compute unit has
    // to bring of whole memories goes by latency: some 45 GB/s from the last-level cache, 22 (32 with heads of 128, whose steps are twice as large) if they come from memory;
    // parts come at 5.1 TB/s, some of it lost, and the join costs 5 us.  us, whole / split, 8 heads of 64, bf16, requests x keys: 1 x 500 5.7 / 7.1, 1 x 1000 8.3 / 7.1, 8 x 1000 8.4 /
    // 8.6, 8 x 4000 23.7 / 18.0, 16 x 4000 24.4 / 28.4, 24 x 16000 178 / 146, 32 x 16000 210 / 232, 40 x 16000 351 / 250, 48 x 500 .. 8000 149 /
    // 97; 4 x 27000, 8 heads of 128 that four share each, 339 / 88 (5.05 TB/s).
    const double row = 2.0 * a.head_dim * sizeof(T), all = keys * row, rate = all <= 256 << 20 ? 45e3 : D == 64 ? 22e3 : 32e3;
    const double here = (longest + (double)((wgs - 1) / n_cu) * keys / wgs) * row;       // of a compute unit: the longest, and others
    // The shortest parts that compute units hold all of at once (24 x 16000 in 960 of them 146 us, in 1152 166; 16 x 8000 with heads of 128 in 512 101, in 1024 105); shorter ones, so
    // that it comes to even shares, where memories differ (64 x 500 .. 8000 in 1024 142, in 2048 123).
    const bool alike = longest * (double)wgs <= 1.25 * keys;
    const int most = std::min(MAX_PARTS, (D == 128 ? 2 : alike ? 4 : 8) * n_cu);
    if (2 * wgs <= most && here / rate > 1.1 * all / 5.1e6 + 5) {
        auto cut = [&](int share) {
            long long items = 0, row = 0;
            for (int i = 0; i < a.n; ++i) {
                a.req[i].first = (int)items;
                a.row[i] = (int)row;
                items += ((long long)a.req[i].q_len * group + 15) / 16 * a.n_kv_heads * parts_of(a.req[i], share);
                row += (long long)a.req[i].q_len * a.n_heads;
            }
            return items;
        };
        // (memories' last parts are half as long on average; all of them whole at one and a half times this)
        double share = std::max({keys / (most - 0.5 * wgs), (double)longest / MAX_SPLITS, 128.0});
        while (share < longest && cut((int)std::ceil(share)) > most) share *= 1.0625;
        if (share < longest) {
            const int parts = (longest - 1) / (int)std::ceil(share) + 1, even = (longest - 1) / parts + 1;
            a.share = cut(even) <= most ? even : (int)std::ceil(share);
            wgs = cut(a.share);
            rows = a.row[a.n - 1] + (long long)a.req[a.n - 1].q_len * a.n_heads;
            a.single = false;
        }
    }
    a.items = (int)wgs;
    // In a step, heads of which several share a line of 128 bytes are one XCD's; others go round, which spreads long requests.  us, round / runs, 64 x 1925 keys, 4 heads that four
    // share: heads of 40 29.0 / 15.2, of 64 23.4 / 22.1; 32 x 4000, 8 heads of 64 45 / 49; 8 x 200 .. 500 queries over 200 .. 600 keys, 8 fp32 heads of 40 39 / 45.
    a.runs = step && a.head_dim * sizeof(T) % 128 != 0;
    auto launch = [&](const auto& args) {
        using Args = std::decay_t<decltype(args)>;
        const auto kernel = a.keep ? k_cross_few<T, D, FULL, true, Args> : k_cross_few<T, D, FULL, false, Args>;
        hipLaunchKernelGGL(kernel, dim3(a.runs ? (a.items + 7) / 8 * 8 : a.items), dim3(FEW_WAVES * 64), 0, s, args);
        if (a.share) hipLaunchKernelGGL((k_cross_join<T, D, Args>), dim3((unsigned)rows), dim3(JOIN), 0, s, args);
        return hipGetLastError();
    };
    if (a.n > CROSS_SMALL) return launch(a);
    CrossArgsOf<CROSS_SMALL> small;
    static_cast<CrossCommon&>(small) = a;
    std::copy_n(a.req, a.n, small.req);
    if (a.share) std::copy_n(a.row, a.n, small.row);
    return launch(small);
}

}  // namespace

size_t cross_parts_bytes() { return (size_t)MAX_PARTS * part_floats(128) * 4; }

hipError_t allow_cross()
{
    hipError_t e = allow<64, 4, 3>();
    if (e == hipSuccess) e = allow<64, 8, 3>();
    if (e == hipSuccess) e = allow<128, 4, 2>();
    if (e == hipSuccess) e = allow<128, 8, 3>();
    return e;
}

hipError_t launch_cross_few(CrossArgs& a, bool bf16, int n_cu, hipStream_t s)
{
    const bool wide = a.head_dim > 64, full = a.head_dim % 64 == 0;
    if (bf16 && wide) return full ? go_few<bf16_t, 128, true>(a, n_cu, s) : go_few<bf16_t, 128, false>(a, n_cu, s);
    if (bf16) return full ? go_few<bf16_t, 64, true>(a, n_cu, s) : go_few<bf16_t, 64, false>(a, n_cu, s);
    if (wide) return full ? go_few<float, 128, true>(a, n_cu, s) : go_few<float, 128, false>(a, n_cu, s);
    return full ? go_few<float, 64, true>(a, n_cu, s) : go_few<float, 64, false>(a, n_cu, s);
}

hipError_t launch_cross_many(CrossArgs& a, int n_cu, hipStream_t s)
{
    const bool eight = cross_many_large(a.req, a.n, a.n_heads / a.n_kv_heads, a.n_kv_heads, n_cu);
    if (a.head_dim > 64) return eight ? go_many<128, 8, 3>(a, s) : go_many<128, 4, 2>(a, s);
    return eight ? go_many<64, 8, 3>(a, s) : go_many<64, 4, 3>(a, s);
}

}  // namespace tts
