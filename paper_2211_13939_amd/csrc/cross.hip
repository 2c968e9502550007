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

namespace tts {

namespace {

constexpr int FEW_WAVES = 4;
constexpr int MAX_PARTS = 1024, MAX_SPLITS = 64;     // parts of one launch, of one row tile
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
__device__ __forceinline__ void finish_row(const CrossArgs& p, const CrossReq& r, int kv, int row, int chunk, int n_parts, At at)
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
template <typename T, int D, bool FULL, bool MASK> __global__ __launch_bounds__(FEW_WAVES * 64) void k_cross_few(CrossArgs p, int splits)
{
    using G = Geometry<T, D>;
    constexpr int NE = G::NE, PITCH = D + 4, STRIDE = FEW_WAVES * G::N;
    __shared__ __align__(16) float s_o[FEW_WAVES][16][PITCH];
    __shared__ float s_ml[FEW_WAVES][2][16];
    const CrossReq r = p.req[blockIdx.z];
    const int kv = blockIdx.y, split = blockIdx.x % splits, tile = blockIdx.x / splits;
    const int group = p.n_heads / p.n_kv_heads, rows = r.q_len * group;
    if (16 * tile >= rows) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, g = lane >> 4;
    const int share = ((r.mem_len + splits - 1) / splits + G::N - 1) / G::N * G::N;
    const int begin = split * share, end = min(r.mem_len, begin + share);
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
    if (splits == 1) {
        finish_row<T, D>(p, r, kv, 16 * tile + in_tile, chunk, FEW_WAVES,
                         [&](int i, int what) -> const float* { return what < 2 ? &s_ml[i][what][in_tile] : &s_o[i][in_tile][NE * chunk]; });
        return;
    }
    // a part: rows of columns, then the rows' maxima and sums
    float* part = p.parts + (((size_t)blockIdx.z * p.n_kv_heads + kv) * gridDim.x + blockIdx.x) * part_floats(D);
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

template <typename T, int D> __global__ __launch_bounds__(256) void k_cross_join(CrossArgs p, int splits)
{
    constexpr int NE = D / 16;
    const CrossReq r = p.req[blockIdx.z];
    const int kv = blockIdx.y, tile = blockIdx.x, in_tile = threadIdx.x / 16, chunk = threadIdx.x & 15;
    const float* parts = p.parts + (((size_t)blockIdx.z * p.n_kv_heads + kv) * gridDim.x + tile) * splits * part_floats(D);
    finish_row<T, D>(p, r, kv, 16 * tile + in_tile, chunk, splits, [&](int i, int what) -> const float* {
        const float* part = parts + (size_t)i * part_floats(D);
        return what == 2 ? part + in_tile * D + NE * chunk : part + 16 * D + 16 * what + in_tile;
    });
}

template <typename T, int D, bool FULL> void go(const CrossArgs& a, int n_cu, hipStream_t s)
{
    int tiles = 0, longest = 0;
    const int group = a.n_heads / a.n_kv_heads;
    for (int i = 0; i < a.n; ++i) {
        tiles = std::max(tiles, (a.req[i].q_len * group + 15) / 16);
        longest = std::max(longest, a.req[i].mem_len);
    }
    const long long wgs = (long long)tiles * a.n_kv_heads * a.n;
    int splits = (int)std::min<long long>({MAX_PARTS / wgs, (long long)MAX_SPLITS, (long long)longest / 256});
    if (splits < 2) splits = 1;
    const auto kernel = a.keep ? k_cross_few<T, D, FULL, true> : k_cross_few<T, D, FULL, false>;
    hipLaunchKernelGGL(kernel, dim3(tiles * splits, a.n_kv_heads, a.n), dim3(FEW_WAVES * 64), 0, s, a, splits);
    if (splits > 1) hipLaunchKernelGGL((k_cross_join<T, D>), dim3(tiles, a.n_kv_heads, a.n), dim3(256), 0, s, a, splits);
}

}  // namespace

size_t cross_parts_bytes() { return (size_t)MAX_PARTS * part_floats(128) * 4; }

hipError_t launch_cross(CrossArgs& a, bool bf16, int n_cu, hipStream_t s)
{
    const bool wide = a.head_dim > 64, full = a.head_dim % 64 == 0;
    if (bf16 && wide) full ? go<bf16_t, 128, true>(a, n_cu, s) : go<bf16_t, 128, false>(a, n_cu, s);
    else if (bf16) full ? go<bf16_t, 64, true>(a, n_cu, s) : go<bf16_t, 64, false>(a, n_cu, s);
    else if (wide) full ? go<float, 128, true>(a, n_cu, s) : go<float, 128, false>(a, n_cu, s);
    else full ? go<float, 64, true>(a, n_cu, s) : go<float, 64, false>(a, n_cu, s);
    return hipGetLastError();
}

}  // namespace tts
