// What the attentions (cross.hip, paged.hip) have in common: a wave's products of queries with keys and of weights with values, 16 rows of queries by registers alone (few rows), 32
// over a tile of 64 keys in LDS (many).
//
// Scores are formed transposed, keys as the matrix instruction's rows: a lane then holds four neighbouring keys of ONE query row, and so
// do its exponentials, which are the second product's operand (values as rows, query rows as columns) without leaving their registers.  The second product
// sums over keys in whatever order both operands share.
#pragma once
#include "mfma.h"

namespace tts {

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

template <typename T, int D> struct Operands {
    using G = Geometry<T, D>;
    uint4 k[G::TILES][G::NF];
    uint32_t v[G::PER_LANE][G::NE * sizeof(T) / 4];
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
            // products, of their upper and lower halves, would keep them at twice the matrix instructions; against 64 bits, in the norm over a call's outputs: 0.0018 for few rows, 0.0023 for many,
            // whose largest weight is no exact 1, where weights in fp32 have 0.0017, the results' own rounding)
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

// Many rows
constexpr int KEYS = 64;
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
// All but the last N loads of every wave are there, and all waves have read what they needed.
template <int N> __device__ __forceinline__ void arrived()
{
    static_assert(N < 64, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
// (written out, as in lds_loads.h; addresses are the lanes')
__device__ __forceinline__ void to_lds(const char* from, uint32_t to)
{
    uint32_t m0;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off" : "={m0}"(m0) : "s"(to), "v"(from) : "memory");
}

// 32 query rows of a wave over a tile of 64 keys, two bytes.  Lane l holds row l % 32 and of each 16 keys 4 h .. 4 h + 3 and 8 + 4 h .. + 3 (h = l / 32), which are eight of the second
// product's operand.  Its other operand, values with the keys along a lane, comes by LDS's transposing reads.  Keys' 16-byte pieces and values' 64-byte ones change places
// from row to row, so that reads down a column find all banks (key_piece, value_piece: which piece lies at a place).  The sums are rescaled when a row's maximum has grown by more than 2^8: weights
// are at most that large until then, and their quotient is the same.
template <int D> __device__ __forceinline__ int key_piece(int row, int piece) { return piece ^ (row & (D / 8 - 1)); }
template <int D> __device__ __forceinline__ int value_piece(int row, int piece) { return piece ^ (D == 128 ? row & 3 : row >> 1 & 1) << 2; }
template <int D> struct ManyRunning {
    static constexpr int ROW = 2 * D, ND = D / 32, NK = D / 16;
    uint4 q[NK];
    floatx16 o[ND] = {};
    float m = -__builtin_inff(), l = 0;
    // 16 values of four keys (k * 16 + 4 h .. and 8 behind) each along a lane: an operand of 32 columns from 32 d on
    static __device__ __forceinline__ bf16x8 values(const char* tile, int k, int d, int lane)
    {
        using Four = __attribute__((address_space(3))) shortx4*;
        const int turn = D == 128 ? lane >> 2 & 3 : lane >> 3 & 1;
        const char* at = tile + (4 * (lane >> 5) + (lane >> 2 & 3)) * ROW + 32 * (lane >> 4 & 1) + 8 * (lane & 3) + 16 * k * ROW + 64 * (d ^ turn);
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)(at + 8 * ROW));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // Scores and weights of a tile (N 2), or of its first 32 keys where there are no others (N 1); `hidden`: of some keys there is no score, those whose bit in `mask` is 0
    template <int N> __device__ __forceinline__ void weights(const char* keys, bool hidden, uint64_t mask, float scale, int lane, floatx16 (&s)[N])
    {
        const int c = lane & 31, h = lane >> 5;
        const char* kt = keys + c * ROW;
#pragma unroll
        for (int t = 0; t < N; ++t) s[t] = floatx16{};
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
        if (hidden) {
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
        top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * scale;
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
            s[i / 16][i % 16] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 16][i % 16], scale, -base));
            l += s[i / 16][i % 16];
        }
    }
    // eight weights of the k-th 16 keys
    template <int N> static __device__ __forceinline__ bf16x8 operand(const floatx16 (&s)[N], int k)
    {
        uint4 w;                                         // (rounded to bf16, as in Operands::add)
        const int i = 8 * (k & 1);
        w.x = pack_bf16x2(s[k / 2][i], s[k / 2][i + 1]);
        w.y = pack_bf16x2(s[k / 2][i + 2], s[k / 2][i + 3]);
        w.z = pack_bf16x2(s[k / 2][i + 4], s[k / 2][i + 5]);
        w.w = pack_bf16x2(s[k / 2][i + 6], s[k / 2][i + 7]);
        return __builtin_bit_cast(bf16x8, w);
    }
    template <int N> __device__ __forceinline__ void add(const char* tile, const floatx16 (&s)[N], int lane)
    {
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) {
            const bf16x8 w = operand<N>(s, k);
#pragma unroll
            for (int d = 0; d < ND; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values(tile, k, d, lane), w, o[d], 0, 0, 0);
        }
    }
    template <int N> __device__ __forceinline__ void take(const char* keys, const char* tile, bool hidden, uint64_t mask, float scale, int lane)
    {
        floatx16 s[N];
        weights<N>(keys, hidden, mask, scale, lane, s);
        add<N>(tile, s, lane);
    }
    // of the two lanes that share a row
    __device__ __forceinline__ float sum() const
    {
        const auto sums = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        return __uint_as_float(sums[0]) + __uint_as_float(sums[1]);
    }
    // The row's columns times `by`, in two bytes, 8 neighbouring ones a store: the lanes that share a row exchange halves.
    __device__ __forceinline__ void store(bf16_t* out, float by, bool there, int head_dim, int lane) const
    {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[d][i] * by, o[d][i + 1] * by), pack_bf16x2(o[d][i + 4] * by, o[d][i + 5] * by), false, false);
                const auto y = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[d][i + 2] * by, o[d][i + 3] * by), pack_bf16x2(o[d][i + 6] * by, o[d][i + 7] * by), false, false);
                const int column = 32 * d + 2 * i + 8 * (lane >> 5);
                if (there && column < head_dim) *reinterpret_cast<uint4*>(out + column) = make_uint4(x[0], y[0], x[1], y[1]);
            }
    }
};

}  // namespace tts
