// The product of 8-bit rows with 8-bit weights, a power of two for each 128 columns of either: y = x w^T + bias.
//
// A matrix instruction takes whole blocks of columns or half ones, and both operands' scales, so that a block costs no work beside it.  Channels are
// the instruction's rows and rows of x its columns: a lane ends with neighbouring channels of one row.  Weights lie in units of 32
// channels and 64 columns, as the 32 x 32 instruction takes them: 32 bytes a lane, of row l % 32 the columns from 32 * (l / 32) on.  Row 8 a + 4 h + j of
// the t-th of two units is channel 32 h + 16 t + 4 a + j of the 64: a lane of that instruction has 16 neighbouring channels of a unit.
#include "operator_kernels.h"
#include "mfma.h"
#include "lds_loads.h"

namespace tts {

namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));

struct Frag8 { uint4 half[2]; };

__device__ __forceinline__ intx8 operand(const Frag8& f) { return __builtin_bit_cast(intx8, f); }

// Two forms of the sums.  Fast: the 8-bit instruction's own.  It aligns the products of an instruction to the largest and drops bits some 2^-17 below it, 1.4e-5
// of the result for normal values, far below a bf16 result's rounding.  Exact: operands brought to bf16 with their scales (e4m3's four bits and
// a power of two from 2^-124 to 2^119 fit; of smaller ones bf16's least number, 2^-133, cuts bits off, and 256 * 2^120 is no bf16 number), four instructions of 32 columns: 4e-8 to 8e-8.
template <bool EXACT> struct Operand;
template <> struct Operand<false> {
    Frag8 f;
    int scale;
    Operand() = default;
    __device__ __forceinline__ Operand(const Frag8& v, uint32_t byte) : f(v), scale((int)byte) {}
};
template <> struct Operand<true> {
    bf16x8 part[4];
    Operand() = default;
    __device__ __forceinline__ Operand(const Frag8& v, uint32_t byte)
    {
        const float by = __uint_as_float(byte << 23);     // (the conversion takes its exponent's field alone: 0 is 2^-127 to it)
        const intx8 w = operand(v);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * q + d], by, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * q + d], by, true);
                part[q][4 * d] = lo[0];
                part[q][4 * d + 1] = lo[1];
                part[q][4 * d + 2] = hi[0];
                part[q][4 * d + 3] = hi[1];
            }
        }
    }
};
typedef float floatx16 __attribute__((ext_vector_type(16)));
// 16 x 16 results of 128 columns, or 32 x 32 of 64
__device__ __forceinline__ floatx4 product(const Operand<false>& a, const Operand<false>& b, floatx4 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a.f), operand(b.f), acc, 0, 0, 0, a.scale, 0, b.scale);
}
__device__ __forceinline__ floatx16 product(const Operand<false>& a, const Operand<false>& b, floatx16 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(a.f), operand(b.f), acc, 0, 0, 0, a.scale, 0, b.scale);
}
__device__ __forceinline__ floatx4 product(const Operand<true>& a, const Operand<true>& b, floatx4 acc)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.part[q], b.part[q], acc, 0, 0, 0);
    return acc;
}
__device__ __forceinline__ floatx16 product(const Operand<true>& a, const Operand<true>& b, floatx16 acc)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.part[q], b.part[q], acc, 0, 0, 0);
    return acc;
}
// In front of the first other use of accumulators.  The compiler has placed reads of the scaled instructions' results too few cycles behind
// them where a branch lay between (garbage, seen on a loop that copied its accumulator); 32 cycles are what the longest takes.
template <typename V, int N> __device__ __forceinline__ void settle(V (&acc)[N])
{
    asm volatile("s_nop 15\n\ts_nop 15" : "+v"(acc[0]));
#pragma unroll
    for (int i = 1; i < N; ++i) asm volatile("" : "+v"(acc[i]));
}

// Four channels of a row from `n0` on, at an address that is aligned to an element (the hardware takes wide accesses at any).
struct __attribute__((packed, aligned(2))) Four16 { uint32_t w[2]; };
struct __attribute__((packed, aligned(4))) Four32 { float w[4]; };
template <typename YT> __device__ __forceinline__ void store_four(const Linear8Args& p, int row, int n0, floatx4 v)
{
    if (row >= p.rows || n0 >= p.out_dim) return;
    YT* y = static_cast<YT*>(p.y) + row * p.y_stride + n0;
    if (n0 + 4 <= p.out_dim) {
        if constexpr (sizeof(YT) == 2) *reinterpret_cast<Four16*>(y) = Four16{{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}};
        else *reinterpret_cast<Four32*>(y) = Four32{{v[0], v[1], v[2], v[3]}};
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (n0 + i < p.out_dim) y[i] = from_float<YT>(v[i]);
    }
}

// Up to 16 rows: the weights are what there is to read.  A workgroup forms 16 channels; its waves take blocks in turn, straight from memory into
// registers, and add their sums up through LDS in their order.
constexpr int FEW_WAVES = 8;
template <typename YT> __global__ __launch_bounds__(FEW_WAVES * 64) void k_linear8_few(Linear8Args p)
{
    constexpr bool EXACT = sizeof(YT) == 4;
    __shared__ floatx4 red[FEW_WAVES][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, g = lane >> 4;
    const int half = blockIdx.x, row = lane & 15, words = (p.blocks + 3) / 4;
    // the 16 x 16 instruction's operand, 32 columns from 32 g on, from two units of columns
    const uint4* w = p.w + ((size_t)(half >> 1) * p.blocks * 2 + (g >> 1)) * 128 + 32 * (g & 1) + 16 * (half & 1) + row;
    const uint32_t* sw = p.sw + (size_t)(half >> 1) * words * 32 + 16 * (half & 1) + row;
    const uint8_t* x = p.x8 + (size_t)min(row, p.rows - 1) * p.blocks * E8_BLOCK + 32 * g;
    const uint8_t* sx = p.sx + (size_t)min(row, p.rows - 1) * words * 4;
    floatx4 acc[1] = {};
    for (int b = wave; b < p.blocks; b += FEW_WAVES) {
        const Frag8 wf = {w[(size_t)b * 256], w[(size_t)b * 256 + 64]};
        const uint8_t* at = x + (size_t)b * E8_BLOCK;
        const Frag8 xf = {*reinterpret_cast<const uint4*>(at), *reinterpret_cast<const uint4*>(at + 16)};
        acc[0] = product(Operand<EXACT>(wf, sw[b / 4 * 32] >> (8 * (b & 3)) & 255), Operand<EXACT>(xf, sx[b]), acc[0]);
    }
    settle(acc);
    red[wave][lane] = acc[0];
    __syncthreads();
    if (wave == 0) {
        const int n0 = half / 4 * 64 + 32 * (g & 1) + 16 * (half >> 1 & 1) + 4 * (2 * (half & 1) + (g >> 1));
        floatx4 y = *reinterpret_cast<const floatx4*>(p.bias + n0);
#pragma unroll
        for (int i = 0; i < FEW_WAVES; ++i) y += red[i][lane];
        store_four<YT>(p, row, n0, y);
    }
}

// Many rows: tiles of 32 * TN * WN channels and 32 * TM * WM rows, in steps of 64 * SUB columns.  A step of both operands lies in LDS while the next
// STEPS - 1 are on their way there, 16 bytes a lane straight from memory; one barrier a step.  Weights lie in operand order.  Of x four
// lanes bring the 64 bytes of a row (lanes of rows apart, as the operand has them, take a cycle of the load path each: 128 x 128 tiles of
// 16384 x 4096 x 4096 353 in place of 305 us), each the quarter that its place is for: rows' quarters change places every four rows, so that the
// operand's reads of 16 bytes find all banks.

// All but the last N loads of every wave are there, and all waves have read what they needed.
template <int N> __device__ __forceinline__ void arrived()
{
    static_assert(N < 64, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }

// 16 bytes of a row
struct __attribute__((packed, aligned(2))) Piece { uint32_t w[4]; };
template <typename YT> __device__ __forceinline__ void store_piece(const Linear8Args& p, int row, int n0, uint4 v)
{
    constexpr int N = 16 / sizeof(YT);
    if (row >= p.rows || n0 >= p.out_dim) return;
    YT* y = static_cast<YT*>(p.y) + row * p.y_stride + n0;
    if (n0 + N <= p.out_dim) *reinterpret_cast<Piece*>(y) = Piece{{v.x, v.y, v.z, v.w}};
    else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
            if (n0 + i < p.out_dim) {
                if constexpr (sizeof(YT) == 2) reinterpret_cast<uint16_t*>(y)[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
                else reinterpret_cast<uint32_t*>(y)[i] = w[i];
            }
    }
}

template <typename YT, int TN, int TM, int WN, int WM, int SUB, int STEPS> struct Many {
    static constexpr bool EXACT = sizeof(YT) == 4;
    static constexpr int WAVES = WN * WM, NT = TN * WN, MT = TM * WM;            // units of a workgroup
    static constexpr int PART = (NT + MT) * 2048, STEP = SUB * PART, SCALES = (NT + MT) * 128, LDS = STEPS * STEP + 2 * SCALES;
    static constexpr int W_LOADS = SUB * NT * 2 / WAVES, X_LOADS = SUB * MT * 2 / WAVES, LOADS = W_LOADS + X_LOADS;      // of a wave a step
    static constexpr int S_LOADS = ((NT + MT) / 2 + WAVES - 1) / WAVES;                      // ... every four blocks
    static_assert(W_LOADS * WAVES == SUB * NT * 2 && X_LOADS * WAVES == SUB * MT * 2 && SUB <= 2 && NT % 2 == 0 && MT % 2 == 0, "shares of the waves");
    static constexpr int PITCH = NT * 32 * sizeof(YT) + 16;                                 // of rows on their way out
    static_assert(32 * WM * PITCH <= STEPS * STEP && 64 * WAVES % (NT * 2 * sizeof(YT)) == 0, "the results' way out");
    const Linear8Args& p;
    int wave, lane, wn, wm, unit0, row0;
    uint32_t lds_at;
    const uint8_t *w_at[W_LOADS], *x_at, *s_base[S_LOADS];      // this wave's share of a step, and of the scales
    uint32_t x_off[X_LOADS], s_off[S_LOADS], s_step[S_LOADS];
    uint8_t* lds;
    floatx16 acc[TN * TM] = {};

    __device__ __forceinline__ Many(const Linear8Args& a, uint8_t* l, int n_tile, int m_tile) : p(a), lds(l)
    {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        lane = threadIdx.x & 63;
        wn = wave % WN;
        wm = wave / WN;
        unit0 = n_tile * NT;
        row0 = m_tile * MT * 32;
        const int units = channel_units(p.out_dim), words = (p.blocks + 3) / 4;
        const uint32_t width = p.blocks * E8_BLOCK;
        const uint8_t* w = reinterpret_cast<const uint8_t*>(p.w);
#pragma unroll
        for (int i = 0; i < W_LOADS; ++i) {
            const int c = wave + i * WAVES, sub = c / (2 * NT), u = c % (2 * NT) / 2;
            w_at[i] = w + ((size_t)min(unit0 + u, units - 1) * p.blocks * 4 + 2 * sub + (c & 1)) * 1024;
        }
        x_at = p.x8 + (size_t)row0 * width;
#pragma unroll
        for (int i = 0; i < X_LOADS; ++i) {
            const int c = wave + i * WAVES, sub = c / (2 * MT), r = c % (2 * MT) * 16;
            x_off[i] = (uint32_t)min(r + (lane >> 2), p.rows - 1 - row0) * width + 64 * sub + 16 * ((lane ^ (lane >> 4)) & 3);
        }
        // a load brings the scales of two units
#pragma unroll
        for (int i = 0; i < S_LOADS; ++i) {
            const int c = 2 * (wave + i * WAVES);
            if (c < NT) {
                s_base[i] = reinterpret_cast<const uint8_t*>(p.sw + (size_t)min(unit0 + c, units - 2) * words * 32);
                s_off[i] = (uint32_t)((lane >> 5) * words * 32 + (lane & 31)) * 4;
                s_step[i] = 128;
            } else {
                s_base[i] = p.sx + (size_t)row0 * words * 4;
                s_off[i] = (uint32_t)min((c - NT) * 32 + lane, p.rows - 1 - row0) * words * 4;
                s_step[i] = 4;
            }
        }
        lds_at = lds_address(lds);
    }
    __device__ __forceinline__ void bring(int step, int slot) const
    {
        const uint32_t to = lds_at + slot * STEP;
#pragma unroll
        for (int i = 0; i < W_LOADS; ++i) {
            const int c = wave + i * WAVES;
            to_lds_from<16>(w_at[i] + (size_t)step * (2048 * SUB), lane * 16, to + c / (2 * NT) * PART + c % (2 * NT) * 1024);
        }
#pragma unroll
        for (int i = 0; i < X_LOADS; ++i) {
            const int c = wave + i * WAVES;
            to_lds_from<16>(x_at + (size_t)step * (64 * SUB), x_off[i], to + c / (2 * MT) * PART + NT * 2048 + c % (2 * MT) * 1024);
        }
    }
    __device__ __forceinline__ void bring_scales(int word) const
    {
#pragma unroll
        for (int i = 0; i < S_LOADS; ++i)
            if (2 * (wave + i * WAVES) < NT + MT) to_lds_from<4>(s_base[i] + (size_t)word * s_step[i], s_off[i], lds_at + STEPS * STEP + (word & 1) * SCALES + (wave + i * WAVES) * 256);
    }
    __device__ __forceinline__ Frag8 w_frag(int part, int unit) const
    {
        const uint4* at = reinterpret_cast<const uint4*>(lds + part + unit * 2048) + lane;
        return Frag8{at[0], at[64]};
    }
    __device__ __forceinline__ Frag8 x_frag(int part, int unit) const
    {
        const uint4* at = reinterpret_cast<const uint4*>(lds + part + (NT + unit) * 2048) + 4 * (lane & 31);
        const int q = 2 * (lane >> 5) ^ (lane >> 2 & 3);
        return Frag8{at[q], at[q ^ 1]};
    }
    __device__ __forceinline__ void multiply(int block, int part, const uint32_t (&sw)[TN], const uint32_t (&sx)[TM])
    {
        const int shift = 8 * (block & 3);               // a word holds the scales of four blocks
        Operand<EXACT> x[TM];
#pragma unroll
        for (int m = 0; m < TM; ++m) x[m] = Operand<EXACT>(x_frag(part, wm * TM + m), sx[m] >> shift & 255);
        Frag8 w = w_frag(part, wn * TN);
        __builtin_amdgcn_sched_group_barrier(0x100, 2 + 2 * TM, 0);
#pragma unroll
        for (int n = 0; n < TN; ++n) {
            Frag8 next;
            if (n + 1 < TN) next = w_frag(part, wn * TN + n + 1);
            const Operand<EXACT> a(w, sw[n] >> shift & 255);
#pragma unroll
            for (int m = 0; m < TM; ++m) acc[n * TM + m] = product(a, x[m], acc[n * TM + m]);
            // a unit's products behind the next one's reads: left alone, the compiler puts each read in front of its use
            if (n + 1 < TN) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, (EXACT ? 4 : 1) * TM, 0);
            if (n + 1 < TN) w = next;
        }
    }
    // first of a lane's 16 channels of a unit
    __device__ __forceinline__ int channel(int unit) const { return unit / 2 * 64 + 32 * (lane >> 5) + 16 * (unit & 1); }
    __device__ __forceinline__ void run()
    {
        constexpr int PER_WORD = 8 / SUB;
        const int steps = 2 / SUB * p.blocks;
        bring_scales(0);
        for (int i = 0; i < STEPS - 1 && i < steps; ++i) bring(i, i);
        uint32_t sw[TN], sx[TM];
        for (int step = 0, slot = 0, free = STEPS - 1; step < steps; ++step) {
            // (the steps behind this one that are on their way: STEPS - 2 but at the end)
            if (step + STEPS - 2 < steps) arrived<(STEPS - 2) * LOADS>();
            else arrived<0>();
            if (step % PER_WORD == 0) {
                const uint32_t* s = reinterpret_cast<const uint32_t*>(lds + STEPS * STEP + (step / PER_WORD & 1) * SCALES) + (lane & 31);
#pragma unroll
                for (int n = 0; n < TN; ++n) sw[n] = s[(wn * TN + n) * 32];
#pragma unroll
                for (int m = 0; m < TM; ++m) sx[m] = s[(NT + wm * TM + m) * 32];
                if (step + PER_WORD < steps) bring_scales(step / PER_WORD + 1);
            }
            if (step + STEPS - 1 < steps) bring(step + STEPS - 1, free);
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) multiply(SUB == 2 ? step : step >> 1, slot * STEP + sub * PART, sw, sx);
            free = slot;                                  // (the slot that the step before this one was in)
            slot = slot + 1 == STEPS ? 0 : slot + 1;
        }
        settle(acc);
        // Rows leave by way of LDS, 32 * WM of them at a time, 16 bytes a lane along a row: lanes as the products have them would write to 64 lines an
        // instruction, a cycle each.
        floatx16 bias[TN] = {};
#pragma unroll
        for (int n = 0; n < TN; ++n) {
            const int n0 = channel(wn * TN + n);
            if (unit0 * 32 + n0 < p.out_dim) bias[n] = *reinterpret_cast<const floatx16*>(p.bias + unit0 * 32 + n0);
        }
#pragma unroll
        for (int m = 0; m < TM; ++m) {
            __syncthreads();                              // (steps, and the rows before these, are read)
#pragma unroll
            for (int n = 0; n < TN; ++n) {
                uint8_t* to = lds + (wm * 32 + (lane & 31)) * PITCH + channel(wn * TN + n) * sizeof(YT);
                const floatx16 v = acc[n * TM + m] + bias[n];
#pragma unroll
                for (int i = 0; i < 16; i += 16 / sizeof(YT)) {
                    if constexpr (sizeof(YT) == 2)
                        *reinterpret_cast<uint4*>(to + 2 * i) = make_uint4(pack_bf16x2(v[i], v[i + 1]), pack_bf16x2(v[i + 2], v[i + 3]), pack_bf16x2(v[i + 4], v[i + 5]), pack_bf16x2(v[i + 6], v[i + 7]));
                    else *reinterpret_cast<float4*>(to + 4 * i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                }
            }
            __syncthreads();
            constexpr int ACROSS = NT * 32 * sizeof(YT) / 16, ROWS = 64 * WAVES / ACROSS;
#pragma unroll
            for (int i = 0; i < 32 * WM / ROWS; ++i) {
                const int r = i * ROWS + threadIdx.x / ACROSS, at = threadIdx.x % ACROSS;
                store_piece<YT>(p, row0 + (r / 32 * TM + m) * 32 + r % 32, unit0 * 32 + at * (16 / (int)sizeof(YT)), *reinterpret_cast<const uint4*>(lds + r * PITCH + 16 * at));
            }
        }
    }
};

template <typename YT, int TN, int TM, int WN, int WM, int SUB, int STEPS>
__global__ __launch_bounds__(64 * WN * WM, WN * WM / 4) void k_linear8_many(Linear8Args p, int n_tiles, int m_tiles, int across)
{
    extern __shared__ __align__(16) uint8_t lds[];
    // An XCD's run of tiles is 4 rows of tiles high, so that its L2 holds what they share.
    const int total = n_tiles * m_tiles, id = linear8_tile(blockIdx.y * across + blockIdx.x, total);
    if (id >= total) return;
    const int band = id / (4 * n_tiles), in_band = id - band * 4 * n_tiles, high = min(4, m_tiles - 4 * band);
    Many<YT, TN, TM, WN, WM, SUB, STEPS> many(p, lds, in_band / high, 4 * band + in_band % high);
    many.run();
}

// In between: 32 channels and 32 rows a workgroup, whose waves take steps of 64 columns in turn, each through a ring in LDS of its own (no
// barrier until their sums meet).  A wave's i-th step has its scales in word i.
constexpr int SPLIT_WAVES = 8, SPLIT_RING = 2;
constexpr int SPLIT_SLOT = 2 * 2048 + 256, SPLIT_LOADS = 2 + 2 + 1, SPLIT_LDS = SPLIT_WAVES * SPLIT_RING * SPLIT_SLOT;      // weights, rows of x, the scales of both
static_assert(SPLIT_LDS >= SPLIT_WAVES * 4096 && SPLIT_LDS <= 160 * 1024, "the sums meet in the rings");
// All but the last N loads of this wave are there.
template <int N> __device__ __forceinline__ void brought()
{
    static_assert(N < 64, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void lane_to_lds(const void* from, uint32_t to)
{
    uint32_t m0;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, off" : "={m0}"(m0) : "s"(to), "v"(from) : "memory");
}
template <typename YT> __global__ __launch_bounds__(SPLIT_WAVES * 64, 2) void k_linear8_split(Linear8Args p)
{
    constexpr bool EXACT = sizeof(YT) == 4;
    extern __shared__ __align__(16) uint8_t lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
    const int units = channel_units(p.out_dim), unit = blockIdx.x % units, row0 = blockIdx.x / units * 32;
    const int words = (p.blocks + 3) / 4, steps = 2 * p.blocks;
    const uint32_t width = p.blocks * E8_BLOCK;
    const uint8_t* w_at = reinterpret_cast<const uint8_t*>(p.w) + (size_t)unit * p.blocks * 4096;
    const uint8_t* x_at = p.x8 + (size_t)row0 * width;
    uint32_t x_off[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) x_off[c] = (uint32_t)min(c * 16 + (lane >> 2), p.rows - 1 - row0) * width + 16 * ((lane ^ (lane >> 4)) & 3);
    // the scales: 32 channels' and 32 rows', one load
    const uint8_t* s_at = lane < 32 ? reinterpret_cast<const uint8_t*>(p.sw + (size_t)unit * words * 32 + lane) : p.sx + (size_t)min(row0 + lane - 32, p.rows - 1) * words * 4;
    const int s_step = lane < 32 ? 128 : 4;
    uint8_t* ring = lds + wave * SPLIT_RING * SPLIT_SLOT;
    const uint32_t ring_at = lds_address(ring);
    const int turns = steps > wave ? (steps - wave + SPLIT_WAVES - 1) / SPLIT_WAVES : 0;
    auto bring = [&](int turn) {
        const uint32_t to = ring_at + turn % SPLIT_RING * SPLIT_SLOT;
        const size_t step = (size_t)turn * SPLIT_WAVES + wave;
        to_lds_from<16>(w_at + step * 2048, lane * 16, to);
        to_lds_from<16>(w_at + step * 2048 + 1024, lane * 16, to + 1024);
#pragma unroll
        for (int c = 0; c < 2; ++c) to_lds_from<16>(x_at + step * 64, x_off[c], to + 2048 + c * 1024);
        lane_to_lds(s_at + turn * s_step, to + 4096);
    };
    floatx16 acc[1] = {};
    for (int i = 0; i < SPLIT_RING && i < turns; ++i) bring(i);
    for (int turn = 0; turn < turns; ++turn) {
        if (turn + SPLIT_RING <= turns) brought<(SPLIT_RING - 1) * SPLIT_LOADS>();
        else brought<0>();
        const uint8_t* slot = ring + turn % SPLIT_RING * SPLIT_SLOT;
        const uint4* w = reinterpret_cast<const uint4*>(slot) + lane;
        const uint4* x = reinterpret_cast<const uint4*>(slot + 2048) + 4 * (lane & 31);
        const uint32_t* s = reinterpret_cast<const uint32_t*>(slot + 4096) + (lane & 31);
        const int q = 2 * (lane >> 5) ^ (lane >> 2 & 3), shift = 8 * (wave >> 1 & 3);
        const Frag8 wf = {w[0], w[64]}, xf = {x[q], x[q ^ 1]};
        const uint32_t ws = s[0], xs = s[32];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (the slot is free)
        if (turn + SPLIT_RING < turns) bring(turn + SPLIT_RING);
        acc[0] = product(Operand<EXACT>(wf, ws >> shift & 255), Operand<EXACT>(xf, xs >> shift & 255), acc[0]);
    }
    settle(acc);
    __syncthreads();                                              // (the rings are read)
    float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int i = 0; i < 16; ++i) sums[(wave * 16 + i) * 64 + lane] = acc[0][i];
    __syncthreads();
    if (wave >= 4) return;
    const int i0 = 4 * wave, n0 = unit / 2 * 64 + 32 * (lane >> 5) + 16 * (unit & 1) + i0;
    floatx4 y = n0 < p.out_dim ? *reinterpret_cast<const floatx4*>(p.bias + n0) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < SPLIT_WAVES; ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += sums[(w * 16 + i0 + i) * 64 + lane];
    store_four<YT>(p, row0 + (lane & 31), n0, y);
}
template <typename YT> hipError_t allow_split()
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(k_linear8_split<YT>), hipFuncAttributeMaxDynamicSharedMemorySize, SPLIT_LDS);
}
template <typename YT> hipError_t go_split(const Linear8Args& a, hipStream_t s)
{
    hipLaunchKernelGGL((k_linear8_split<YT>), dim3(channel_units(a.out_dim) * ((a.rows + 31) / 32)), dim3(SPLIT_WAVES * 64), SPLIT_LDS, s, a);
    return hipGetLastError();
}

template <typename YT, int TN, int TM, int WN, int WM, int SUB, int STEPS> hipError_t allow()
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(k_linear8_many<YT, TN, TM, WN, WM, SUB, STEPS>), hipFuncAttributeMaxDynamicSharedMemorySize, Many<YT, TN, TM, WN, WM, SUB, STEPS>::LDS);
}
template <typename YT, int TN, int TM, int WN, int WM, int SUB, int STEPS> hipError_t go_many(const Linear8Args& a, hipStream_t s)
{
    using M = Many<YT, TN, TM, WN, WM, SUB, STEPS>;
    const int n_tiles = (channel_units(a.out_dim) + M::NT - 1) / M::NT, m_tiles = (a.rows + M::MT * 32 - 1) / (M::MT * 32);
    const Linear8Grid grid = linear8_grid(n_tiles * m_tiles);
    hipLaunchKernelGGL((k_linear8_many<YT, TN, TM, WN, WM, SUB, STEPS>), dim3(grid.across, grid.down), dim3(64 * WN * WM), M::LDS, s, a, n_tiles, m_tiles, grid.across);
    return hipGetLastError();
}

template <typename YT> hipError_t go(const Linear8Args& a, int n_cu, hipStream_t s)
{
    constexpr bool TWO = sizeof(YT) == 2;
    switch (linear8_form(a.rows, a.out_dim, a.blocks, TWO, n_cu)) {
    case Linear8Form::FEW:
        hipLaunchKernelGGL((k_linear8_few<YT>), dim3(2 * channel_units(a.out_dim)), dim3(FEW_WAVES * 64), 0, s, a);
        return hipGetLastError();
    case Linear8Form::SPLIT: return go_split<YT>(a, s);
    case Linear8Form::TILE_64_64: return go_many<YT, 1, 1, 2, 2, 2, TWO ? 3 : 2>(a, s);
    case Linear8Form::TILE_64_128: return go_many<YT, 1, 2, 2, 2, 2, 2>(a, s);
    case Linear8Form::TILE_128_128: return go_many<YT, 2, 2, 2, 2, 2, 2>(a, s);
    case Linear8Form::TILE_256_128: break;
    }
    return go_many<YT, 4, 2, 2, 2, 1, 3>(a, s);
}

}  // namespace

// (more than 64 KB of LDS a workgroup has to be allowed, on each device)
template <typename YT> static hipError_t allow_all()
{
    hipError_t e = allow_split<YT>();
    if (e == hipSuccess) e = allow<YT, 4, 2, 2, 2, 1, 3>();
    if (e == hipSuccess) e = allow<YT, 2, 2, 2, 2, 2, 2>();
    if (e == hipSuccess) e = allow<YT, 1, 2, 2, 2, 2, 2>();
    if (e == hipSuccess) e = allow<YT, 1, 1, 2, 2, 2, sizeof(YT) == 2 ? 3 : 2>();
    return e;
}
hipError_t allow_linear8()
{
    const hipError_t e = allow_all<bf16_t>();
    return e == hipSuccess ? allow_all<float>() : e;
}

hipError_t launch_linear8(const Linear8Args& a, bool y_bf16, int n_cu, hipStream_t s)
{
    return y_bf16 ? go<bf16_t>(a, n_cu, s) : go<float>(a, n_cu, s);
}

}  // namespace tts
