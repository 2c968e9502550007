// The product of 8-bit rows with 8-bit weights, a power of two for each 128 columns of either: y = x w^T + bias.
//
// A matrix instruction of 16 x 16 results takes 128 columns, a block, and both blocks' scales, so that a block costs no work beside it.
// Channels are the instruction's rows and rows of x its columns: a lane ends with four neighbouring channels of one row.  Row 4 g + j of the t-th of
// four tiles is channel 16 g + 4 t + j of their 64, so that with all four a lane has 16 neighbouring channels and a row's 64 are stored
// together.  An operand is 32 bytes a lane: of row l % 16 the 16 bytes from column 16 * (l / 16) of either half of the block; both operands share
// this map, so the order in which the instruction walks the columns does not matter.
#include "operator_kernels.h"
#include "mfma.h"

namespace tts {

namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));

struct Frag8 { uint4 half[2]; };

__device__ __forceinline__ intx8 operand(const Frag8& f) { return __builtin_bit_cast(intx8, f); }

// Two forms of the sums.  Fast: the 8-bit instruction's own.  It aligns the products of an instruction to the largest and drops bits some 2^-17 below it, 1.4e-5
// of the result for normal values, far below a bf16 result's rounding.  Exact: operands brought to bf16 with their scales (e4m3's four bits and
// any power of two fit), four instructions of 32 columns: 4e-8 to 8e-8.
template <bool EXACT> struct Operand;
template <> struct Operand<false> {
    Frag8 f;
    int scale;
    __device__ __forceinline__ Operand(const Frag8& v, uint32_t byte) : f(v), scale((int)byte) {}
};
template <> struct Operand<true> {
    bf16x8 part[4];
    __device__ __forceinline__ Operand(const Frag8& v, uint32_t byte)
    {
        const float by = __uint_as_float(byte << 23);
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
__device__ __forceinline__ floatx4 product(const Operand<false>& a, const Operand<false>& b, floatx4 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a.f), operand(b.f), acc, 0, 0, 0, a.scale, 0, b.scale);
}
__device__ __forceinline__ floatx4 product(const Operand<true>& a, const Operand<true>& b, floatx4 acc)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.part[q], b.part[q], acc, 0, 0, 0);
    return acc;
}
// In front of the first other use of accumulators.  The compiler has placed reads of the scaled instructions' results too few cycles behind
// them where a branch lay between (garbage, seen on a loop that copied its accumulator); 32 cycles are what the longest takes.
template <int N> __device__ __forceinline__ void settle(floatx4 (&acc)[N])
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

// Few rows: the weights are what there is to read.  A workgroup forms 16 channels of up to 16 * MT rows; its waves take blocks in turn, straight from
// memory into registers, and add their sums up through LDS in their order.
constexpr int FEW_WAVES = 8;
template <typename YT, int MT> __global__ __launch_bounds__(FEW_WAVES * 64) void k_linear8_few(Linear8Args p)
{
    constexpr bool EXACT = sizeof(YT) == 4;
    __shared__ floatx4 red[FEW_WAVES][MT][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
    const int tiles = channel_tiles(p.out_dim), tile = blockIdx.x % tiles, row0 = blockIdx.x / tiles * 16 * MT;
    const int width = p.blocks * E8_BLOCK, words = (p.blocks + 3) / 4;
    const uint4* w = p.w + (size_t)tile * p.blocks * 128 + lane;
    const uint32_t* sw = p.sw + (size_t)tile * words * 16 + (lane & 15);
    const uint8_t* x[MT];
    const uint8_t* sx[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const size_t row = min(row0 + 16 * m + (lane & 15), p.rows - 1);
        x[m] = p.x8 + row * width + 16 * (lane >> 4);
        sx[m] = p.sx + row * words * 4;
    }
    floatx4 acc[MT] = {};
#pragma unroll 2
    for (int b = wave; b < p.blocks; b += FEW_WAVES) {
        const Frag8 wf = {w[(size_t)b * 128], w[(size_t)b * 128 + 64]};
        const uint32_t ws = sw[b / 4 * 16] >> (8 * (b & 3)) & 255;
        const Operand<EXACT> a(wf, ws);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const uint8_t* at = x[m] + (size_t)b * E8_BLOCK;
            const Frag8 xf = {*reinterpret_cast<const uint4*>(at), *reinterpret_cast<const uint4*>(at + 64)};
            acc[m] = product(a, Operand<EXACT>(xf, sx[m][b]), acc[m]);
        }
    }
    settle(acc);
#pragma unroll
    for (int m = 0; m < MT; ++m) red[wave][m][lane] = acc[m];
    __syncthreads();
    if (wave < MT) {
        const int n0 = tile / 4 * 64 + 16 * (lane >> 4) + 4 * (tile & 3);
        floatx4 y = *reinterpret_cast<const floatx4*>(p.bias + n0);
#pragma unroll
        for (int i = 0; i < FEW_WAVES; ++i) y += red[i][wave][lane];
        store_four<YT>(p, row0 + 16 * wave + (lane & 15), n0, y);
    }
}

// Many rows: tiles of 16 * TN * WN channels and 16 * TM * WM rows, a block of columns of both in LDS while the next one is on its way there
// (16 bytes a lane straight from memory, in operand order: the loads place them, no exchange and no conflict is left).
//
// These loads are written out: of the builtin the compiler does not know which of two buffers it fills, and waits for it in front of every read of the
// other.  They have no registers to come back to; what they bring is there behind arrived().  (m0 has no other user in these kernels.)
template <int BYTES> __device__ __forceinline__ void to_lds(const uint8_t* base, uint32_t offset, uint32_t to)
{
    static_assert(BYTES == 16 || BYTES == 4, "");
    if constexpr (BYTES == 16) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
// What all waves brought is in LDS, and all have read what they needed.
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }

// The scale's byte J of a word
template <int J> __device__ __forceinline__ floatx4 product_of(const Frag8& a, uint32_t sa, const Frag8& b, uint32_t sb, floatx4 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a), operand(b), acc, 0, 0, J, (int)sa, J, (int)sb);
}

template <typename YT, int TN, int TM, int WN, int WM> struct Many {
    static constexpr bool EXACT = sizeof(YT) == 4;
    static constexpr int WAVES = WN * WM, NT = TN * WN, MT = TM * WM;            // tiles of a workgroup
    static constexpr int STAGE = (NT + MT) * 2048, SCALES = (NT + MT) * 64, LDS = 2 * STAGE + 2 * SCALES;
    static_assert(NT * 2 % WAVES == 0 && MT * 2 % WAVES == 0 && (NT + MT) == 4 * WAVES && NT % 4 == 0, "shares of the waves");
    const Linear8Args& p;
    uint8_t* lds;
    int wave, lane, wn, wm, tile0, row0;
    const uint8_t *w_at[NT * 2 / WAVES], *x_at;          // this wave's share of a stage
    uint32_t x_off[MT * 2 / WAVES];
    const uint8_t* s_base;                               // of the scales that it brings
    uint32_t s_off, s_step, lds_at;
    floatx4 acc[TN * TM] = {};

    __device__ __forceinline__ Many(const Linear8Args& a, uint8_t* l, int n_tile, int m_tile) : p(a), lds(l)
    {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        lane = threadIdx.x & 63;
        wn = wave % WN;
        wm = wave / WN;
        tile0 = n_tile * NT;
        row0 = m_tile * MT * 16;
        const int tiles = channel_tiles(p.out_dim), words = (p.blocks + 3) / 4;
        const uint32_t width = p.blocks * E8_BLOCK;
        const uint8_t* w = reinterpret_cast<const uint8_t*>(p.w);
#pragma unroll
        for (int i = 0; i < NT * 2 / WAVES; ++i) {
            const int c = wave + i * WAVES;
            w_at[i] = w + ((size_t)min(tile0 + c / 2, tiles - 1) * p.blocks * 128 + (c & 1) * 64) * 16;
        }
        x_at = p.x8 + (size_t)row0 * width;
#pragma unroll
        for (int i = 0; i < MT * 2 / WAVES; ++i) {
            const int c = wave + i * WAVES;
            x_off[i] = (uint32_t)min(c / 2 * 16 + (lane & 15), p.rows - 1 - row0) * width + (c & 1) * 64 + 16 * (lane >> 4);
        }
        // a wave brings the scales of four tiles
        if (4 * wave < NT) {
            s_base = reinterpret_cast<const uint8_t*>(p.sw + (size_t)min(tile0 + 4 * wave, tiles - 4) * words * 16);
            s_off = (uint32_t)((lane >> 4) * words * 16 + (lane & 15)) * 4;
            s_step = 64;
        } else {
            s_base = p.sx + (size_t)row0 * words * 4;
            s_off = (uint32_t)min((4 * wave - NT) * 16 + lane, p.rows - 1 - row0) * words * 4;
            s_step = 4;
        }
        lds_at = lds_address(lds);
    }
    __device__ __forceinline__ void bring(int b, int buf) const
    {
        const uint32_t to = lds_at + buf * STAGE + wave * 1024;
#pragma unroll
        for (int i = 0; i < NT * 2 / WAVES; ++i) to_lds<16>(w_at[i] + (size_t)b * 2048, lane * 16, to + i * WAVES * 1024);
#pragma unroll
        for (int i = 0; i < MT * 2 / WAVES; ++i) to_lds<16>(x_at + (size_t)b * E8_BLOCK, x_off[i], to + NT * 2048 + i * WAVES * 1024);
    }
    __device__ __forceinline__ void bring_scales(int word, int buf) const { to_lds<4>(s_base + (size_t)word * s_step, s_off, lds_at + 2 * STAGE + buf * SCALES + wave * 256); }
    __device__ __forceinline__ Frag8 frag(int buf, int tile) const
    {
        const uint4* at = reinterpret_cast<const uint4*>(lds + buf * STAGE + tile * 2048) + lane;
        return Frag8{at[0], at[64]};
    }
    template <int J> __device__ __forceinline__ void block(const uint32_t (&sw)[TN], const uint32_t (&sx)[TM])
    {
        constexpr int buf = J & 1;
        if constexpr (EXACT) {
            bf16x8 x[TM][4];
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                const Operand<true> o(frag(buf, NT + wm * TM + m), sx[m] >> (8 * J) & 255);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[m][q] = o.part[q];
            }
#pragma unroll
            for (int n = 0; n < TN; ++n) {
                const Operand<true> o(frag(buf, wn * TN + n), sw[n] >> (8 * J) & 255);
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int m = 0; m < TM; ++m) acc[n * TM + m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(o.part[q], x[m][q], acc[n * TM + m], 0, 0, 0);
            }
        } else {
            Frag8 x[TM];
#pragma unroll
            for (int m = 0; m < TM; ++m) x[m] = frag(buf, NT + wm * TM + m);
#pragma unroll
            for (int n = 0; n < TN; ++n) {
                const Frag8 w = frag(buf, wn * TN + n);
#pragma unroll
                for (int m = 0; m < TM; ++m) acc[n * TM + m] = product_of<J>(w, sw[n], x[m], sx[m], acc[n * TM + m]);
            }
        }
    }
    // block 4 * word + J of the columns; false: it was the last
    template <int J> __device__ __forceinline__ bool turn(int word, const uint32_t (&sw)[TN], const uint32_t (&sx)[TM])
    {
        const int b = 4 * word + J;
        if (b + 1 < p.blocks) bring(b + 1, (J + 1) & 1);
        block<J>(sw, sx);
        arrived();
        return b + 1 < p.blocks;
    }
    __device__ __forceinline__ void run()
    {
        bring_scales(0, 0);
        bring(0, 0);
        arrived();
        for (int word = 0;; ++word) {
            if (4 * word + 4 < p.blocks) bring_scales(word + 1, (word + 1) & 1);
            uint32_t sw[TN], sx[TM];
            const uint32_t* s = reinterpret_cast<const uint32_t*>(lds + 2 * STAGE + (word & 1) * SCALES) + (lane & 15);
#pragma unroll
            for (int n = 0; n < TN; ++n) sw[n] = s[(wn * TN + n) * 16];
#pragma unroll
            for (int m = 0; m < TM; ++m) sx[m] = s[(NT + wm * TM + m) * 16];
            if (!turn<0>(word, sw, sx) || !turn<1>(word, sw, sx) || !turn<2>(word, sw, sx) || !turn<3>(word, sw, sx)) break;
        }
        settle(acc);
#pragma unroll
        for (int n = 0; n < TN; ++n) {
            const int t = tile0 + wn * TN + n, n0 = t / 4 * 64 + 16 * (lane >> 4) + 4 * (t & 3);
            const floatx4 bias = n0 < p.out_dim ? *reinterpret_cast<const floatx4*>(p.bias + n0) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < TM; ++m) store_four<YT>(p, row0 + (wm * TM + m) * 16 + (lane & 15), n0, acc[n * TM + m] + bias);
        }
    }
};

template <typename YT, int TN, int TM, int WN, int WM> __global__ __launch_bounds__(64 * WN * WM, WN * WM / 4) void k_linear8_many(Linear8Args p, int n_tiles, int m_tiles)
{
    extern __shared__ __align__(16) uint8_t lds[];
    // Workgroups are dealt to the eight XCDs in turn; an XCD takes a run of tiles, 4 rows of tiles high, so that its L2 holds what they share.
    const int total = n_tiles * m_tiles, per = (total + 7) / 8;
    const int id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if (id >= total || (int)(blockIdx.x >> 3) >= per) return;
    const int band = id / (4 * n_tiles), in_band = id - band * 4 * n_tiles, high = min(4, m_tiles - 4 * band);
    Many<YT, TN, TM, WN, WM> many(p, lds, in_band / high, 4 * band + in_band % high);
    many.run();
}

template <typename YT, int TN, int TM, int WN, int WM> hipError_t allow()
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(k_linear8_many<YT, TN, TM, WN, WM>), hipFuncAttributeMaxDynamicSharedMemorySize, Many<YT, TN, TM, WN, WM>::LDS);
}
template <typename YT, int TN, int TM, int WN, int WM> hipError_t go_many(const Linear8Args& a, hipStream_t s)
{
    using M = Many<YT, TN, TM, WN, WM>;
    const int n_tiles = (channel_tiles(a.out_dim) + M::NT - 1) / M::NT, m_tiles = (a.rows + M::MT * 16 - 1) / (M::MT * 16);
    hipLaunchKernelGGL((k_linear8_many<YT, TN, TM, WN, WM>), dim3((n_tiles * m_tiles + 7) / 8 * 8), dim3(64 * WN * WM), M::LDS, s, a, n_tiles, m_tiles);
    return hipGetLastError();
}

template <typename YT> hipError_t go(const Linear8Args& a, int n_cu, hipStream_t s)
{
    const int tiles = channel_tiles(a.out_dim);
    const dim3 block(FEW_WAVES * 64);
    if (a.rows <= 16) hipLaunchKernelGGL((k_linear8_few<YT, 1>), dim3(tiles), block, 0, s, a);
    else if (a.rows <= 32) hipLaunchKernelGGL((k_linear8_few<YT, 2>), dim3(tiles), block, 0, s, a);
    else if (a.rows <= 64) hipLaunchKernelGGL((k_linear8_few<YT, 4>), dim3(tiles), block, 0, s, a);
    else {
        const long long large = (long long)((tiles + 15) / 16) * ((a.rows + 255) / 256);
        return large >= n_cu ? go_many<YT, 8, 4, 2, 4>(a, s) : go_many<YT, 4, 4, 2, 2>(a, s);
    }
    return hipGetLastError();
}

}  // namespace

// (more than 64 KB of LDS a workgroup has to be allowed, on each device)
hipError_t allow_linear8()
{
    hipError_t e = allow<bf16_t, 8, 4, 2, 4>();
    if (e == hipSuccess) e = allow<bf16_t, 4, 4, 2, 2>();
    if (e == hipSuccess) e = allow<float, 8, 4, 2, 4>();
    if (e == hipSuccess) e = allow<float, 4, 4, 2, 2>();
    return e;
}

hipError_t launch_linear8(const Linear8Args& a, bool y_bf16, int n_cu, hipStream_t s)
{
    return y_bf16 ? go<bf16_t>(a, n_cu, s) : go<float>(a, n_cu, s);
}

}  // namespace tts
