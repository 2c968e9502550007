// The product of 8-bit rows with 8-bit weights, a power of two for each 128 columns of either: y = x w^T + bias.
//
// A matrix instruction of 16 x 16 results takes 128 columns, a block, and both blocks' scales, so that a block costs no work beside it.
// Channels are the instruction's rows and rows of x its columns: a lane ends with four neighbouring channels of one row.  An operand is 32 bytes a
// lane: of row l % 16 the 16 bytes from column 16 * (l / 16) of either half of the block; both operands share this map, so the order in which the
// instruction walks the columns does not matter.
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
    const int tiles = (p.out_dim + 15) / 16, tile = blockIdx.x % tiles, row0 = blockIdx.x / tiles * 16 * MT;
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
        const int n0 = 16 * tile + 4 * (lane >> 4);
        floatx4 y = *reinterpret_cast<const floatx4*>(p.bias + n0);
#pragma unroll
        for (int i = 0; i < FEW_WAVES; ++i) y += red[i][wave][lane];
        store_four<YT>(p, row0 + 16 * wave + (lane & 15), n0, y);
    }
}

template <typename YT> void go(const Linear8Args& a, int n_cu, hipStream_t s)
{
    const int tiles = (a.out_dim + 15) / 16;
    const dim3 block(FEW_WAVES * 64);
    if (a.rows <= 16) hipLaunchKernelGGL((k_linear8_few<YT, 1>), dim3(tiles), block, 0, s, a);
    else if (a.rows <= 32) hipLaunchKernelGGL((k_linear8_few<YT, 2>), dim3(tiles), block, 0, s, a);
    else hipLaunchKernelGGL((k_linear8_few<YT, 4>), dim3(tiles * ((a.rows + 63) / 64)), block, 0, s, a);
}

}  // namespace

hipError_t launch_linear8(const Linear8Args& a, bool y_bf16, int n_cu, hipStream_t s)
{
    if (y_bf16) go<bf16_t>(a, n_cu, s);
    else go<float>(a, n_cu, s);
    return hipGetLastError();
}

}  // namespace tts
