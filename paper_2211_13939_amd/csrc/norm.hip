// The norm in front of a block's products: total = x + res, y = gain * total / sqrt(mean(total^2) + eps), y rounded to 8 bits with a
// power of two for each 128 columns.  One pass: a row lies in registers from its loads to its stores.
//
// Bound by bytes (some 6 operations an element).  A lane holds chunks of 8 neighbouring columns, so that loads and stores are 16 or 32
// bytes a lane and 16 lanes hold a block of 128: its largest magnitude is found by four exchanges inside a row of 16 lanes.  Rows of up to
// 2048 columns are a wave's in large calls (no barrier); wider ones, and those of calls with fewer rows than the chip has waves for, a
// workgroup's.  us: 16384 x 4096 with residual, total and 8-bit rows 82 (468 MB, 5.7 TB/s), 8574 x 896 fp32 to fp32 and 8 bits 16 (69 MB), one row of 512 2.3 in a graph.
#include "operator_kernels.h"
#include "mfma.h"

namespace tts {

namespace {

// Eight elements from an address that is aligned to its elements alone (the hardware takes wide accesses at any address): rows
// of odd widths cost no loads of single elements but in their last chunk.
struct __attribute__((packed, aligned(2))) Raw16 { uint32_t w[4]; };
typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(2)));
// LATER: what this writes is read some kernels later (total, by the next norm): past the caches, which leaves them to what the next product reads.  bf16, a norm and
// the product of its rows by square weights in turn, us before / after: 2000 x 512 8.6 / 8.6, 8192 x 1024 26.5 / 27.6, 8192 x 2048 60.6 / 58.3, 16384 x 2048 109.8 /
// 105.9; a norm by itself, 6831 x 448 7.0 / 5.8.  (y and y8 so as well: 28.7, 60.9 and 112.8 us of the same; they are read next.)
template <bool LATER> __device__ __forceinline__ void put(void* p, const Raw16& a)
{
    if constexpr (LATER) __builtin_nontemporal_store(Words4{a.w[0], a.w[1], a.w[2], a.w[3]}, static_cast<Words4*>(p));
    else *static_cast<Raw16*>(p) = a;
}

template <typename T> struct Eight;
template <> struct Eight<float> {
    Raw16 a, b;
    __device__ __forceinline__ void load(const float* p)
    {
        a = *reinterpret_cast<const Raw16*>(p);
        b = *reinterpret_cast<const Raw16*>(p + 4);
    }
    __device__ __forceinline__ void load_some(const float* p, int n)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) (i < 4 ? a.w[i & 3] : b.w[i & 3]) = i < n ? __float_as_uint(p[i]) : 0;
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) a.w[i] = b.w[i] = 0;
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i < 4 ? a.w[i & 3] : b.w[i & 3]); }
};
template <> struct Eight<bf16_t> {
    Raw16 a;
    __device__ __forceinline__ void load(const bf16_t* p) { a = *reinterpret_cast<const Raw16*>(p); }
    __device__ __forceinline__ void load_some(const bf16_t* p, int n)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) a.w[i] = (2 * i < n ? p[2 * i].bits : 0) | (2 * i + 1 < n ? (uint32_t)p[2 * i + 1].bits << 16 : 0);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) a.w[i] = 0;
    }
    __device__ __forceinline__ float get(int i) const { return i & 1 ? bf16_hi(a.w[i >> 1]) : bf16_lo(a.w[i >> 1]); }
};

template <bool LATER> __device__ __forceinline__ void store_eight(float* p, const float* v, int n)
{
    if (n >= 8) {
        Raw16 a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a.w[i] = __float_as_uint(v[i]);
            b.w[i] = __float_as_uint(v[4 + i]);
        }
        put<LATER>(p, a);
        put<LATER>(p + 4, b);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i] = v[i];
    }
}
template <bool LATER> __device__ __forceinline__ void store_eight(bf16_t* p, const float* v, int n)
{
    if (n >= 8) {
        Raw16 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a.w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        put<LATER>(p, a);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i] = from_float<bf16_t>(v[i]);
    }
}

// Exchanges inside rows of 16 lanes: quads of lanes by their order, then eights and sixteens by mirroring, which pairs lanes whose quads
// (eights) hold different parts.
template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float row16_max(float x)
{
    x = fmaxf(x, dpp<0xB1>(x));
    x = fmaxf(x, dpp<0x4E>(x));
    x = fmaxf(x, dpp<0x141>(x));
    return fmaxf(x, dpp<0x140>(x));
}
__device__ __forceinline__ float row16_sum(float x)
{
    x += dpp<0xB1>(x);
    x += dpp<0x4E>(x);
    x += dpp<0x141>(x);
    return x + dpp<0x140>(x);
}
__device__ __forceinline__ float lane_value(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }

// The least k with m <= 448 * 2^k = 1.75 * 2^(k + 8), as the byte k + 127 (0 .. 247); m is finite and not negative.
__device__ __forceinline__ int scale_byte(float m)
{
    const uint32_t u = __float_as_uint(m);
    const int byte = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u);     // (subnormals have exponent bits 0: the least scale)
    return m == 0.f ? 127 : max(byte, 0);
}

template <typename XT, typename RT, int LPR, int NC> __global__ __launch_bounds__(256) void k_norm(NormArgs p)
{
    constexpr int ROWS = 256 / LPR;
    __shared__ float part[LPR > 64 ? LPR / 64 : 1];
    const int lane = threadIdx.x % LPR;
    const int row = (blockIdx.y * gridDim.x + blockIdx.x) * ROWS + (LPR == 256 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / LPR));
    if (row >= p.rows) return;
    const XT* x = static_cast<const XT*>(p.x) + row * p.x_stride;
    const RT* res = p.res ? static_cast<const RT*>(p.res) + row * p.res_stride : nullptr;
    Eight<XT> xv[NC];
    Eight<RT> rv[NC];
    float t[NC][8], g[NC][8];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int at = (c * LPR + lane) * 8, n = p.dim - at;
        if (n >= 8) xv[c].load(x + at);
        else if (n > 0) xv[c].load_some(x + at, n);
        else xv[c].zero();
    }
    if (res) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * LPR + lane) * 8, n = p.dim - at;
            if (n >= 8) rv[c].load(res + at);
            else if (n > 0) rv[c].load_some(res + at, n);
            else rv[c].zero();
        }
    }
    if (p.gain) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * LPR + lane) * 8, n = p.dim - at;
            Eight<float> gv;
            if (n >= 8) gv.load(p.gain + at);
            else if (n > 0) gv.load_some(p.gain + at, n);
            else gv.zero();
#pragma unroll
            for (int i = 0; i < 8; ++i) g[c][i] = gv.get(i);
        }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) t[c][i] = res ? xv[c].get(i) + rv[c].get(i) : xv[c].get(i);
    if (p.total) {
        RT* total = static_cast<RT*>(p.total) + row * p.total_stride;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * LPR + lane) * 8;
            if (at < p.dim) store_eight<true>(total + at, t[c], p.dim - at);
        }
    }
    if (!p.y && !p.y8) return;
    if (p.gain) {
        // (the mean of the squares of a row times `by`)
        auto mean_square = [&](float by) {
            float sum = 0;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += (t[c][i] * by) * (t[c][i] * by);
            sum = row16_sum(sum);
            sum = (lane_value(sum, 0) + lane_value(sum, 16)) + (lane_value(sum, 32) + lane_value(sum, 48));
            if constexpr (LPR > 64) {
                if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = sum;
                __syncthreads();
                sum = (part[0] + part[1]) + (part[2] + part[3]);
            }
            return sum / p.dim;
        };
        const float mean = mean_square(1.0f) + p.eps;
        float inv = 1.0f / sqrtf(mean);
        if (!(mean >= 0x1p-100f && mean < __builtin_inff())) {
            // Squares that leave fp32's range: the row times a power of two has the same quotient, its squares' sum another that is undone.  (Elements lie below 2^-43 in the first case.  In the second most
            // of the factor is the sum's alone, small ones beside large ones would lose bits to it.)
            const bool small = mean < 0x1p-100f;
            const float row_by = small ? 0x1p100f : 0x1p-4f, sum_by = small ? 1.0f : 0x1p-76f, by = row_by * sum_by;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) t[c][i] *= row_by;
            if constexpr (LPR > 64) __syncthreads();      // (the first sum is read)
            inv = sum_by / sqrtf(mean_square(sum_by) + p.eps * by * by);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) t[c][i] = t[c][i] * inv * g[c][i];
        // 0 times an infinity or a NaN (a row with a NaN in it, or of zeros without an eps) is NaN, and what lies past dim stays zero.
        if (!(inv < __builtin_inff())) {
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) t[c][i] = (c * LPR + lane) * 8 + i < p.dim ? t[c][i] : 0.f;
        }
    }
    if (p.y) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * LPR + lane) * 8;
            if (at >= p.dim) continue;
            if (p.y_bf16) store_eight<false>(static_cast<bf16_t*>(p.y) + row * p.y_stride + at, t[c], p.dim - at);
            else store_eight<false>(static_cast<float*>(p.y) + row * p.y_stride + at, t[c], p.dim - at);
        }
    }
    if (p.y8) {
        const int width = width8(p.dim), n_scales = scale_columns(p.dim);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * LPR + lane) * 8, block = at / E8_BLOCK;
            float m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fabsf(t[c][i]) < __builtin_inff() ? fmaxf(m, fabsf(t[c][i])) : m;
            m = row16_max(m);
            const int byte = scale_byte(m);
            const float by = __uint_as_float((uint32_t)(254 - byte) << 23);          // 2^(127 - byte)
            if (at < width) {
                int w[2] = {0, 0};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(t[c][4 * i] * by, t[c][4 * i + 1] * by, w[i], false);
                    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(t[c][4 * i + 2] * by, t[c][4 * i + 3] * by, w[i], true);
                }
                *reinterpret_cast<int2*>(p.y8 + (size_t)row * width + at) = make_int2(w[0], w[1]);
            }
            if (lane % 16 == 0 && block < n_scales) p.scales[(size_t)row * n_scales + block] = (uint8_t)(at < width ? byte : 127);
        }
    }
}

template <int LPR, int NC> void go(const NormArgs& a, bool x_bf16, bool res_bf16, hipStream_t s)
{
    constexpr int ROWS = 256 / LPR;
    const int wgs = (a.rows + ROWS - 1) / ROWS, high = (wgs >> 23) + 1;       // (a grid has fewer than 2^32 threads a side)
    const dim3 grid((wgs + high - 1) / high, high), block(256);
    if (x_bf16 && res_bf16) hipLaunchKernelGGL((k_norm<bf16_t, bf16_t, LPR, NC>), grid, block, 0, s, a);
    else if (x_bf16) hipLaunchKernelGGL((k_norm<bf16_t, float, LPR, NC>), grid, block, 0, s, a);
    else if (res_bf16) hipLaunchKernelGGL((k_norm<float, bf16_t, LPR, NC>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_norm<float, float, LPR, NC>), grid, block, 0, s, a);
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, bool x_bf16, bool res_bf16, int n_cu, hipStream_t s)
{
    const bool many = a.rows >= 8 * n_cu;
    if (a.dim <= 512) go<64, 1>(a, x_bf16, res_bf16, s);
    else if (a.dim <= 1024 && many) go<64, 2>(a, x_bf16, res_bf16, s);
    else if (a.dim <= 2048 && many) go<64, 4>(a, x_bf16, res_bf16, s);
    else if (a.dim <= 2048) go<256, 1>(a, x_bf16, res_bf16, s);
    else if (a.dim <= 4096) go<256, 2>(a, x_bf16, res_bf16, s);
    else if (a.dim <= 8192) go<256, 4>(a, x_bf16, res_bf16, s);
    else go<256, 8>(a, x_bf16, res_bf16, s);
    return hipGetLastError();
}

}  // namespace tts
