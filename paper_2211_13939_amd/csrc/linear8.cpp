// Host side of the tts_linear8 C ABI: argument checks, and the weights' rounding to 8 bits and layout at creation.  All arithmetic of a call is in
// linear8.hip.
#include "../../include/tts_linear8.h"
#include "../../include/tts_norm.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <memory>
#include <new>

#include "operator_host.h"
#include "operator_kernels.h"

using namespace tts;

namespace {

int check(const tts_linear8_config* c)
{
    if (!c) return fail(TTS_E_INVAL, "config is null");
    if (c->in_dim < 1 || c->in_dim > TTS_LINEAR8_MAX_DIM) return fail(TTS_E_INVAL, "in_dim must be in 1..%d", TTS_LINEAR8_MAX_DIM);
    if (c->out_dim < 1 || c->out_dim > TTS_LINEAR8_MAX_DIM) return fail(TTS_E_INVAL, "out_dim must be in 1..%d", TTS_LINEAR8_MAX_DIM);
    if (!is_dtype(c->y_dtype)) return fail(TTS_E_INVAL, "y_dtype must be 0 (fp32) or 1 (bf16)");
    return TTS_OK;
}

struct Layout {
    int units, blocks, words;
    size_t w, sw, bias, total;
};
Layout layout_of(const tts_linear8_config& c)
{
    Layout l;
    l.units = channel_units(c.out_dim);
    l.blocks = width8(c.in_dim) / E8_BLOCK;
    l.words = scale_columns(c.in_dim) / 4;
    Carver a;
    l.w = a.take((size_t)l.units * l.blocks * 4096);
    l.sw = a.take((size_t)l.units * l.words * 128);
    l.bias = a.take((size_t)l.units * 128);
    l.total = a.off;
    return l;
}

// fp32 -> e4m3, round to nearest even; |v| <= 448 or not finite (NaN then).  Without branches: creation goes over every weight (16 million in 26 ms, in 93 with them).
inline uint8_t host_f2e4m3(float v)
{
    uint32_t u, s;
    memcpy(&u, &v, 4);
    const uint32_t sign = u >> 24 & 0x80;
    u &= 0x7FFFFFFFu;
    float a;
    memcpy(&a, &u, 4);
    a += 16384.f;                   // below 2^-6 a multiple of 2^-9, which is the sum's last bit
    memcpy(&s, &a, 4);
    const uint32_t normal = ((u + 0x7FFFFu + (u >> 20 & 1u)) >> 20) - (120u << 3);
    const uint32_t code = u >= 0x7F800000u ? 0x7Fu : u < 0x3C800000u ? s & 0xFu : normal;
    return (uint8_t)(sign | code);
}

// the least k with m <= 448 * 2^k = 1.75 * 2^(k + 8), as the byte k + 127, from 0 up; 127 where m = 0 (the rule of k_norm)
int scale_byte(float m)
{
    uint32_t u;
    memcpy(&u, &m, 4);
    if (!u) return 127;
    const int byte = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u);
    return byte > 0 ? byte : 0;
}

}  // namespace

struct tts_linear8 {
    tts_linear8_config cfg;
    Linear8Args args;
    hipStream_t stream = nullptr;
    int device = 0, n_cu = 0;
};

extern "C" size_t tts_linear8_workspace_bytes(const tts_linear8_config* cfg)
{
    if (check(cfg) != TTS_OK) return 0;
    return layout_of(*cfg).total;
}

extern "C" int tts_linear8_create(const tts_linear8_config* cfg, const float* w, const float* bias, void* dev_arena, size_t arena_bytes, void* hip_stream,
                                  tts_linear8** out)
{
    if (!out) return fail(TTS_E_INVAL, "out is null");
    *out = nullptr;
    int rc = check(cfg);
    if (rc) return rc;
    if (!w) return fail(TTS_E_INVAL, "null argument");
    const Layout lay = layout_of(*cfg);
    int device = 0, n_cu = 0;
    if ((rc = check_arena(dev_arena, arena_bytes, lay.total, &device))) return rc;
    OnDevice on(device);
    HIP_TRY(on.err);
    HIP_TRY(hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, device));
    HIP_TRY(allow_linear8());
    // the arena's contents, as one host copy
    std::unique_ptr<uint8_t[]> host(new (std::nothrow) uint8_t[lay.total]());
    tts_linear8* p = new (std::nothrow) tts_linear8();
    if (!host || !p) {
        delete p;
        return fail(TTS_E_INVAL, "out of host memory");
    }
    const int K = cfg->in_dim, N = cfg->out_dim;
    memset(host.get() + lay.sw, 127, (size_t)lay.units * lay.words * 128);
    for (int n = 0; n < N; ++n) {
        const float* row = w + (size_t)n * K;
        const int u = channel_unit(n), r = channel_row(n);
        for (int b = 0; b < lay.blocks; ++b) {
            const int k0 = b * E8_BLOCK, kn = K - k0 < E8_BLOCK ? K - k0 : E8_BLOCK;
            uint32_t most = 0;                          // (magnitudes are in the order of their bits)
            for (int k = 0; k < kn; ++k) {
                uint32_t u;
                memcpy(&u, row + k0 + k, 4);
                u &= 0x7FFFFFFFu;
                most = std::max(most, u < 0x7F800000u ? u : 0u);
            }
            float m;
            memcpy(&m, &most, 4);
            const int byte = scale_byte(m);
            host[lay.sw + (((size_t)u * lay.words + b / 4) * 32 + r) * 4 + b % 4] = (uint8_t)byte;
            const uint32_t bits = (uint32_t)(254 - byte) << 23;
            float by;
            memcpy(&by, &bits, 4);
            uint8_t* unit = host.get() + lay.w + ((size_t)u * lay.blocks + b) * 4096;
            uint8_t codes[E8_BLOCK] = {};
            for (int k = 0; k < kn; ++k) codes[k] = host_f2e4m3(row[k0 + k] * by);
            for (int k = 0; k < E8_BLOCK; k += 16) memcpy(unit + (k / 64 * 2 + k / 16 % 2) * 1024 + (k / 32 % 2 * 32 + r) * 16, codes + k, 16);
        }
        if (bias) memcpy(host.get() + lay.bias + (size_t)n * 4, bias + n, 4);
    }
    const hipError_t e = hipMemcpy(dev_arena, host.get(), lay.total, hipMemcpyHostToDevice);
    if (e != hipSuccess) {
        delete p;
        return fail(TTS_E_HIP, "upload of the weights: %s", hipGetErrorString(e));
    }
    const char* base = (const char*)dev_arena;
    p->cfg = *cfg;
    p->args = Linear8Args{};
    p->args.w = (const uint4*)(base + lay.w);
    p->args.sw = (const uint32_t*)(base + lay.sw);
    p->args.bias = (const float*)(base + lay.bias);
    p->args.out_dim = N;
    p->args.blocks = lay.blocks;
    p->stream = (hipStream_t)hip_stream;
    p->device = device;
    p->n_cu = n_cu;
    *out = p;
    return TTS_OK;
}

extern "C" int tts_linear8_run(tts_linear8* p, const void* x8, const void* scales, int rows, void* y, long long y_stride)
{
    if (!p) return fail(TTS_E_INVAL, "null argument");
    if (rows < 0 || rows > TTS_MAX_ROWS) return fail(TTS_E_INVAL, "rows = %d, at most %d per call", rows, TTS_MAX_ROWS);
    if (rows == 0) return TTS_OK;
    if (!x8 || !scales || !y) return fail(TTS_E_INVAL, "null argument");
    if (!aligned(x8, 16) || !aligned(scales, 4)) return fail(TTS_E_INVAL, "x8 must be 16-byte aligned, scales 4-byte");
    if (!aligned(y, dtype_bytes(p->cfg.y_dtype))) return fail(TTS_E_INVAL, "y is not aligned to its elements");
    if (y_stride == 0) y_stride = p->cfg.out_dim;
    if (y_stride < p->cfg.out_dim || y_stride > (1LL << 40)) return fail(TTS_E_INVAL, "y: a stride of %lld for %d columns", y_stride, p->cfg.out_dim);
    Linear8Args a = p->args;
    a.x8 = (const uint8_t*)x8;
    a.sx = (const uint8_t*)scales;
    a.rows = rows;
    a.y = y;
    a.y_stride = y_stride;
    OnDevice on(p->device);
    HIP_TRY(on.err);
    HIP_TRY(launch_linear8(a, p->cfg.y_dtype == TTS_DTYPE_BF16, p->n_cu, p->stream));
    return TTS_OK;
}

extern "C" void tts_linear8_destroy(tts_linear8* p) { delete p; }
