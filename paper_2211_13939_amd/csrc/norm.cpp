// Host side of the tts_norm C ABI: argument checks and the gain's upload.  All arithmetic is in norm.hip.
#include "../../include/tts_norm.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "operator_host.h"
#include "operator_kernels.h"

using namespace tts;

namespace {

int check(const tts_norm_config* c)
{
    if (!c) return fail(TTS_E_INVAL, "config is null");
    if (c->dim < 1 || c->dim > TTS_NORM_MAX_DIM) return fail(TTS_E_INVAL, "dim must be in 1..%d", TTS_NORM_MAX_DIM);
    if (c->kind != TTS_NORM_RMS && c->kind != TTS_NORM_NONE) return fail(TTS_E_INVAL, "kind must be 0 (root mean square) or 1 (none)");
    if (!is_dtype(c->x_dtype) || !is_dtype(c->res_dtype) || !is_dtype(c->y_dtype)) return fail(TTS_E_INVAL, "dtypes must be 0 (fp32) or 1 (bf16)");
    if (c->kind == TTS_NORM_RMS && !(c->eps >= 0 && std::isfinite(c->eps))) return fail(TTS_E_INVAL, "eps must be finite and not negative");
    return TTS_OK;
}

}  // namespace

struct tts_norm {
    tts_norm_config cfg;
    const float* gain = nullptr;         // device
    hipStream_t stream = nullptr;
    int device = 0, n_cu = 0;
};

extern "C" size_t tts_norm_workspace_bytes(const tts_norm_config* cfg)
{
    if (check(cfg) != TTS_OK) return 0;
    Carver a;
    a.take((size_t)cfg->dim * 4);
    return a.off;
}

extern "C" int tts_norm_create(const tts_norm_config* cfg, const float* gain, void* dev_arena, size_t arena_bytes, void* hip_stream, tts_norm** out)
{
    if (!out) return fail(TTS_E_INVAL, "out is null");
    *out = nullptr;
    int rc = check(cfg);
    if (rc) return rc;
    if ((cfg->kind == TTS_NORM_RMS) != (gain != nullptr)) return fail(TTS_E_INVAL, cfg->kind == TTS_NORM_RMS ? "gain is null" : "no norm, but a gain");
    int device = 0, n_cu = 0;
    if ((rc = check_arena(dev_arena, arena_bytes, tts_norm_workspace_bytes(cfg), &device))) return rc;
    OnDevice on(device);
    HIP_TRY(on.err);
    HIP_TRY(hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, device));
    if (gain) HIP_TRY(hipMemcpy(dev_arena, gain, (size_t)cfg->dim * 4, hipMemcpyHostToDevice));
    tts_norm* p = new (std::nothrow) tts_norm();
    if (!p) return fail(TTS_E_INVAL, "out of host memory");
    p->cfg = *cfg;
    p->gain = gain ? (const float*)dev_arena : nullptr;
    p->stream = (hipStream_t)hip_stream;
    p->device = device;
    p->n_cu = n_cu;
    *out = p;
    return TTS_OK;
}

extern "C" int tts_norm_run(tts_norm* p, const tts_norm_rows* r)
{
    if (!p || !r) return fail(TTS_E_INVAL, "null argument");
    if (r->rows < 0 || r->rows > TTS_MAX_ROWS) return fail(TTS_E_INVAL, "rows = %d, at most %d per call", r->rows, TTS_MAX_ROWS);
    if (r->rows == 0) return TTS_OK;
    if (!r->x || !(r->total || r->y || r->y8)) return fail(TTS_E_INVAL, "x or every output is null");
    if (!r->y8 != !r->scales) return fail(TTS_E_INVAL, "y8 and scales come together");
    struct { const char* name; const void* at; long long stride; int dtype; } arrays[4] = {
        {"x", r->x, r->x_stride, p->cfg.x_dtype}, {"res", r->res, r->res_stride, p->cfg.res_dtype},
        {"total", r->total, r->total_stride, p->cfg.res_dtype}, {"y", r->y, r->y_stride, p->cfg.y_dtype}};
    long long stride[4];
    for (int i = 0; i < 4; ++i) {
        stride[i] = arrays[i].stride ? arrays[i].stride : p->cfg.dim;
        if (!arrays[i].at) continue;
        if (stride[i] < p->cfg.dim || stride[i] > (1LL << 40)) return fail(TTS_E_INVAL, "%s: a stride of %lld for %d columns", arrays[i].name, stride[i], p->cfg.dim);
        if (!aligned(arrays[i].at, dtype_bytes(arrays[i].dtype))) return fail(TTS_E_INVAL, "%s is not aligned to its elements", arrays[i].name);
    }
    if (!aligned(r->y8, 16) || !aligned(r->scales, 4)) return fail(TTS_E_INVAL, "y8 must be 16-byte aligned, scales 4-byte");
    NormArgs a{};
    a.x = r->x; a.res = r->res; a.total = r->total; a.y = r->y;
    a.y8 = (uint8_t*)r->y8; a.scales = (uint8_t*)r->scales;
    a.gain = p->gain;
    a.x_stride = stride[0]; a.res_stride = stride[1]; a.total_stride = stride[2]; a.y_stride = stride[3];
    a.rows = r->rows; a.dim = p->cfg.dim;
    a.eps = p->cfg.eps;
    a.y_bf16 = p->cfg.y_dtype == TTS_DTYPE_BF16;
    OnDevice on(p->device);
    HIP_TRY(on.err);
    HIP_TRY(launch_norm(a, p->cfg.x_dtype == TTS_DTYPE_BF16, p->cfg.res_dtype == TTS_DTYPE_BF16, p->n_cu, p->stream));
    return TTS_OK;
}

extern "C" void tts_norm_destroy(tts_norm* p) { delete p; }
