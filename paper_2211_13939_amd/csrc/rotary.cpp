// Host side of the tts_rotary C ABI: argument checks and the frequencies.  All other arithmetic is in rotary.hip.
#include "../../include/tts_rotary.h"

#include <hip/hip_runtime.h>

#include <new>

#include "past_host.h"

using namespace tts;

namespace {

int check(const tts_rotary_config* c)
{
    if (!c) return fail(TTS_E_INVAL, "config is null");
    if (c->n_heads < 1 || c->n_heads > TTS_ROTARY_MAX_HEADS) return fail(TTS_E_INVAL, "n_heads must be in 1..%d", TTS_ROTARY_MAX_HEADS);
    if (c->head_dim < 8 || c->head_dim > TTS_ROTARY_MAX_HEAD_DIM || c->head_dim % 8)
        return fail(TTS_E_UNSUPPORTED, "kernels are built for head_dim in multiples of 8 up to %d", TTS_ROTARY_MAX_HEAD_DIM);
    if (!is_dtype(c->x_dtype) || !is_dtype(c->y_dtype)) return fail(TTS_E_INVAL, "dtypes must be 0 (fp32) or 1 (bf16)");
    return check_angles(c->angles, c->head_dim);
}

}  // namespace

struct tts_rotary {
    tts_rotary_config cfg;
    const uint64_t* freqs = nullptr;     // device
    hipStream_t stream = nullptr;
    int device = 0, n_cu = 0;
};

extern "C" size_t tts_rotary_workspace_bytes(const tts_rotary_config* cfg)
{
    if (check(cfg) != TTS_OK) return 0;
    Carver a;
    a.take((size_t)cfg->angles.rot_dim / 2 * 8);
    return a.off;
}

extern "C" int tts_rotary_create(const tts_rotary_config* cfg, void* dev_arena, size_t arena_bytes, void* hip_stream, tts_rotary** out)
{
    if (!out) return fail(TTS_E_INVAL, "out is null");
    *out = nullptr;
    int rc = check(cfg);
    if (rc) return rc;
    int device = 0, n_cu = 0;
    if ((rc = check_arena(dev_arena, arena_bytes, tts_rotary_workspace_bytes(cfg), &device))) return rc;
    OnDevice on(device);
    HIP_TRY(on.err);
    HIP_TRY(hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, device));
    try {
        const std::vector<uint64_t> freqs = turn_freqs(cfg->angles);
        HIP_TRY(hipMemcpy(dev_arena, freqs.data(), freqs.size() * 8, hipMemcpyHostToDevice));
    } catch (const std::bad_alloc&) {
        return fail(TTS_E_INVAL, "out of host memory");
    }
    tts_rotary* p = new (std::nothrow) tts_rotary();
    if (!p) return fail(TTS_E_INVAL, "out of host memory");
    p->cfg = *cfg;
    p->freqs = (const uint64_t*)dev_arena;
    p->stream = (hipStream_t)hip_stream;
    p->device = device;
    p->n_cu = n_cu;
    *out = p;
    return TTS_OK;
}

extern "C" int tts_rotary_run(tts_rotary* p, const tts_rotary_rows* r)
{
    if (!p || !r) return fail(TTS_E_INVAL, "null argument");
    if (r->rows < 0 || r->rows > TTS_ROTARY_MAX_ROWS) return fail(TTS_E_INVAL, "rows = %d, at most %d per call", r->rows, TTS_ROTARY_MAX_ROWS);
    if (r->back != 0 && r->back != 1) return fail(TTS_E_INVAL, "back must be 0 or 1");
    if (r->rows == 0) return TTS_OK;
    if (!r->x || !r->y) return fail(TTS_E_INVAL, "null argument");
    if (!aligned(r->positions, 4)) return fail(TTS_E_INVAL, "positions must be 4-byte aligned");
    if (!r->positions && (long long)r->first + r->rows > (1LL << 31)) return fail(TTS_E_INVAL, "the last position, %lld, is more than 32 bits hold", (long long)r->first + r->rows - 1);
    RotaryArgs a{};
    const long long width = (long long)p->cfg.n_heads * p->cfg.head_dim;
    a.x_stride = r->x_stride;
    a.y_stride = r->y_stride;
    int rc = check_rows("x", r->x, width, a.x_stride);
    if (!rc) rc = check_rows("y", r->y, width, a.y_stride);
    if (rc) return rc;
    if (r->x == r->y && (a.x_stride != a.y_stride || p->cfg.x_dtype != p->cfg.y_dtype)) return fail(TTS_E_INVAL, "y is x, but with another type or stride");
    a.x = r->x;
    a.y = r->y;
    a.positions = r->positions;
    a.turn = turn_angles(p->cfg.angles, p->cfg.head_dim, p->freqs);
    a.rows = r->rows;
    a.first = r->positions ? 0 : r->first;
    a.heads = p->cfg.n_heads;
    a.head_dim = p->cfg.head_dim;
    a.back = r->back;
    OnDevice on(p->device);
    HIP_TRY(on.err);
    HIP_TRY(launch_rotary(a, p->cfg.x_dtype == TTS_DTYPE_BF16, p->cfg.y_dtype == TTS_DTYPE_BF16, p->n_cu, p->stream));
    return TTS_OK;
}

extern "C" void tts_rotary_destroy(tts_rotary* p) { delete p; }
