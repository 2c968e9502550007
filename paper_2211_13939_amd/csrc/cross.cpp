// Host side of the tts_cross C ABI: argument checks and the batch's way into the launches' arguments.  All arithmetic is in cross.hip.
#include "../../include/tts_cross.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "operator_host.h"
#include "operator_kernels.h"

using namespace tts;

namespace {

int check(const tts_cross_config* c)
{
    if (!c) return fail(TTS_E_INVAL, "config is null");
    if (c->n_heads < 1 || c->n_heads > TTS_CROSS_MAX_HEADS) return fail(TTS_E_INVAL, "n_heads must be in 1..%d", TTS_CROSS_MAX_HEADS);
    if (c->n_kv_heads < 1 || c->n_kv_heads > c->n_heads || c->n_heads % c->n_kv_heads) return fail(TTS_E_INVAL, "n_heads must be a multiple of n_kv_heads");
    if (c->head_dim < 8 || c->head_dim > TTS_CROSS_MAX_HEAD_DIM || c->head_dim % 8)
        return fail(TTS_E_UNSUPPORTED, "kernels are built for head_dim in multiples of 8 up to %d", TTS_CROSS_MAX_HEAD_DIM);
    if (!is_dtype(c->dtype)) return fail(TTS_E_INVAL, "dtype must be 0 (fp32) or 1 (bf16)");
    return TTS_OK;
}

struct Layout { size_t parts, zeros, total; };
Layout layout_of()
{
    Layout l;
    Carver a;
    l.parts = a.take(cross_parts_bytes());
    l.zeros = a.take(256);
    l.total = a.off;
    return l;
}

}  // namespace

struct tts_cross {
    tts_cross_config cfg;
    float* parts = nullptr;              // device
    const void* zeros = nullptr;
    hipStream_t stream = nullptr;
    int device = 0, n_cu = 0;
};

extern "C" size_t tts_cross_workspace_bytes(const tts_cross_config* cfg)
{
    if (check(cfg) != TTS_OK) return 0;
    return layout_of().total;
}

extern "C" int tts_cross_create(const tts_cross_config* cfg, void* dev_arena, size_t arena_bytes, void* hip_stream, tts_cross** out)
{
    if (!out) return fail(TTS_E_INVAL, "out is null");
    *out = nullptr;
    int rc = check(cfg);
    if (rc) return rc;
    int device = 0, n_cu = 0;
    const Layout lay = layout_of();
    if ((rc = check_arena(dev_arena, arena_bytes, lay.total, &device))) return rc;
    OnDevice on(device);
    HIP_TRY(on.err);
    HIP_TRY(allow_cross());
    HIP_TRY(fill_now((char*)dev_arena + lay.zeros, 0, 256));
    HIP_TRY(hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, device));
    tts_cross* p = new (std::nothrow) tts_cross();
    if (!p) return fail(TTS_E_INVAL, "out of host memory");
    p->cfg = *cfg;
    p->parts = (float*)((char*)dev_arena + lay.parts);
    p->zeros = (char*)dev_arena + lay.zeros;
    p->stream = (hipStream_t)hip_stream;
    p->device = device;
    p->n_cu = n_cu;
    *out = p;
    return TTS_OK;
}

extern "C" int tts_cross_run(tts_cross* p, const tts_cross_batch* b, const tts_cross_tensors* t)
{
    if (!p || !b || !t || !b->q_len || !b->mem_row || !b->mem_len) return fail(TTS_E_INVAL, "null argument");
    if (b->n < 1 || b->n > TTS_CROSS_MAX_BATCH) return fail(TTS_E_INVAL, "n = %d requests, at most %d per call", b->n, TTS_CROSS_MAX_BATCH);
    long long queries = 0, memory = 0;
    for (int i = 0; i < b->n; ++i) {
        if (b->q_len[i] < 0 || b->q_len[i] > TTS_CROSS_MAX_LEN) return fail(TTS_E_INVAL, "request %d has %d queries", i, b->q_len[i]);
        if (b->mem_len[i] < 0 || b->mem_len[i] > TTS_CROSS_MAX_LEN) return fail(TTS_E_INVAL, "request %d has a memory of %d rows", i, b->mem_len[i]);
        if (b->mem_row[i] < 0 || b->mem_row[i] > (1LL << 40)) return fail(TTS_E_INVAL, "request %d has its memory at row %lld", i, b->mem_row[i]);
        queries += b->q_len[i];
        memory += b->mem_len[i];
    }
    if (queries > 0x7FFFFFFF) return fail(TTS_E_INVAL, "%lld queries in one call", queries);
    const float scale = (t->scale > 0 ? t->scale : 1.0f / sqrtf((float)p->cfg.head_dim)) * 1.4426950408889634f;       // times log2(e)
    if (!(t->scale >= 0 && std::isfinite(scale))) return fail(TTS_E_INVAL, "scale must not be negative, and finite times log2(e)");
    if (queries == 0) return TTS_OK;
    if (!t->q || !t->out || (memory && (!t->k || !t->v))) return fail(TTS_E_INVAL, "null argument");
    struct { const char* name; const void* at; long long stride; int heads; } arrays[4] = {{"q", t->q, t->q_stride, p->cfg.n_heads}, {"k", t->k, t->k_stride, p->cfg.n_kv_heads},
                                                                                       {"v", t->v, t->v_stride, p->cfg.n_kv_heads}, {"out", t->out, t->out_stride, p->cfg.n_heads}};
    long long stride[4];
    for (int i = 0; i < 4; ++i) {
        const long long width = (long long)arrays[i].heads * p->cfg.head_dim;
        stride[i] = arrays[i].stride ? arrays[i].stride : width;
        if (stride[i] < width || stride[i] > (1LL << 24) || stride[i] % 8) return fail(TTS_E_INVAL, "%s: a stride of %lld for %lld columns", arrays[i].name, stride[i], width);
        if (!aligned(arrays[i].at, 16)) return fail(TTS_E_INVAL, "%s must be 16-byte aligned", arrays[i].name);
    }
    if (!aligned(t->lse, 4)) return fail(TTS_E_INVAL, "lse must be 4-byte aligned");
    CrossArgs a;                             // (4 KB; of the requests what is used is filled in)
    a.q = t->q; a.k = t->k; a.v = t->v; a.out = t->out;
    a.keep = t->keep;
    a.lse = t->lse;
    a.parts = p->parts;
    a.zeros = p->zeros;
    a.q_stride = stride[0]; a.k_stride = stride[1]; a.v_stride = stride[2]; a.out_stride = stride[3];
    a.scale = scale;
    a.n_heads = p->cfg.n_heads; a.n_kv_heads = p->cfg.n_kv_heads; a.head_dim = p->cfg.head_dim;
    OnDevice on(p->device);
    HIP_TRY(on.err);
    // two launches' worth: requests of few rows, and of many
    const int group = p->cfg.n_heads / p->cfg.n_kv_heads;
    const bool bf16 = p->cfg.dtype == TTS_DTYPE_BF16;
    long long few_tiles = 0;
    for (int i = 0; i < b->n; ++i) few_tiles += ((long long)b->q_len[i] * group + 15) / 16 * p->cfg.n_kv_heads;
    if (few_tiles > CROSS_MAX_TILES) return fail(TTS_E_INVAL, "%lld tiles of 16 rows in one call", few_tiles);
    const bool any_many = bf16 && cross_many(few_tiles, p->n_cu);
    for (int many = 0; many < 1 + any_many; ++many) {
        int q_row = 0;
        a.n = 0;
        for (int i = 0; i < b->n; ++i) {
            if (b->q_len[i] && (any_many && (long long)b->q_len[i] * group >= CROSS_MANY_ROWS) == many) a.req[a.n++] = CrossReq{b->mem_row[i], b->mem_len[i], q_row, b->q_len[i], 0};
            q_row += b->q_len[i];
            if (a.n == CROSS_BATCH || (a.n && i + 1 == b->n)) {
                HIP_TRY(many ? launch_cross_many(a, p->n_cu, p->stream) : launch_cross_few(a, bf16, p->n_cu, p->stream));
                a.n = 0;
            }
        }
    }
    return TTS_OK;
}

extern "C" void tts_cross_destroy(tts_cross* p) { delete p; }
