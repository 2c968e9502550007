// Host side of the tts_cache C ABI: argument checks and the batch's way into the launches' arguments.  All arithmetic is in rotary.hip.
#include "../../include/tts_cache.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>

#include "past_host.h"

using namespace tts;

namespace {

int check(const tts_cache_config* c)
{
    if (!c) return fail(TTS_E_INVAL, "config is null");
    if (c->n_kv_heads < 1 || c->n_kv_heads > TTS_CACHE_MAX_HEADS) return fail(TTS_E_INVAL, "n_kv_heads must be in 1..%d", TTS_CACHE_MAX_HEADS);
    if (c->n_heads < 0 || c->n_heads > TTS_CACHE_MAX_HEADS) return fail(TTS_E_INVAL, "n_heads must be in 0..%d", TTS_CACHE_MAX_HEADS);
    if (c->head_dim < 8 || c->head_dim > TTS_CACHE_MAX_HEAD_DIM || c->head_dim % 8)
        return fail(TTS_E_UNSUPPORTED, "kernels are built for head_dim in multiples of 8 up to %d", TTS_CACHE_MAX_HEAD_DIM);
    if (!is_page_rows(c->page_rows, TTS_CACHE_MIN_PAGE, TTS_CACHE_MAX_PAGE))
        return fail(TTS_E_INVAL, "page_rows must be a power of two in %d..%d", TTS_CACHE_MIN_PAGE, TTS_CACHE_MAX_PAGE);
    if (!is_dtype(c->x_dtype) || !is_dtype(c->dtype)) return fail(TTS_E_INVAL, "dtypes must be 0 (fp32) or 1 (bf16)");
    return c->angles.rot_dim == 0 ? TTS_OK : check_angles(c->angles, c->head_dim);
}

struct Span { int table_row, first, last; };

// Whether two requests' rows meet in a table row (an empty request has none).  `spans`: room for all of them.
bool rows_meet(const tts_cache_batch& b, Span* spans)
{
    int n = 0;
    bool in_order = true;
    for (int i = 0; i < b.n; ++i) {
        if (!b.len[i]) continue;
        spans[n++] = {b.table_row[i], b.row[i], b.row[i] + b.len[i]};
        in_order &= n < 2 || spans[n - 2].table_row < spans[n - 1].table_row;
    }
    if (in_order) return false;
    std::sort(spans, spans + n, [](const Span& x, const Span& y) { return x.table_row != y.table_row ? x.table_row < y.table_row : x.first < y.first; });
    for (int i = 1; i < n; ++i)
        if (spans[i].table_row == spans[i - 1].table_row && spans[i].first < spans[i - 1].last) return true;
    return false;
}

}  // namespace

struct tts_cache {
    tts_cache_config cfg;
    const uint64_t* freqs = nullptr;     // device
    hipStream_t stream = nullptr;
    int device = 0, n_cu = 0;
};

extern "C" size_t tts_cache_workspace_bytes(const tts_cache_config* cfg)
{
    if (check(cfg) != TTS_OK) return 0;
    Carver a;
    a.take(std::max<size_t>(1, (size_t)cfg->angles.rot_dim / 2 * 8));
    return a.off;
}

extern "C" int tts_cache_create(const tts_cache_config* cfg, void* dev_arena, size_t arena_bytes, void* hip_stream, tts_cache** out)
{
    if (!out) return fail(TTS_E_INVAL, "out is null");
    *out = nullptr;
    int rc = check(cfg);
    if (rc) return rc;
    int device = 0, n_cu = 0;
    if ((rc = check_arena(dev_arena, arena_bytes, tts_cache_workspace_bytes(cfg), &device))) return rc;
    OnDevice on(device);
    HIP_TRY(on.err);
    HIP_TRY(hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, device));
    if (cfg->angles.rot_dim) {
        try {
            const std::vector<uint64_t> freqs = turn_freqs(cfg->angles);
            HIP_TRY(hipMemcpy(dev_arena, freqs.data(), freqs.size() * 8, hipMemcpyHostToDevice));
        } catch (const std::bad_alloc&) {
            return fail(TTS_E_INVAL, "out of host memory");
        }
    }
    tts_cache* p = new (std::nothrow) tts_cache();
    if (!p) return fail(TTS_E_INVAL, "out of host memory");
    p->cfg = *cfg;
    if (!cfg->angles.rot_dim) p->cfg.angles = tts_rotary_angles{};
    p->freqs = (const uint64_t*)dev_arena;
    p->stream = (hipStream_t)hip_stream;
    p->device = device;
    p->n_cu = n_cu;
    *out = p;
    return TTS_OK;
}

extern "C" int tts_cache_run(tts_cache* p, const tts_cache_batch* b, const tts_cache_tensors* t)
{
    if (!p || !b || !t || !b->len || !b->row || !b->table_row) return fail(TTS_E_INVAL, "null argument");
    const tts_cache_config& c = p->cfg;
    if (b->n < 1 || b->n > TTS_CACHE_MAX_BATCH) return fail(TTS_E_INVAL, "n = %d requests, at most %d per call", b->n, TTS_CACHE_MAX_BATCH);
    if (t->n_pages < 1 || t->table_rows < 1 || t->table_cols < 1) return fail(TTS_E_INVAL, "n_pages, table_rows and table_cols must be positive");
    const int shift = log2_of(c.page_rows);
    long long rows = 0;
    for (int i = 0; i < b->n; ++i) {
        if (b->len[i] < 0 || b->len[i] > TTS_CACHE_MAX_LEN) return fail(TTS_E_INVAL, "request %d has %d rows", i, b->len[i]);
        if (b->row[i] < 0 || b->row[i] > TTS_CACHE_MAX_LEN - b->len[i]) return fail(TTS_E_INVAL, "request %d has %d rows from row %d on", i, b->len[i], b->row[i]);
        if (!b->len[i]) continue;
        if (b->table_row[i] < 0 || b->table_row[i] >= t->table_rows) return fail(TTS_E_INVAL, "request %d has table row %d of %d", i, b->table_row[i], t->table_rows);
        if ((b->row[i] + b->len[i] - 1) >> shift >= t->table_cols) return fail(TTS_E_INVAL, "request %d ends at row %d, a table row has %d pages of %d", i, b->row[i] + b->len[i], t->table_cols, c.page_rows);
        if (b->position && (long long)b->position[i] + b->len[i] > (1LL << 31)) return fail(TTS_E_INVAL, "request %d's positions go past 32 bits", i);
        rows += b->len[i];
    }
    if (rows > TTS_ROTARY_MAX_ROWS) return fail(TTS_E_INVAL, "%lld rows, at most %d per call", rows, TTS_ROTARY_MAX_ROWS);
    Span spans[TTS_CACHE_MAX_BATCH];
    if (rows_meet(*b, spans)) return fail(TTS_E_INVAL, "two requests' rows go to the same place");
    if (!t->q != !t->q_out) return fail(TTS_E_INVAL, "q and q_out come together");
    if (t->q && !c.n_heads) return fail(TTS_E_INVAL, "queries, but n_heads is 0");
    if (rows == 0) return TTS_OK;
    if (!t->k || !t->v || !t->k_pages || !t->v_pages || !t->table) return fail(TTS_E_INVAL, "null argument");
    AppendArgs a;                            // (of the requests what is used is filled in)
    a.k_stride = t->k_stride; a.v_stride = t->v_stride; a.q_stride = t->q_stride; a.q_out_stride = t->q_out_stride; a.page_stride = t->page_stride;
    const long long kv_width = (long long)c.n_kv_heads * c.head_dim, q_width = (long long)c.n_heads * c.head_dim;
    int rc = check_rows("k", t->k, kv_width, a.k_stride);
    if (!rc) rc = check_rows("v", t->v, kv_width, a.v_stride);
    if (!rc) rc = check_rows("k_pages", t->k_pages, kv_width * c.page_rows, a.page_stride);
    if (!rc && t->q) rc = check_rows("q", t->q, q_width, a.q_stride);
    if (!rc && t->q) rc = check_rows("q_out", t->q_out, q_width, a.q_out_stride);
    if (rc) return rc;
    if (!aligned(t->v_pages, 16)) return fail(TTS_E_INVAL, "v_pages must be 16-byte aligned");
    if (!aligned(t->table, 4)) return fail(TTS_E_INVAL, "the table must be 4-byte aligned");
    if (t->q && t->q == t->q_out && (a.q_stride != a.q_out_stride || c.x_dtype != c.dtype)) return fail(TTS_E_INVAL, "q_out is q, but with another type or stride");
    a.k_pages = t->k_pages; a.v_pages = t->v_pages;
    a.table = t->table;
    a.turn = turn_angles(c.angles, c.head_dim, p->freqs);
    a.heads = c.n_heads; a.kv_heads = c.n_kv_heads; a.head_dim = c.head_dim;
    a.n_pages = t->n_pages; a.table_cols = t->table_cols; a.page_shift = shift;
    const bool x_bf16 = c.x_dtype == TTS_DTYPE_BF16, bf16 = c.dtype == TTS_DTYPE_BF16;
    OnDevice on(p->device);
    HIP_TRY(on.err);
    long long from = 0;                      // the launch's first row
    a.n = a.rows = 0;
    for (int i = 0; i < b->n; ++i) {
        if (b->len[i]) {
            a.req[a.n++] = AppendReq{a.rows, b->row[i], b->table_row[i], b->position ? b->position[i] : b->row[i]};
            a.rows += b->len[i];
        }
        if (a.n == APPEND_BATCH || (a.n && i + 1 == b->n)) {
            auto rows_from = [&](const void* at, long long stride, int dtype) { return (const char*)at + from * stride * dtype_bytes(dtype); };
            a.k = rows_from(t->k, a.k_stride, c.x_dtype);
            a.v = rows_from(t->v, a.v_stride, c.x_dtype);
            a.q = t->q ? rows_from(t->q, a.q_stride, c.x_dtype) : nullptr;
            a.q_out = t->q ? (void*)rows_from(t->q_out, a.q_out_stride, c.dtype) : nullptr;
            HIP_TRY(launch_append(a, x_bf16, bf16, p->n_cu, p->stream));
            from += a.rows;
            a.n = a.rows = 0;
        }
    }
    return TTS_OK;
}

extern "C" void tts_cache_destroy(tts_cache* p) { delete p; }
