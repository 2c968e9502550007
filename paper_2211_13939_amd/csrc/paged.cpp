// Host side of the tts_paged C ABI: argument checks and the batch's way into the launches' arguments.  All arithmetic is in paged.hip.
#include "../../include/tts_paged.h"

#include <hip/hip_runtime.h>

#include <new>

#include "paged_plan.h"
#include "past_host.h"

using namespace tts;

namespace {

int check(const tts_paged_config* c)
{
    if (!c) return fail(TTS_E_INVAL, "config is null");
    if (c->n_heads < 1 || c->n_heads > TTS_CACHE_MAX_HEADS) return fail(TTS_E_INVAL, "n_heads must be in 1..%d", TTS_CACHE_MAX_HEADS);
    if (c->n_kv_heads < 1 || c->n_kv_heads > c->n_heads || c->n_heads % c->n_kv_heads) return fail(TTS_E_INVAL, "n_heads must be a multiple of n_kv_heads");
    if (c->head_dim < 8 || c->head_dim > TTS_CACHE_MAX_HEAD_DIM || c->head_dim % 8)
        return fail(TTS_E_UNSUPPORTED, "kernels are built for head_dim in multiples of 8 up to %d", TTS_CACHE_MAX_HEAD_DIM);
    if (!is_page_rows(c->page_rows, TTS_CACHE_MIN_PAGE, TTS_CACHE_MAX_PAGE))
        return fail(TTS_E_INVAL, "page_rows must be a power of two in %d..%d", TTS_CACHE_MIN_PAGE, TTS_CACHE_MAX_PAGE);
    if (!is_dtype(c->dtype)) return fail(TTS_E_INVAL, "dtype must be 0 (fp32) or 1 (bf16)");
    if (c->causal != 0 && c->causal != 1) return fail(TTS_E_INVAL, "causal must be 0 or 1");
    return TTS_OK;
}

int check_sequence(const char* what, int i, int len, int table_row, int page_shift, const tts_paged_tensors& t)
{
    if (len < 0 || len > TTS_CACHE_MAX_LEN) return fail(TTS_E_INVAL, "%s %d has %d rows", what, i, len);
    if (!len) return TTS_OK;
    if (table_row < 0 || table_row >= t.table_rows) return fail(TTS_E_INVAL, "%s %d has table row %d of %d", what, i, table_row, t.table_rows);
    if ((len - 1) >> page_shift >= t.table_cols) return fail(TTS_E_INVAL, "%s %d has %d rows, a table row %d pages of %d", what, i, len, t.table_cols, 1 << page_shift);
    return TTS_OK;
}

struct Layout { size_t parts, arrived, total; };
size_t part_floats(const tts_paged_config& c) { return paged_room(c.n_kv_heads) * paged_part_floats(PAGED_FEW_ROWS, paged_width(c.head_dim)); }
size_t arrived_bytes(const tts_paged_config& c) { return (size_t)paged_room(c.n_kv_heads) * PAGED_FEW_ROWS * 4; }
Layout layout_of(const tts_paged_config& c)
{
    Layout l;
    Carver a;
    l.parts = a.take(part_floats(c) * 4);
    l.arrived = a.take(arrived_bytes(c));
    l.total = a.off;
    return l;
}

enum class Form { FEW, WHOLE, MANY };                // tiles of 16 rows, prefixes apart if that pays; tiles of 16 over whole sequences; tiles of 128, or of 16 where that takes less

}  // namespace

struct tts_paged {
    tts_paged_config cfg;
    float* parts = nullptr;              // device
    int* arrived = nullptr;
    hipStream_t stream = nullptr;
    int device = 0, n_cu = 0;
};

extern "C" size_t tts_paged_workspace_bytes(const tts_paged_config* cfg)
{
    if (check(cfg) != TTS_OK) return 0;
    return layout_of(*cfg).total;
}

extern "C" int tts_paged_create(const tts_paged_config* cfg, void* dev_arena, size_t arena_bytes, void* hip_stream, tts_paged** out)
{
    if (!out) return fail(TTS_E_INVAL, "out is null");
    *out = nullptr;
    int rc = check(cfg);
    if (rc) return rc;
    int device = 0, n_cu = 0;
    const Layout lay = layout_of(*cfg);
    if ((rc = check_arena(dev_arena, arena_bytes, lay.total, &device))) return rc;
    OnDevice on(device);
    HIP_TRY(on.err);
    HIP_TRY(allow_paged());
    HIP_TRY(fill_now((char*)dev_arena + lay.arrived, 0, arrived_bytes(*cfg)));
    HIP_TRY(hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, device));
    tts_paged* p = new (std::nothrow) tts_paged();
    if (!p) return fail(TTS_E_INVAL, "out of host memory");
    p->cfg = *cfg;
    p->parts = (float*)((char*)dev_arena + lay.parts);
    p->arrived = (int*)((char*)dev_arena + lay.arrived);
    p->stream = (hipStream_t)hip_stream;
    p->device = device;
    p->n_cu = n_cu;
    *out = p;
    return TTS_OK;
}

extern "C" int tts_paged_run(tts_paged* p, const tts_paged_batch* b, const tts_paged_tensors* t)
{
    if (!p || !b || !t || !b->q_len || !b->own_len || !b->table_row) return fail(TTS_E_INVAL, "null argument");
    const tts_paged_config& c = p->cfg;
    if (b->n < 1 || b->n > TTS_CACHE_MAX_BATCH) return fail(TTS_E_INVAL, "n = %d requests, at most %d per call", b->n, TTS_CACHE_MAX_BATCH);
    if (b->n_prefixes < 0 || b->n_prefixes > TTS_PAGED_MAX_PREFIXES) return fail(TTS_E_INVAL, "n_prefixes = %d, at most %d per call", b->n_prefixes, TTS_PAGED_MAX_PREFIXES);
    if (b->n_prefixes && (!b->prefix_len || !b->prefix_table_row)) return fail(TTS_E_INVAL, "null argument");
    if (t->n_pages < 1 || t->table_rows < 1 || t->table_cols < 1) return fail(TTS_E_INVAL, "n_pages, table_rows and table_cols must be positive");
    const int shift = log2_of(c.page_rows), group = c.n_heads / c.n_kv_heads;
    long long queries = 0, keys = 0, few_tiles = 0;
    int rc = TTS_OK;
    for (int g = 0; g < b->n_prefixes; ++g) {
        if ((rc = check_sequence("prefix", g, b->prefix_len[g], b->prefix_table_row[g], shift, *t))) return rc;
        keys += b->prefix_len[g];
    }
    for (int i = 0; i < b->n; ++i) {
        if (b->q_len[i] < 0 || b->q_len[i] > TTS_CACHE_MAX_LEN) return fail(TTS_E_INVAL, "request %d has %d queries", i, b->q_len[i]);
        if ((rc = check_sequence("request", i, b->own_len[i], b->table_row[i], shift, *t))) return rc;
        if (b->prefix && (b->prefix[i] < -1 || b->prefix[i] >= b->n_prefixes)) return fail(TTS_E_INVAL, "request %d has prefix %d of %d", i, b->prefix[i], b->n_prefixes);
        queries += b->q_len[i];
        keys += b->own_len[i];
        few_tiles += ((long long)b->q_len[i] * group + 15) / 16 * c.n_kv_heads;
    }
    if (queries > 0x7FFFFFFF) return fail(TTS_E_INVAL, "%lld queries in one call", queries);
    if (few_tiles > PAGED_MAX_TILES) return fail(TTS_E_INVAL, "%lld tiles of 16 rows in one call", few_tiles);
    const float scale = (t->scale > 0 ? t->scale : 1.0f / sqrtf((float)c.head_dim)) * 1.4426950408889634f;                // times log2(e)
    if (!(t->scale >= 0 && std::isfinite(scale))) return fail(TTS_E_INVAL, "scale must not be negative, and finite times log2(e)");
    if (queries == 0) return TTS_OK;
    if (!t->q || !t->out || (keys && (!t->k_pages || !t->v_pages || !t->table))) return fail(TTS_E_INVAL, "null argument");
    PagedArgs a;                             // (of the arrays what is used is filled in)
    const long long width = (long long)c.n_heads * c.head_dim;
    a.q_stride = t->q_stride;
    a.out_stride = t->out_stride;
    a.page_stride = t->page_stride;
    if ((rc = check_rows("q", t->q, width, a.q_stride)) || (rc = check_rows("out", t->out, width, a.out_stride)) ||
        (rc = check_rows("k_pages", t->k_pages, (long long)c.n_kv_heads * c.page_rows * c.head_dim, a.page_stride)))
        return rc;
    if (!aligned(t->v_pages, 16)) return fail(TTS_E_INVAL, "v_pages must be 16-byte aligned");
    if (!aligned(t->table, 4) || !aligned(t->lse, 4)) return fail(TTS_E_INVAL, "the table and lse must be 4-byte aligned");
    a.q = t->q; a.k_pages = t->k_pages; a.v_pages = t->v_pages; a.out = t->out;
    a.table = t->table;
    a.lse = t->lse;
    a.parts = a.pool_parts = p->parts;
    a.part_floats = (int)part_floats(c);
    a.arrived = p->arrived;
    a.scale = scale;
    a.n_heads = c.n_heads; a.n_kv_heads = c.n_kv_heads; a.head_dim = c.head_dim;
    a.n_pages = t->n_pages; a.table_cols = t->table_cols; a.page_shift = shift;
    a.causal = c.causal;
    // the requests in the order of their prefixes, those without one first (an empty one is none)
    const bool bf16 = c.dtype == TTS_DTYPE_BF16;
    auto prefix_of = [&](int i) { return b->prefix && b->prefix[i] >= 0 && b->prefix_len[b->prefix[i]] > 0 ? b->prefix[i] : -1; };
    int order[TTS_CACHE_MAX_BATCH], q_row[TTS_CACHE_MAX_BATCH], count[TTS_PAGED_MAX_PREFIXES + 2] = {};
    for (int i = 0, at = 0; i < b->n; ++i) {
        q_row[i] = at;
        at += b->q_len[i];
        ++count[prefix_of(i) + 2];
    }
    for (int g = 0; g <= b->n_prefixes; ++g) count[g + 1] += count[g];
    for (int i = 0; i < b->n; ++i) order[count[prefix_of(i) + 1]++] = i;
    auto rows_of = [&](int i) { return (long long)b->q_len[i] * group; };
    // small requests beside large ones are a launch with them, if that is a small one
    bool small = false, large = false;
    for (int i = 0; i < b->n; ++i) {
        const long long rows = rows_of(i);
        small |= rows > 0 && rows < PAGED_MANY_ROWS;
        large |= rows >= PAGED_MANY_ROWS;
    }
    const bool any_many = bf16 && (!small || paged_many(few_tiles, p->n_cu)), any_whole = large && !any_many && few_tiles > 1024;
    auto form_of = [&](int i) {
        return any_many && rows_of(i) >= PAGED_MANY_ROWS ? Form::MANY : rows_of(i) < PAGED_MANY_ROWS || few_tiles <= 1024 ? Form::FEW : Form::WHOLE;
    };
    OnDevice on(p->device);
    HIP_TRY(on.err);
    const int room = paged_room(c.n_kv_heads);
    for (Form form : {Form::FEW, Form::WHOLE, Form::MANY}) {
        if (form == Form::FEW ? !small && (any_many || any_whole) : form == Form::WHOLE ? !any_whole : !any_many || !large) continue;
        auto tiles_of = [&](long long rows) { return (rows + 15) / 16 * c.n_kv_heads; };
        long long tiles = 0;                 // of the requests and of the prefixes before the last one, which need room for a part each
        int last_prefix = -1;
        auto clear = [&]() {
            a.n = a.n_pools = 0;
            a.row[0] = 0;
            tiles = 0;
            last_prefix = -1;
        };
        auto launch = [&]() -> hipError_t {
            if (!a.n) return hipSuccess;
            a.pooled = false;
            a.rows = a.row[a.n];
            a.by_group = (long long)a.rows * group <= 1LL << 32 || (group & (group - 1)) == 0 ? by_of(group) : NOT_BY;
            a.each = a.row[1];
            a.q_first = a.req[0].q_row;
            for (int i = 1; i < a.n; ++i) {
                if (a.row[i + 1] - a.row[i] != a.row[1]) a.each = 0;
                if ((a.req[i].q_row - a.req[i - 1].q_row) * group != a.row[i] - a.row[i - 1]) a.q_first = -1;
            }
            hipError_t e;
            // what the cheapest way should take: prefixes ahead of each request's own rows, as tiles of their own beside them, or as a launch of larger ones; larger tiles for requests, too
            const int bytes = bf16 ? 2 : 4;
            double unique = 0;
            for (int i = 0; i < a.n; ++i) unique += own_len_of(a.req[i]);
            for (int g = 0; g < a.n_pools; ++g) unique += a.pool[g].len;
            unique *= 2.0 * c.n_kv_heads * c.head_dim * bytes;
            PagedCut cut = paged_cut(a, PagedPools::NONE, bytes, p->n_cu, unique, room);
            int height = 0;
            bool many = false;
            if (form != Form::WHOLE && a.n_pools) {
                const PagedCut beside = paged_cut(a, PagedPools::TILES, bytes, p->n_cu, unique, room);
                if (beside.ns < cut.ns) cut = beside;
                height = bf16 ? paged_pool_height(a, p->n_cu) : 0;
                const double pools_ns = height ? paged_pools_ns(a, height, p->n_cu) : 0;
                if (height && pools_ns >= cut.ns) height = 0;
                if (height) {
                    PagedCut apart = paged_cut(a, PagedPools::APART, bytes, p->n_cu, unique, 8 * p->n_cu);
                    apart.ns += pools_ns;
                    if (apart.ns < cut.ns) cut = apart;
                    else height = 0;
                }
            }
            if (form == Form::MANY) {
                const PagedCut larger = paged_many_cut(a, p->n_cu, unique);
                many = larger.ns < cut.ns;
                if (many) cut = larger;
            }
            if (many) {
                plan_paged_many(a, cut);
                e = launch_paged_many(a, PAGED_MANY_HEIGHT, p->stream);
            } else {
                even_parts(a, cut);
                plan_paged_few(a, cut);
                e = launch_paged_few(a, bf16, p->n_cu, p->stream);
                if (e == hipSuccess && height) {
                    plan_paged_pools(a, height, p->n_cu);
                    e = launch_paged_many(a, height, p->stream);
                }
            }
            if (e == hipSuccess && !a.join && ((a.pooled && a.n_pools) || a.share)) e = launch_paged_join(a, bf16, p->stream);
            clear();
            return e;
        };
        clear();
        for (int k = 0; k < b->n; ++k) {
            const int i = order[k], prefix = prefix_of(i);
            if (!b->q_len[i] || form_of(i) != form) continue;
            const bool same = prefix >= 0 && prefix == last_prefix;
            const long long of_last = a.n_pools ? a.row[a.n] - a.row[a.pool[a.n_pools - 1].begin] : 0, mine = tiles_of(rows_of(i));
            const long long of_prefixes = same ? tiles_of(of_last + rows_of(i)) : tiles_of(of_last) + (prefix >= 0 ? mine : 0);
            if (a.n == PAGED_BATCH || (prefix >= 0 && !same && a.n_pools == PAGED_POOLS) || (form == Form::FEW && a.n && tiles + mine + of_prefixes > room)) HIP_TRY(launch());
            if (prefix >= 0 && prefix != last_prefix) {
                if (a.n_pools) tiles += tiles_of(of_last);
                a.pool[a.n_pools++] = PagedPool{b->prefix_table_row[prefix], b->prefix_len[prefix], a.n, a.n, 0};
                last_prefix = prefix;
            }
            a.req[a.n] = PagedReq{(unsigned)b->own_len[i] | (unsigned)(prefix >= 0 ? a.n_pools : 0) << 25, b->table_row[i], q_row[i], 0};
            a.row[a.n + 1] = a.row[a.n] + (int)rows_of(i);
            ++a.n;
            if (prefix >= 0) a.pool[a.n_pools - 1].end = a.n;
            tiles += mine;
        }
        HIP_TRY(launch());
    }
    return TTS_OK;
}

extern "C" void tts_paged_destroy(tts_paged* p) { delete p; }
