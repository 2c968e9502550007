/*
 * tts_paged.h -- C ABI of attention to a paged cache (tts_cache.h): queries of a dynamic batch of requests, each of which attends the rows of its own that lie there and, ahead of them, those of a
 * prefix that it may share with others (a voice's recording, a common beginning).  Cross attention (tts_cross.h) is the one to memories that lie in one piece and that every query
 * sees whole.  For request i with own_len rows and q_len queries, query t and head h
 *
 *     keys    rows 0 .. prefix_len - 1 of its prefix, if it has one; rows j of its own, j <= own_len - q_len + t if causal, all of them otherwise
 *     w[j]      = softmax over the keys of scale * (q[t][h] . k[j][g])                    g = h / (n_heads / n_kv_heads)
 *     out[t][h] = sum over the keys of w[j] * v[j][g]
 *     lse[t][h] = log sum over the keys of exp(scale * (q[t][h] . k[j][g]))
 *
 * (the queries are those of the last q_len rows, which have been appended; with more queries than rows the first ones see no row of their own).  Rows whose page number is outside
 * 0 .. n_pages - 1 (pages given back, say) are no keys.  Where no key is left out is 0 and lse is -infinity.  What a query does not see is not used for it, whatever
 * it is (infinities and NaN included).
 *
 * A prefix that several requests with few rows (pairs of a query and a head of its group) share is read once for all of them, and joined with what their own rows give.
 *
 * Sums, the softmax's maximum and sum, the outputs' sums and what is joined are fp32; bf16 weights w are rounded to bf16 for their product with v (relative error up to 2^-8 each).  The
 * order of a request's sums follows from all numbers of the call (what is read apart and in which parts, and which kernel takes it): a call repeats itself bit for bit, but a request in other company may
 * differ in its last bits.  Everything is queued on the stream given at creation; device memory comes from the caller's arena; nothing is allocated on the
 * device.  The batch's numbers travel with the launches: a call may be captured, and its graph holds them, but reads the table anew.  Parts meet in the arena: calls of one object run
 * one after another, as they do on its stream, and so do graphs that hold them.
 * Conventions as in tts_pool.h: 0 on success, negative tts_status otherwise, text in tts_last_error(); one owner thread per object.
 */
#ifndef TTS_PAGED_H
#define TTS_PAGED_H

#include "tts_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tts_paged tts_paged;

#define TTS_PAGED_MAX_PREFIXES 1024      /* of one call */

typedef struct {
    int n_heads;      /* 1 .. TTS_CACHE_MAX_HEADS, a multiple of n_kv_heads */
    int n_kv_heads;   /* heads of k and v */
    int head_dim;     /* a multiple of 8, 8 .. TTS_CACHE_MAX_HEAD_DIM */
    int page_rows;    /* a power of two, TTS_CACHE_MIN_PAGE .. TTS_CACHE_MAX_PAGE */
    int dtype;        /* of q, the cache and out: TTS_DTYPE_F32 / TTS_DTYPE_BF16 of tts_pool.h (0 / 1) */
    int causal;       /* 0 / 1 */
} tts_paged_config;

/* HOST arrays: of n where nothing else is said; the queries of the requests lie back to back. */
typedef struct {
    int n;                        /* 1 .. TTS_CACHE_MAX_BATCH */
    const int *q_len;             /* 0 .. TTS_CACHE_MAX_LEN */
    const int *own_len;           /* 0 .. TTS_CACHE_MAX_LEN */
    const int *table_row;         /* of its own rows; not used where own_len is 0 */
    const int *prefix;            /* 0 .. n_prefixes - 1, -1: none; null: none has one */
    int n_prefixes;               /* 0 .. TTS_PAGED_MAX_PREFIXES */
    const int *prefix_len;        /* [n_prefixes] 0 .. TTS_CACHE_MAX_LEN */
    const int *prefix_table_row;  /* [n_prefixes] not used where prefix_len is 0 */
} tts_paged_batch;

/* DEVICE pointers.  A row of q and out holds n_heads * head_dim elements; strides are distances in elements, multiples of 8: of rows at most 2^40 (0: back to back), of pages at most 2^40
 * (0: n_kv_heads * page_rows * head_dim).  q, out and the pages are 16-byte aligned, the table and lse by 4.  out and lse overlap nothing. */
typedef struct {
    const void *q;      long long q_stride;
    const void *k_pages, *v_pages;
    long long page_stride;                        /* of both */
    int n_pages;                                  /* 1 .. */
    const int *table;                             /* [table_rows][table_cols] */
    int table_rows, table_cols;                   /* 1 .. */
    void *out;          long long out_stride;
    float *lse;                                   /* fp32 [queries][n_heads]; null: not wanted */
    float scale;                                  /* > 0, at most 2^127; 0: 1 / sqrt(head_dim) */
} tts_paged_tensors;

/* Bytes of device memory tts_paged_create needs for this configuration (0 if the configuration is invalid). */
size_t tts_paged_workspace_bytes(const tts_paged_config *cfg);

/*
 * Create an attention.  `dev_arena` is DEVICE memory of at least tts_paged_workspace_bytes(cfg) bytes, 256-byte aligned,
 * owned by the caller and kept alive until tts_paged_destroy.  `hip_stream` is a hipStream_t.
 */
int tts_paged_create(const tts_paged_config *cfg, void *dev_arena, size_t arena_bytes, void *hip_stream, tts_paged **out);

/*
 * Attend, asynchronously on the stream (the batch's arrays are consumed before the call returns).  Errors: TTS_E_INVAL for null pointers, a number outside its range, a sequence that the table has no row
 * or not enough columns for, more than 2^31 - 1 queries or 2^23 tiles in all (a tile: 16 pairs of a query and a head, of one request and one head of k), a stride that is too
 * small, too large or no multiple of 8, an array that is not aligned as above, or a scale that is negative or, times log2(e), not finite.
 */
int tts_paged_run(tts_paged *att, const tts_paged_batch *batch, const tts_paged_tensors *tensors);

/* Does not wait: the arena stays the caller's to keep until the calls that were queued, and graphs that hold any, have run. */
void tts_paged_destroy(tts_paged *att);

#ifdef __cplusplus
}
#endif
#endif
