/*
 * tts_cache.h -- C ABI of the way into a paged cache: new rows of keys and values of a dynamic batch go behind the rows that their requests have there
 * already, keys turned to their positions on the way (tts_rotary.h), and queries, if there are any, beside them in the same launch.  tts_paged.h attends the cache.
 *
 * A cache is two arrays of pages, of keys and of values, [n_pages][n_kv_heads][page_rows][head_dim], and a table of page numbers [table_rows][table_cols]:
 * row r of a sequence whose table row is T lies in page table[T][r / page_rows], at row r % page_rows of it.  All three are the caller's, who hands out pages:
 * a page number outside 0 .. n_pages - 1 (-1, say) is no page, and rows that would go there are not written.  Nothing but the new rows is written.
 * No two rows of a call go to one place: its requests' rows do not overlap where table rows are equal (which the call checks), and a table that is appended to has
 * each page once among what the call writes (which it cannot).
 *
 * The batch's numbers travel with the launches: a call may be captured, and its graph holds them, but reads the table anew.  Everything is queued on the stream given at creation;
 * device memory comes from the caller's arena; nothing is allocated on the device.  What a row becomes does not depend on the others.
 * Conventions as in tts_pool.h: 0 on success, negative tts_status otherwise, text in tts_last_error(); one owner thread per object.
 */
#ifndef TTS_CACHE_H
#define TTS_CACHE_H

#include "tts_rotary.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tts_cache tts_cache;

#define TTS_CACHE_MAX_HEADS 256
#define TTS_CACHE_MAX_HEAD_DIM 128
#define TTS_CACHE_MIN_PAGE 16            /* rows of a page: a power of two from here .. */
#define TTS_CACHE_MAX_PAGE 1024          /* .. to here */
#define TTS_CACHE_MAX_BATCH 1024         /* requests in one call */
#define TTS_CACHE_MAX_LEN (1 << 24)      /* rows of one sequence */

typedef struct {
    int n_kv_heads;       /* 1 .. TTS_CACHE_MAX_HEADS */
    int n_heads;          /* of queries, 0 .. TTS_CACHE_MAX_HEADS; 0: none come along */
    int head_dim;         /* a multiple of 8, 8 .. TTS_CACHE_MAX_HEAD_DIM */
    int page_rows;        /* a power of two, TTS_CACHE_MIN_PAGE .. TTS_CACHE_MAX_PAGE */
    int x_dtype;          /* of k, v and q: TTS_DTYPE_F32 / TTS_DTYPE_BF16 of tts_pool.h (0 / 1) */
    int dtype;            /* of the cache and q_out */
    tts_rotary_angles angles;     /* rot_dim 0: nothing turns */
} tts_cache_config;

/* HOST arrays of n: the new rows of the requests lie back to back. */
typedef struct {
    int n;                        /* 1 .. TTS_CACHE_MAX_BATCH */
    const int *len;               /* new rows, 0 .. TTS_CACHE_MAX_LEN */
    const int *row;               /* where the first of them goes: rows that the sequence has; row + len at most TTS_CACHE_MAX_LEN */
    const int *table_row;         /* the sequence's row of the table */
    const int *position;          /* of the first new row, position + len within what 32 bits hold; null: row */
} tts_cache_batch;

/* DEVICE pointers.  A row of k and v holds n_kv_heads * head_dim elements, one of q and q_out n_heads * head_dim; strides are distances in elements, multiples of 8: of rows at
 * most 2^40 (0: back to back), of pages at most 2^40 (0: n_kv_heads * page_rows * head_dim).  k, v, q, q_out and the pages are 16-byte aligned, the table is by 4.
 * q_out may be q, with its type and stride; otherwise nothing that is written overlaps anything else. */
typedef struct {
    const void *k;      long long k_stride;
    const void *v;      long long v_stride;
    const void *q;      long long q_stride;       /* both null: no queries come along */
    void *q_out;        long long q_out_stride;
    void *k_pages, *v_pages;
    long long page_stride;                        /* of both */
    int n_pages;                                  /* 1 .. */
    const int *table;
    int table_rows, table_cols;                   /* 1 .. */
} tts_cache_tensors;

/* Bytes of device memory tts_cache_create needs for this configuration (0 if the configuration is invalid). */
size_t tts_cache_workspace_bytes(const tts_cache_config *cfg);

/*
 * Create an appender.  `dev_arena` is DEVICE memory of at least tts_cache_workspace_bytes(cfg) bytes, 256-byte aligned,
 * owned by the caller and kept alive until tts_cache_destroy.  `hip_stream` is a hipStream_t.
 */
int tts_cache_create(const tts_cache_config *cfg, void *dev_arena, size_t arena_bytes, void *hip_stream, tts_cache **out);

/*
 * Append, asynchronously on the stream (the batch's arrays are consumed before the call returns).  Errors: TTS_E_INVAL for null pointers, a number outside its range, more than
 * TTS_ROTARY_MAX_ROWS rows in all, a sequence that the table has no row or not enough columns for, requests whose rows overlap in one table row, a stride that is too small, too large or no multiple of
 * 8, an array that is not aligned as above, one of q and q_out without the other, queries where n_heads is 0, or q_out at q with another type or stride.
 */
int tts_cache_run(tts_cache *cache, const tts_cache_batch *batch, const tts_cache_tensors *tensors);

/* Does not wait: the arena stays the caller's to keep until the calls that were queued, and graphs that hold any, have run. */
void tts_cache_destroy(tts_cache *cache);

#ifdef __cplusplus
}
#endif
#endif
