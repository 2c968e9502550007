/*
 * tts_cross.h -- C ABI of cross attention to the encoder's states: queries of a dynamic batch of requests, each of which attends
 * its own memory, of another length than its queries (the pool's attention, tts_pool.h, is the location-sensitive one of a single
 * query; this one has several heads and any number of queries).  For request i, query t and head h
 *
 *     w[j]      = softmax over j of scale * (q[t][h] . k[j][g])        j < mem_len[i], keep[j] != 0
 *     out[t][h] = sum over j of w[j] * v[j][g]                          g = h / (n_heads / n_kv_heads)
 *     lse[t][h] = log sum over j of exp(scale * (q[t][h] . k[j][g]))
 *
 * Where nothing is left to attend (mem_len 0, or every position hidden) out is 0 and lse is -infinity.  What lies in hidden positions
 * and behind a request's memory is not used, whatever it is (infinities and NaN included).
 *
 * Sums, the softmax's maximum and sum and the outputs' sums are fp32; bf16 weights w are rounded to bf16 for their
 * product with v (relative error up to 2^-8 each).  The order of a request's sums follows from all lengths of the call (whether its memory is read in
 * parts, and of which length, and which kernel takes it): a call repeats itself bit for bit, but a request in other company may differ in its last bits, unlike in the
 * pool.  One call = one dynamic batch of requests of any lengths, from one query (a
 * step) to many (all frames at once).  Everything is queued on the stream given at creation; device memory comes from the caller's
 * arena; nothing is allocated on the device.  The lengths travel with the launches: a call may be captured, and its
 * graph holds the lengths it was captured with.  Long memories that few queries attend are split, and the parts
 * meet in the arena: calls of one object run one after another, as they do on its stream, and so do graphs that hold them.
 * Conventions as in tts_pool.h: 0 on success, negative tts_status otherwise, text in tts_last_error(); one owner
 * thread per object.
 */
#ifndef TTS_CROSS_H
#define TTS_CROSS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tts_cross tts_cross;

#define TTS_CROSS_MAX_HEADS 256
#define TTS_CROSS_MAX_HEAD_DIM 128
#define TTS_CROSS_MAX_BATCH 1024         /* requests in one call */
#define TTS_CROSS_MAX_LEN (1 << 24)      /* queries, or memory rows, of one request */

typedef struct {
    int n_heads;      /* 1 .. TTS_CROSS_MAX_HEADS, a multiple of n_kv_heads */
    int n_kv_heads;   /* heads of k and v */
    int head_dim;     /* a multiple of 8, 8 .. TTS_CROSS_MAX_HEAD_DIM */
    int dtype;        /* of q, k, v and out: TTS_DTYPE_F32 / TTS_DTYPE_BF16 of tts_pool.h (0 / 1) */
} tts_cross_config;

/* HOST arrays of n: the queries of the requests lie back to back; request i's memory is rows mem_row[i] .. + mem_len[i] of k and v
 * (slots of a fixed size, or memories back to back; several requests may share one). */
typedef struct {
    int n;                        /* 1 .. TTS_CROSS_MAX_BATCH */
    const int *q_len;             /* 0 .. TTS_CROSS_MAX_LEN */
    const long long *mem_row;     /* 0 .. 2^40 */
    const int *mem_len;           /* 0 .. TTS_CROSS_MAX_LEN */
} tts_cross_batch;

/* DEVICE pointers.  A row of q and out holds n_heads * head_dim elements, one of k and v n_kv_heads * head_dim; a stride is the distance between
 * rows in elements, a multiple of 8, at most 2^24 (0: the rows lie back to back).  q, k, v and out are
 * 16-byte aligned; k and v may be null where every mem_len is 0.  out and lse overlap nothing. */
typedef struct {
    const void *q;  long long q_stride;
    const void *k;  long long k_stride;
    const void *v;  long long v_stride;
    void *out;      long long out_stride;
    const unsigned char *keep;    /* a byte for each memory row (of all of them, indexed as k), 0 = hidden; null: none is */
    float *lse;                   /* fp32 [queries][n_heads], 4-byte aligned; null: not wanted */
    float scale;                  /* > 0, at most 2^127; 0: 1 / sqrt(head_dim) */
} tts_cross_tensors;

/* Bytes of device memory tts_cross_create needs for this configuration (0 if the configuration is invalid). */
size_t tts_cross_workspace_bytes(const tts_cross_config *cfg);

/*
 * Create an attention.  `dev_arena` is DEVICE memory of at least tts_cross_workspace_bytes(cfg) bytes, 256-byte aligned,
 * owned by the caller and kept alive until tts_cross_destroy.  `hip_stream` is a hipStream_t.
 */
int tts_cross_create(const tts_cross_config *cfg, void *dev_arena, size_t arena_bytes, void *hip_stream, tts_cross **out);

/*
 * Attend, asynchronously on the stream (the batch's arrays are consumed before the call returns).
 * Errors: TTS_E_INVAL for null pointers, a number of requests, a length or a row outside its range, more than 2^31 - 1 queries or 2^23 tiles in all
 * (a tile: 16 pairs of a query and a head, of one request and one head of k),
 * a stride that is too small, too large or no multiple of 8, an array that is not aligned, or a scale that is negative or, times log2(e), not finite.
 */
int tts_cross_run(tts_cross *att, const tts_cross_batch *batch, const tts_cross_tensors *tensors);

/* Does not wait: the arena stays the caller's to keep until the calls that were queued, and graphs that hold any, have run. */
void tts_cross_destroy(tts_cross *att);

#ifdef __cplusplus
}
#endif
#endif
