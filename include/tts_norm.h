/*
 * tts_norm.h -- C ABI of the norm in front of a block's products: the residual's addition, the root-mean-square
 * norm and its output, in 8 bits with scales if the next product takes them (tts_linear8.h), in one pass:
 *
 *     total = x + res
 *     y     = gain * total / sqrt(mean(total^2) + eps)         (mean over the dim columns of a row)
 *
 * TTS_NORM_NONE leaves the second line out (y = total): the rounding to 8 bits alone, for rows that need no norm
 * (F_enc on its way to keys and values, attention's output).
 *
 * 8-bit rows.  y8 holds e4m3 numbers (4 exponent bits, bias 7, 3 mantissa bits, no infinity), scales a power of
 * two for each 128 columns of a row, as a byte: 2^(byte - 127).  Of a block whose largest magnitude is m the scale is the
 * least power of two, from 2^-127 up, with m <= 448 * scale (1 where m = 0), so that dividing by it is exact and the one
 * rounding is that to e4m3, to nearest even, from the unrounded y.  An infinity or NaN in y becomes NaN and does
 * not count for the scale.
 * y8 rows are TTS_WIDTH8(dim) bytes: columns past dim are zeros.  scales rows are TTS_SCALE_COLUMNS(dim) bytes: what lies
 * past the last block is 127.
 *
 * Sums are fp32, formed in an order that depends on dim and the number of rows alone (calls of many rows have another: a row may differ
 * there in its last bits).  Of a row whose squares leave fp32's range they are those of the row times a power of two, so that rows of any finite
 * magnitude have their norm; a row of zeros without an eps is NaN, as is one with a NaN.  Everything is queued on the stream given
 * at creation; device memory comes from the caller's arena; nothing is allocated on the device.  A call is one
 * launch and may be captured into a graph.  Conventions as in tts_pool.h: 0 on success, negative tts_status otherwise,
 * text in tts_last_error(); one owner thread per object.
 */
#ifndef TTS_NORM_H
#define TTS_NORM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tts_norm tts_norm;

#define TTS_SCALE_BLOCK 128                                                      /* columns under one scale */
#define TTS_WIDTH8(dim) (((dim) + 127) / 128 * 128)                              /* bytes of an 8-bit row */
#define TTS_SCALE_COLUMNS(dim) ((TTS_WIDTH8(dim) / 128 + 3) / 4 * 4)             /* bytes of its scales: whole words */
#define TTS_NORM_MAX_DIM 16384
#define TTS_MAX_ROWS (1 << 24)                                                   /* rows of one call, here and in tts_linear8.h */

enum { TTS_NORM_RMS = 0, TTS_NORM_NONE = 1 };

typedef struct {
    int dim;          /* columns of a row, 1 .. TTS_NORM_MAX_DIM */
    int kind;         /* TTS_NORM_RMS / TTS_NORM_NONE */
    int x_dtype;      /* TTS_DTYPE_F32 / TTS_DTYPE_BF16 of tts_pool.h (0 / 1) */
    int res_dtype;    /* of res and total (0 / 1) */
    int y_dtype;      /* of y (0 / 1) */
    float eps;        /* >= 0, finite; TTS_NORM_NONE does not use it */
} tts_norm_config;

/* One call.  DEVICE pointers; a stride is the distance between rows in elements (0: dim, the rows lie back to back), y8 and
 * scales rows always lie back to back.  Arrays begin at a multiple of their element, y8 at one of 16 bytes, scales at one of 4.
 * total may be res or x itself, y may be x, each with its type and stride; otherwise no two arrays overlap. */
typedef struct {
    int rows;                                 /* 0 .. TTS_MAX_ROWS; 0 does nothing */
    const void *x;     long long x_stride;
    const void *res;   long long res_stride;  /* null: total = x */
    void *total;       long long total_stride;/* null: not wanted; rounded from fp32 if it is bf16 */
    void *y;           long long y_stride;    /* null: not wanted */
    void *y8;                                 /* null: not wanted; both or neither of these two */
    void *scales;
} tts_norm_rows;

/* Bytes of device memory tts_norm_create needs for this configuration (0 if the configuration is invalid). */
size_t tts_norm_workspace_bytes(const tts_norm_config *cfg);

/*
 * Create a norm.  gain: HOST fp32 [dim], copied (TTS_NORM_NONE: null).  `dev_arena` is DEVICE memory of at least
 * tts_norm_workspace_bytes(cfg) bytes, 256-byte aligned, owned by the caller and kept alive until tts_norm_destroy.
 * `hip_stream` is a hipStream_t.
 */
int tts_norm_create(const tts_norm_config *cfg, const float *gain, void *dev_arena, size_t arena_bytes, void *hip_stream,
                    tts_norm **out);

/*
 * One batch of rows, asynchronous on the stream.  Errors: TTS_E_INVAL for null pointers (x, or every output),
 * a number of rows outside its range, a stride below dim or above 2^40, an array that is not aligned as above, or one of y8 and scales
 * without the other.
 */
int tts_norm_run(tts_norm *norm, const tts_norm_rows *rows);

/* Does not wait: the arena stays the caller's to keep until the calls that were queued, and graphs that hold any, have run. */
void tts_norm_destroy(tts_norm *norm);

#ifdef __cplusplus
}
#endif
#endif
