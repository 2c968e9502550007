/*
 * tts_linear8.h -- C ABI of the matrix product of 8-bit rows with 8-bit weights, each with a scale for every 128
 * columns of a row:
 *
 *     y[m][n] = bias[n] + sum over blocks b of sx[m][b] * sw[n][b] * (sum over the block's columns k of x8[m][k] * w8[n][k])
 *
 * x8 and its scales are those that tts_norm_run writes (e4m3 and powers of two; the layout stands in tts_norm.h).  The
 * weights are given in fp32 and rounded in the same way at creation: a scale for each 128 input columns of an output
 * channel.  The products of e4m3 numbers are summed by the matrix instructions, which apply the scales themselves.
 *
 * With y in bf16 the sums are the 8-bit instructions' (fp32 results; within an instruction of 128 columns, terms are
 * aligned to the largest: an error of some 1.4e-5 of the result, where bf16's rounding is up to 2^-8).  With y in fp32 the operands are
 * brought to bf16 together with their scales, and the sums are fp32 throughout, at up to half the rate.  bf16 holds every e4m3 number times
 * a scale from 2^-124 to 2^119 exactly.  In blocks whose largest magnitude is at most 448 * 2^-125, of either operand, it rounds operands to multiples
 * of 2^-133; in those where it is above 448 * 2^119 (2.98e38) numbers of 256 * 2^120 and more become infinite.  bf16 results know no such limits.
 *
 * The order of a row's sums is fixed for a number of rows, in_dim and out_dim, and another for some other numbers of rows (the kernel's tiles follow from
 * them): a call repeats itself bit for bit, but a row in a call of more or fewer rows may differ in its last bits, unlike in the pool, whose requests do not depend on each other.
 *
 * Everything is queued on the stream given at creation; device memory comes from the caller's arena; nothing is
 * allocated on the device.  A call is one launch and may be captured into a graph.
 * Conventions as in tts_pool.h: 0 on success, negative tts_status otherwise, text in tts_last_error(); one owner
 * thread per object.
 */
#ifndef TTS_LINEAR8_H
#define TTS_LINEAR8_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tts_linear8 tts_linear8;

#define TTS_LINEAR8_MAX_DIM 65536

typedef struct {
    int in_dim;       /* columns of a row of x, 1 .. TTS_LINEAR8_MAX_DIM */
    int out_dim;      /* columns of a row of y, 1 .. TTS_LINEAR8_MAX_DIM */
    int y_dtype;      /* TTS_DTYPE_F32 / TTS_DTYPE_BF16 of tts_pool.h (0 / 1) */
} tts_linear8_config;

/* Bytes of device memory tts_linear8_create needs for this configuration (0 if the configuration is invalid). */
size_t tts_linear8_workspace_bytes(const tts_linear8_config *cfg);

/*
 * Create a product.  w: HOST fp32 [out_dim][in_dim], bias: HOST fp32 [out_dim] or null; both are copied.  `dev_arena` is
 * DEVICE memory of at least tts_linear8_workspace_bytes(cfg) bytes, 256-byte aligned, owned by the caller and kept
 * alive until tts_linear8_destroy.  `hip_stream` is a hipStream_t.
 */
int tts_linear8_create(const tts_linear8_config *cfg, const float *w, const float *bias, void *dev_arena, size_t arena_bytes,
                       void *hip_stream, tts_linear8 **out);

/*
 * One batch of rows, asynchronous on the stream.
 *   x8      DEVICE e4m3 [rows][TTS_WIDTH8(in_dim)], 16-byte aligned; columns past in_dim hold zeros
 *   scales  DEVICE [rows][TTS_SCALE_COLUMNS(in_dim)] bytes, 4-byte aligned
 *   y       DEVICE [rows] rows of out_dim elements, y_stride elements apart (0: out_dim), aligned to its element
 * Errors: TTS_E_INVAL for null pointers, rows outside 0 .. TTS_MAX_ROWS (tts_norm.h; 0 does nothing), a stride below out_dim or above 2^40,
 * or an array that is not aligned.  y overlaps neither of the others.
 */
int tts_linear8_run(tts_linear8 *lin, const void *x8, const void *scales, int rows, void *y, long long y_stride);

/* Does not wait: the arena stays the caller's to keep until the calls that were queued, and graphs that hold any, have run. */
void tts_linear8_destroy(tts_linear8 *lin);

#ifdef __cplusplus
}
#endif
#endif
