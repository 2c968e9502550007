/*
 * tts_rotary.h -- C ABI of rotary positions: the columns of a head turn in pairs, by an angle that grows with the row's position,
 * so that the product of a query and a key depends on how far apart they are.  Pair i of a head (0 .. rot_dim / 2 - 1) at position p:
 *
 *     a   = p * f[i]                              f[i] = base^(-2 i / rot_dim), scaled as below
 *     y_u = magnitude * (x_u cos a - x_w sin a)   HALF: u = i, w = i + rot_dim / 2;  PAIRS: u = 2 i, w = 2 i + 1
 *     y_w = magnitude * (x_w cos a + x_u sin a)
 *
 * Columns from rot_dim on stay as they are.  `back` turns the other way: the gradient of the above for that of y, and for a magnitude of 1
 * what takes a row's position from it.
 *
 * For contexts longer than what was trained on:
 *     TTS_ROTARY_LINEAR   f[i] / factor
 *     TTS_ROTARY_BASE     base * factor^(rot_dim / (rot_dim - 2)) in the place of base: the fastest pair keeps its f, the slowest has f / factor
 *     TTS_ROTARY_PARTS    f[i] * (g + (1 - g) / factor),  g = (trained_len * f[i] / 2 pi - low) / (high - low), within 0 .. 1: pairs that turn more than
 *                         `high` times within trained_len keep their f, those that turn less than `low` times are stretched
 *
 * Angles are formed as turns in 64-bit fixed point, and are exact to 2^-31 of a turn at every position that 32 bits hold, negative ones too; sine and
 * cosine to 2^-23.  Products are fp32, each result rounded once.
 *
 * Everything is queued on the stream given at creation; device memory comes from the caller's arena; nothing is allocated on the device.  A call is one
 * launch and may be captured into a graph, which holds `first` but reads positions anew.  What a row becomes does not depend on the others.
 * Conventions as in tts_pool.h: 0 on success, negative tts_status otherwise, text in tts_last_error(); one owner thread per object.
 */
#ifndef TTS_ROTARY_H
#define TTS_ROTARY_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tts_rotary tts_rotary;

#define TTS_ROTARY_MAX_HEADS 1024
#define TTS_ROTARY_MAX_HEAD_DIM 256
#define TTS_ROTARY_MAX_ROWS (1 << 24)    /* of one call */

enum { TTS_ROTARY_HALF = 0, TTS_ROTARY_PAIRS = 1 };
enum { TTS_ROTARY_PLAIN = 0, TTS_ROTARY_LINEAR = 1, TTS_ROTARY_BASE = 2, TTS_ROTARY_PARTS = 3 };

typedef struct {
    int rot_dim;          /* columns of a head that turn: even, 2 .. head_dim (TTS_ROTARY_BASE: 4 ..) */
    int layout;           /* TTS_ROTARY_HALF / TTS_ROTARY_PAIRS */
    int scaling;          /* TTS_ROTARY_PLAIN .. TTS_ROTARY_PARTS */
    int trained_len;      /* TTS_ROTARY_PARTS: 1 .. ; otherwise not used */
    double base;          /* 1 .. 2^60 */
    double factor;        /* 1 .. 2^30; TTS_ROTARY_PLAIN does not use it */
    double low, high;     /* TTS_ROTARY_PARTS: 0 <= low < high <= 2^30 */
    double magnitude;     /* 2^-60 .. 2^60 */
} tts_rotary_angles;

typedef struct {
    int n_heads;          /* 1 .. TTS_ROTARY_MAX_HEADS */
    int head_dim;         /* a multiple of 8, 8 .. TTS_ROTARY_MAX_HEAD_DIM */
    int x_dtype;          /* TTS_DTYPE_F32 / TTS_DTYPE_BF16 of tts_pool.h (0 / 1) */
    int y_dtype;
    tts_rotary_angles angles;
} tts_rotary_config;

/* One call.  DEVICE pointers.  A row holds n_heads * head_dim elements; a stride is the distance between rows in elements, a multiple of 8, at most 2^40
 * (0: the rows lie back to back).  x and y are 16-byte aligned; y may be x, with its type and stride; otherwise they do not overlap. */
typedef struct {
    int rows;                                 /* 0 .. TTS_ROTARY_MAX_ROWS; 0 does nothing */
    const void *x;     long long x_stride;
    void *y;           long long y_stride;
    const int *positions;                     /* [rows], 4-byte aligned; null: row r is at first + r */
    int first;                                /* first + rows within what 32 bits hold; not used with positions */
    int back;                                 /* 0 / 1 */
} tts_rotary_rows;

/* Bytes of device memory tts_rotary_create needs for this configuration (0 if the configuration is invalid). */
size_t tts_rotary_workspace_bytes(const tts_rotary_config *cfg);

/*
 * Create a rotation.  `dev_arena` is DEVICE memory of at least tts_rotary_workspace_bytes(cfg) bytes, 256-byte aligned,
 * owned by the caller and kept alive until tts_rotary_destroy.  `hip_stream` is a hipStream_t.
 */
int tts_rotary_create(const tts_rotary_config *cfg, void *dev_arena, size_t arena_bytes, void *hip_stream, tts_rotary **out);

/*
 * Turn rows, asynchronously on the stream.  Errors: TTS_E_INVAL for null pointers, a number of rows or a last position outside its range, a stride that is too
 * small, too large or no multiple of 8, an array that is not aligned as above, a `back` that is neither 0 nor 1, or y at x with another type or stride.
 */
int tts_rotary_run(tts_rotary *rotary, const tts_rotary_rows *rows);

/* Does not wait: the arena stays the caller's to keep until the calls that were queued, and graphs that hold any, have run. */
void tts_rotary_destroy(tts_rotary *rotary);

#ifdef __cplusplus
}
#endif
#endif
