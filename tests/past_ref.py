"""The definitions of a decoder block's own past in 64 bits (include/tts_rotary.h, tts_cache.h, tts_paged.h), in numpy, for the tests: written from the formulas, without the library."""
import numpy as np

PI = np.longdouble("3.14159265358979323846264338327950288")

EPS32 = 2.0 ** -24            # half a step of fp32, relative
EPS_BF16 = 2.0 ** -8          # of bf16 (finfo.eps / 2)


def freqs(rot, base=10000.0, scaling=0, factor=1.0, trained_len=0, low=1.0, high=32.0, **_):
    """Radians a position of each pair."""
    i = np.arange(rot // 2, dtype=np.longdouble)
    base = np.longdouble(base) * (np.longdouble(factor) ** (np.longdouble(rot) / (rot - 2)) if scaling == 2 else 1)
    f = base ** (-2 * i / rot)
    if scaling == 1:
        f = f / factor
    if scaling == 3:
        turns = trained_len * f / (2 * PI)
        g = np.clip((turns - low) / (high - low), 0, 1)
        f = f * (g + (1 - g) / factor)
    return f


def rotary(x, positions, rot, pairs=False, magnitude=1.0, back=False, **angles):
    """(y, what a derived tolerance takes: the magnitude times |x_u| + |x_w| of a column's pair, 0 for columns that do not turn) of x [rows, heads, head_dim]."""
    f = freqs(rot, **angles)
    a = np.remainder(np.asarray(positions).astype(np.longdouble)[:, None] * f, 2 * PI)
    c, s = (np.cos(a) * magnitude)[:, None], (np.sin(a) * (-magnitude if back else magnitude))[:, None]
    i = np.arange(rot // 2)
    u, w = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
    x = x.astype(np.longdouble)
    y, size = x.copy(), np.zeros(x.shape)
    y[:, :, u] = x[:, :, u] * c - x[:, :, w] * s
    y[:, :, w] = x[:, :, w] * c + x[:, :, u] * s
    size[:, :, u] = size[:, :, w] = magnitude * (np.abs(x[:, :, u]) + np.abs(x[:, :, w]))
    return y.astype(np.float64), size


def rotary_tolerance(y, size, bf16):
    """Sine and cosine within 2^-23, times the magnitude (rounded), the product with x of one rounded, their sum rounded; then the result's own rounding."""
    return size * (2 * EPS32 + EPS32 + EPS32) + np.abs(y) * (EPS32 + (EPS_BF16 if bf16 else 0)) * (size != 0) + (EPS_BF16 * np.abs(y) if bf16 else 0)


def places(table, table_row, first, n, page):
    """(page, row in it) of rows first .. first + n - 1 of a sequence."""
    j = np.arange(first, first + n)
    return table[table_row, j // page], j % page
