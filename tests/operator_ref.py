"""The operators' definitions in 64 bits (include/tts_norm.h, tts_linear8.h, tts_cross.h), in numpy, for the tests: written from the formulas, without the
library.  8-bit values as bytes."""
import numpy as np

BLOCK = 128
EPS32 = 2.0 ** -24            # half a step of fp32, relative
EPS_BF16 = 2.0 ** -8          # of bf16 (finfo.eps / 2)


def e4m3_table():
    """What the 256 bytes stand for."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b & 128, -v, v)


TABLE = e4m3_table()


def blocks_of(dim):
    return -(-dim // BLOCK)


def scale_of(v):
    """Of each block of [rows, dim]: the least power of two (as its exponent) that brings the largest finite magnitude to 448 at most; 0 where that is zero."""
    rows, dim = v.shape
    out = np.zeros((rows, blocks_of(dim)), np.int64)
    for b in range(out.shape[1]):
        a = np.abs(v[:, b * BLOCK:(b + 1) * BLOCK])
        a = np.where(np.isfinite(a), a, 0).max(1)
        for r in range(rows):
            if a[r] > 0:
                k = int(np.floor(np.log2(a[r]))) - 10
                while a[r] > 448 * 2.0 ** k:
                    k += 1
                out[r, b] = max(k, -127)
    return out


def to_e4m3(v):
    """Nearest e4m3 byte, ties to the even one; |v| <= 448."""
    grid = TABLE[:127]
    at = np.clip(np.searchsorted(grid, np.abs(v)), 1, 126)
    lo, hi = grid[at - 1], grid[at]
    a = np.abs(v)
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (at % 2 == 0))
    byte = np.where(up, at, at - 1)
    return (byte | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def round8(v):
    """([rows, whole blocks] bytes, [rows, whole words] scale bytes) of [rows, dim] in 64 bits."""
    rows, dim = v.shape
    n = blocks_of(dim)
    k = scale_of(v)
    p = np.zeros((rows, n * BLOCK))
    p[:, :dim] = v
    with np.errstate(invalid="ignore"):
        b = to_e4m3((p.reshape(rows, n, BLOCK) * 2.0 ** -k[:, :, None].astype(np.float64)).reshape(rows, -1))
    b[~np.isfinite(p)] = 127
    s = np.full((rows, -(-n // 4) * 4), 127, np.uint8)
    s[:, :n] = k + 127
    return b, s


def values8(b, s):
    """What 8-bit rows stand for."""
    rows, width = b.shape
    k = s[:, : width // BLOCK].astype(np.float64) - 127
    return (TABLE[b].reshape(rows, -1, BLOCK) * 2.0 ** k[:, :, None]).reshape(rows, width)


def norm(x, res, gain, eps):
    t = x.astype(np.float64) + (0 if res is None else res.astype(np.float64))
    return t, gain.astype(np.float64) * t / np.sqrt((t * t).mean(1, keepdims=True) + eps)


def cross(q, k, v, q_len, mem_row, mem_len, keep=None, scale=None):
    """(out, lse, and what a derived tolerance takes: the sum of w |v|, the largest sum of |q| |k| of a row, times the scale)."""
    _, heads, d = q.shape
    group = heads // k.shape[1]
    scale = 1 / np.sqrt(d) if scale is None else scale
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    mass, size = np.zeros(q.shape), np.zeros(q.shape[:2])
    at = 0
    for n, r, m in zip(q_len, mem_row, mem_len):
        rows = np.arange(r, r + m)
        if keep is not None:
            rows = rows[keep[r:r + m] != 0]
        if len(rows):
            for h in range(heads):
                qq, kk, vv = q[at:at + n, h].astype(np.float64), k[rows, h // group].astype(np.float64), v[rows, h // group].astype(np.float64)
                s = scale * qq @ kk.T
                top = s.max(1, keepdims=True) if n else np.zeros((0, 1))
                e = np.exp(s - top)
                w = e / e.sum(1, keepdims=True)
                out[at:at + n, h] = w @ vv
                mass[at:at + n, h] = w @ np.abs(vv)
                lse[at:at + n, h] = (top + np.log(e.sum(1, keepdims=True)))[:, 0]
                size[at:at + n, h] = (scale * np.abs(qq) @ np.abs(kk).T).max(1) if n else 0
        at += n
    return out, lse, mass, size
