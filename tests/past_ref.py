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


def paged(q, k_pages, v_pages, table, page, q_len, own_len, table_row, prefix=None, prefix_len=(), prefix_table_row=(), causal=True, scale=None):
    """(out, lse, and what a derived tolerance takes: the sum of w |v|, the largest sum of |q| |k| of a row, times the scale)."""
    _, heads, d = q.shape
    n_pages, kv = k_pages.shape[:2]
    group = heads // kv
    scale = 1 / np.sqrt(d) if scale is None else scale
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    mass, size = np.zeros(q.shape), np.zeros(q.shape[:2])
    at = 0
    for i, (n, m) in enumerate(zip(q_len, own_len)):
        of = -1 if prefix is None else prefix[i]
        pieces = ([(prefix_table_row[of], prefix_len[of], False)] if of >= 0 else []) + [(table_row[i], m, True)]
        k, v, sees = [np.zeros((0, kv, d))], [np.zeros((0, kv, d))], [np.zeros((n, 0), bool)]
        for row, length, own in pieces:
            j = np.arange(length)
            pg, off = places(table, row, 0, length, page) if length else (j, j)
            there = (pg >= 0) & (pg < n_pages)
            k.append(k_pages[pg[there], :, off[there]].astype(np.float64))
            v.append(v_pages[pg[there], :, off[there]].astype(np.float64))
            sees.append(j[there] <= m - n + np.arange(n)[:, None] if own and causal else np.ones((n, there.sum()), bool))
        k, v, sees = np.concatenate(k), np.concatenate(v), np.concatenate(sees, 1)
        for h in range(heads):
            qq, kk, vv = q[at:at + n, h].astype(np.float64), k[:, h // group], v[:, h // group]
            # (a key that nobody sees may hold anything, and one that some see is not used for the others)
            any_sees = sees.any(0)
            kk, vv, s_h = kk[any_sees], vv[any_sees], sees[:, any_sees]
            if not len(kk) or not n:
                continue
            with np.errstate(invalid="ignore"):
                s = np.where(s_h, scale * (qq @ kk.T), -np.inf)
            top = s.max(1, keepdims=True)
            none = np.isneginf(top[:, 0])
            e = np.exp(s - np.where(np.isneginf(top), 0, top))
            total = e.sum(1, keepdims=True)
            w = e / np.where(total == 0, 1, total)
            with np.errstate(invalid="ignore"):
                odd = ~np.isfinite(vv).all(1)
                out[at:at + n, h] = w[:, ~odd] @ vv[~odd]
                for j in np.flatnonzero(odd):
                    out[at:at + n, h][s_h[:, j]] += w[s_h[:, j], j: j + 1] * vv[j]
                mass[at:at + n, h] = w[:, ~odd] @ np.abs(vv[~odd])
                lse[at:at + n, h] = np.where(none, -np.inf, np.where(none, 0, top[:, 0]) + np.log(np.where(none, 1, total[:, 0])))
                size[at:at + n, h] = np.where(s_h, scale * (np.abs(qq) @ np.abs(kk).T), 0).max(1)
        at += n
    return out, lse, mass, size
