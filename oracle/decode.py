"""Rotary positions, a paged cache and one token's attention over it, in fp64.

TEST INFRASTRUCTURE ONLY (see the package header).  Arrays are NumPy fp64 of the
exact input values; tables, lengths and masks are plain integers.
"""

import numpy as np


def frequencies(rot, base, scaling="none", s=1.0, trained=1):
    """(radians a position of each of rot/2 pairs, factor on turned elements)."""
    i = np.arange(rot // 2)
    if scaling == "ntk":
        base = base * s ** (rot / (rot - 2))
    f = np.power(np.float64(base), -2.0 * i / rot)
    if scaling == "linear":
        return f / s, 1.0
    if scaling == "by_parts":
        turns = trained * f / (2 * np.pi)
        g = np.clip((turns - 1) / 31, 0, 1)
        return (1 - g) * f / s + g * f, 0.1 * np.log(s) + 1
    return f, 1.0


def angles(pos, freq, sections):
    """[rows, pairs] angles of position ids pos [pos_rows, rows]."""
    which = np.repeat(np.arange(len(sections)), sections)
    return pos.astype(np.float64)[which].T * freq


def rotary(x, theta, layout="half", factor=1.0, transpose=False):
    """x [heads, rows, d], its first pairs turned by theta [rows, pairs]."""
    n = theta.shape[1]
    a = slice(0, n) if layout == "half" else slice(0, 2 * n, 2)
    b = slice(n, 2 * n) if layout == "half" else slice(1, 2 * n, 2)
    c, s = factor * np.cos(theta), factor * np.sin(theta) * (-1 if transpose else 1)
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def place(table_row, page_rows, row, n_pages):
    """(page, row in it), or None where a row has no page."""
    if row < 0 or row // page_rows >= len(table_row):
        return None
    p = int(table_row[row // page_rows])
    return (p, row % page_rows) if 0 <= p < n_pages else None


def rows_seen(table_row, page_rows, n_pages, length, max_len, window=0, mask=None):
    """The (page, row in it) of the rows a sequence's new token attends to."""
    lo = max(0, length - window) if window else 0
    out = []
    for r in range(lo, min(length, max_len)):
        at = place(table_row, page_rows, r, n_pages)
        if at is not None and (mask is None or mask[r]):
            out.append(at)
    return out


def attention(q, k, v, scale):
    """q [hq, d], k and v [hkv, rows, d]: (o [hq, d], lse [hq], sum p |v| [hq, d], largest scale * sum |q k| [hq])."""
    hq, d = q.shape
    hkv, n, _ = k.shape
    o, w = np.zeros((hq, d)), np.zeros((hq, d))
    lse, size = np.full(hq, -np.inf), np.zeros(hq)
    for h in range(hq if n else 0):
        g = h // (hq // hkv)
        x = scale * (k[g] @ q[h])
        m = x.max()
        p = np.exp(x - m)
        lse[h] = m + np.log(p.sum())
        p /= p.sum()
        o[h], w[h] = p @ v[g], p @ np.abs(v[g])
        size[h] = scale * (np.abs(k[g]) @ np.abs(q[h])).max()
    return o, lse, w, size
