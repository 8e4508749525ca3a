"""Oracle of the calls of include/eldr_kv_cache.h: plain NumPy, page by page and
token by token, sharing no code with the library.

Values that become codes are worked out in fp32 with the roundings that the header
states (NumPy rounds each operation to nearest even), so that codes are compared
exactly; ``exact=True`` gives the formulas in 64 bits instead.
"""
from __future__ import annotations

import numpy as np


def normed(x, w, eps, exact=False):
    """x [.., D] over the root of its mean square, times w; w None: x."""
    t = np.float64 if exact else np.float32
    x = np.asarray(x, np.float32)
    if w is None:
        return x.astype(t)
    with np.errstate(all="ignore"):
        m = np.square(x.astype(np.float64)).mean(-1, keepdims=True) + np.float64(np.float32(eps))
        i = (1.0 / np.sqrt(m)).astype(t)
        return (x.astype(t) * i) * np.asarray(w, np.float32).astype(t)


def turned(x, positions, pair_axis, cos, sin, interleaved=False):
    """x [T, heads, D] by positions [n_axes, T], in x's own precision: each product and
    the sum rounded."""
    t = x.dtype.type
    y, half = x.copy(), len(pair_axis)
    for n in range(x.shape[0]):
        for i in range(half):
            axis = int(pair_axis[i])
            p = int(positions[axis][n]) if 0 <= axis < len(positions) else -1
            c, s = (t(cos[p][i]), t(sin[p][i])) if 0 <= p < len(cos) else (t(np.nan), t(np.nan))
            lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            a, b = x[n, :, lo], x[n, :, hi]
            with np.errstate(all="ignore"):
                y[n, :, lo], y[n, :, hi] = a * c - b * s, b * c + a * s
    return y


def append_int8(x, query_start, table, lens, codes, scale):
    """(codes, scale) after the rows x [T, Hkv, D] fp32 have been stored; codes int8
    [num_blocks, Hkv, bs, D], scale fp32 [num_blocks, Hkv]."""
    x = np.asarray(x, np.float32)
    codes, scale = codes.copy(), scale.copy()
    nb, Hkv, bs, D = codes.shape
    T, R, N = x.shape[0], len(lens), len(table[0]) * bs
    start = np.clip(query_start, 0, T)
    for r in range(R):
        held, new = int(np.clip(lens[r], 0, N)), int(start[r + 1] - start[r])
        for at in range(held // bs, -(-min(held + new, N) // bs)):
            first, end = max(held, at * bs), min(held + new, (at + 1) * bs, N)
            page = int(table[r][at])
            if first >= end or not 0 <= page < nb:
                continue
            rows = x[start[r] + first - held:start[r] + end - held]
            o0 = first - at * bs
            for h in range(Hkv):
                codes[page, h, :], scale[page, h] = _page(rows[:, h], o0, codes[page, h], scale[page, h])
    return codes, scale


def _page(rows, o0, codes, scale):
    codes = codes.copy()
    end = o0 + len(rows)
    top = np.abs(rows).max()  # NaN where there is one
    if not np.isfinite(top) or (o0 > 0 and not np.isfinite(scale)):
        codes[o0:end] = 0
        return codes, np.float32(np.nan)
    if o0 == 0 or scale == 0:
        after, back = np.float32(top) * (np.float32(1) / np.float32(127)), 0.0
    else:
        after, back = scale, 1.0
        while 127 * np.float64(after) < np.float64(top):
            after, back = np.float32(after * np.float32(2)), back / 2
    if back != 1.0:
        codes[:o0] = np.rint(codes[:o0].astype(np.float64) * back).astype(np.int8)
    with np.errstate(all="ignore"):
        c = np.clip(np.rint(rows / after), -127, 127) if after > 0 else np.zeros_like(rows)
    codes[o0:end] = c.astype(np.int8)
    return codes, after


def fork(parent, child, page, table, lens, caches, scales=()):
    """(table, lens, caches, scales) afterwards: caches [layers, num_blocks, Hkv, bs, D],
    scales [layers, num_blocks, Hkv]."""
    table, lens = table.copy(), lens.copy()
    caches, scales = [c.copy() for c in caches], [s.copy() for s in scales]
    R, mb = table.shape
    nb, bs = caches[0].shape[1], caches[0].shape[3]
    for p, c, to in zip(parent, child, page):
        if not 0 <= p < R or not 0 <= c < R or p == c:
            continue
        n = int(np.clip(lens[p], 0, mb * bs))
        full, rest = divmod(n, bs)
        row = np.full(mb, -1, table.dtype)
        row[:full] = table[p, :full]
        if rest and 0 <= table[p, full] < nb and 0 <= to < nb:
            row[full] = to
            for x in caches:
                x[:, to, :, :rest] = x[:, table[p, full], :, :rest]
            for s in scales:
                s[:, to] = s[:, table[p, full]]
        table[c], lens[c] = row, n
    return table, lens, caches, scales


def compact(remap, table, caches, scales=()):
    """(table, caches, scales) afterwards."""
    nb = len(remap)
    free = [not 0 <= remap[b] < nb for b in range(nb)]

    def after(b):
        if not 0 <= b < nb or free[b]:
            return -1
        return int(remap[b]) if free[remap[b]] else b

    new = [x.copy() for x in caches], [s.copy() for s in scales]
    for b in range(nb):
        to = after(b)
        if to not in (-1, b):
            for was, x in zip(list(caches) + list(scales), new[0] + new[1]):
                x[:, to] = was[:, b]
    return np.array([[after(int(b)) for b in row] for row in table], np.int32).reshape(table.shape), *new
