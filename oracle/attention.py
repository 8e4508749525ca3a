"""64-bit oracle of the attention calls (include/eldr_attention.h): plain NumPy,
token by token, sharing no code with the library.

Caches are float64 arrays [num_blocks, Hkv, block_size, D] of the values that
the device cache stands for (fp8 codes times their scale).
"""
from __future__ import annotations

import numpy as np


def rotate(x, positions, pair_axis, cos, sin, interleaved=False):
    """x [T, heads, D] turned by positions [n_axes, T]: pair i by the angle whose
    cosine is cos[positions[pair_axis[i], t], i] (NaN where there is none)."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    half = len(pair_axis)
    for t in range(x.shape[0]):
        for i in range(half):
            axis = int(pair_axis[i])
            p = int(positions[axis][t]) if 0 <= axis < len(positions) else -1
            c, s = (float(cos[p][i]), float(sin[p][i])) if 0 <= p < len(cos) else (np.nan, np.nan)
            lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            y[t, :, lo] = x[t, :, lo] * c - x[t, :, hi] * s
            y[t, :, hi] = x[t, :, hi] * c + x[t, :, lo] * s
    return y


def shared_reach(lens, group_start, prefix_len, N, window=0):
    """For each request, (first request of its group that holds anything, slots read
    through that one)."""
    R = len(lens)
    lens = np.clip(lens, 0, N)
    out = [(r, 0) for r in range(R)]
    if window > 0 or prefix_len is None:
        return out
    s = min(max(int(group_start[0]), 0), R)
    for g in range(len(prefix_len)):
        e = min(max(int(group_start[g + 1]), s), R)
        full = [r for r in range(s, e) if lens[r] > 0]
        reach = min([min(max(int(prefix_len[g]), 0), N)] + [int(lens[r]) for r in full])
        if e - s > 1:
            for r in range(s, e):
                out[r] = (full[0] if full else s, reach)
        s = e
    return out


def _slot(table, r, j, bs, num_blocks):
    b = int(table[r][j // bs])
    return (b, j % bs) if 0 <= b < num_blocks else None


def _visible(r, n, lo, own, table, bs, num_blocks):
    first, reach = own
    slots = [(j, _slot(table, first if j < reach else r, j, bs, num_blocks)) for j in range(lo, n)]
    return [(j, s) for j, s in slots if s is not None]


def decode(q, k_cache, v_cache, table, lens, scale, group_start=None, prefix_len=None, sinks=None, window=0):
    """(out [R, Hq, D], lse [R, Hq], weight [R, Hq, D]): the third is
    sum_j p_j |v_j|, what rounding errors of the weights are multiplied by."""
    q = np.asarray(q, np.float64)
    R, Hq, D = q.shape
    nb, Hkv, bs, _ = k_cache.shape
    N = len(table[0]) * bs if R else 0
    owners = shared_reach(lens, group_start, prefix_len, N, window)
    out, mass = np.zeros((R, Hq, D)), np.zeros((R, Hq, D))
    lse = np.full((R, Hq), -np.inf)
    for r in range(R):
        n = int(np.clip(lens[r], 0, N))
        vis = _visible(r, n, max(0, n - window) if window else 0, owners[r], table, bs, nb)
        pages = np.array([s[0] for _, s in vis], np.int64)
        offs = np.array([s[1] for _, s in vis], np.int64)
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            s = k_cache[pages, kv, offs] @ q[r, h] * scale if vis else np.zeros(0)
            every = s if sinks is None else np.append(s, float(sinks[h]))
            if not len(every):
                continue
            top = every.max()
            if top == -np.inf:  # the sum is 0: as without a visible slot
                continue
            lse[r, h] = top + np.log(np.exp(every - top).sum())
            if vis:
                p = np.exp(s - lse[r, h])
                v = v_cache[pages, kv, offs]
                out[r, h], mass[r, h] = p @ v, p @ np.abs(v)
    return out, lse, mass


def weights(q, k_cache, table, lens, lse, scale, w_in, w_out, group_start=None, prefix_len=None):
    """What weights_out holds after the call, given what it held before."""
    q = np.asarray(q, np.float64)
    R, Hq, _ = q.shape
    nb, Hkv, bs, _ = k_cache.shape
    N = len(table[0]) * bs if R else 0
    owners = shared_reach(lens, group_start, prefix_len, N)
    got = np.array(w_out, np.float64)
    for r in range(R):
        n = int(np.clip(lens[r], 0, N))
        for h in range(Hkv):
            got[r, h, :n] = 0 if w_in is None else w_in[r, h, :n]
            for j, (b, o) in _visible(r, n, 0, owners[r], table, bs, nb):
                for i in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    got[r, h, j] += np.exp(scale * (q[r, i] @ k_cache[b, h, o]) - lse[r][i])
    return got


def evict(w, pos, lens, seen, budget, recent, protect=None):
    """(src, new_lens, weights, positions): the arrays after the cut, as float64 and
    int lists of rows [R][Hkv]; slots from lens[r] on keep what w and pos hold."""
    R, Hkv, N = w.shape
    src = np.full((R, Hkv, budget), -1, np.int64)
    w2, p2 = np.array(w), np.array(pos)
    new = np.zeros(R, np.int64)
    for r in range(R):
        n = int(np.clip(lens[r], 0, N))
        new[r] = min(n, budget)
        for h in range(Hkv):
            def rank(j):
                sure = (protect is not None and j < protect[r]) or int(pos[r, h, j]) >= int(seen[r]) - recent
                x = float(w[r, h, j])
                if sure:
                    return (0, 0.0, j)
                return (2, 0.0, j) if np.isnan(x) else (1, -x, j)

            if n <= budget:
                src[r, h, :n] = np.arange(n)
                continue
            stays = set(sorted(range(n), key=rank)[:budget])
            movers = iter([j for j in range(budget, n) if j in stays])
            src[r, h] = [j if j in stays else next(movers) for j in range(budget)]
            w2[r, h, :budget], p2[r, h, :budget] = w[r, h, src[r, h]], pos[r, h, src[r, h]]
            w2[r, h, budget:n], p2[r, h, budget:n] = 0, -1
    return src, new, w2, p2


def moved(cache, table, src, lens, budget):
    """The cache after the rows moved as src says."""
    nb, Hkv, bs, _ = cache.shape
    after = cache.copy()
    for r in range(len(lens)):
        if min(int(lens[r]), len(table[r]) * bs) <= budget:
            continue
        for h in range(Hkv):
            for i in range(budget):
                j = int(src[r, h, i])
                a, b = _slot(table, r, i, bs, nb), _slot(table, r, j, bs, nb)
                if j != i and a is not None and b is not None:
                    after[a[0], h, a[1]] = cache[b[0], h, b[1]]
    return after
