"""The paged 8-bit cache in plain numpy, 64 bits: its codes and scales, its tables and its attention.

Written from the definitions in include/kv_evict.h; shares no code with the library. Arrays are the
library's layouts on the host: codes uint8 [pages][H][P][d], scales [pages][H]."""

from __future__ import annotations

import math

import numpy as np


def _value(c):
    sign, exp, frac = (-1.0 if c & 128 else 1.0), (c >> 3) & 15, c & 7
    if exp == 15 and frac == 7:
        return math.nan
    return sign * (frac / 8 * 2.0 ** -6 if exp == 0 else (1 + frac / 8) * 2.0 ** (exp - 7))


VALUES = np.array([_value(c) for c in range(256)])


def encode(x):
    """The nearest e4m3 codes of float64 x (ties to the even code), beyond 448 the largest, NaN 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    mag = VALUES[:127]                                   # ascending; the codes are the indices
    a = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), 448.0)
    hi = np.clip(np.searchsorted(mag, a), 1, 126)
    lo = hi - 1
    up = (mag[hi] - a < a - mag[lo]) | ((mag[hi] - a == a - mag[lo]) & (hi % 2 == 0))
    code = np.where(up, hi, lo)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(np.isnan(x), 127 + 128 * np.signbit(x), code).astype(np.uint8)


def need(rows):
    """The scale of the rows that share it: the smallest 2^e, e >= -126, with 448 * 2^e >= the largest finite
    magnitude."""
    a = np.abs(rows[np.isfinite(rows)])
    a = float(a.max()) if a.size else 0.0
    e = -126
    while a > math.ldexp(448.0, e):
        e += 1
    return math.ldexp(1.0, e)


def write_rows(code, scale, off, rows):
    """Rows [off, off + n) of one page and head: code [P][d] in place, the new scale is returned."""
    s = need(rows)
    if off > 0:
        s = max(s, float(scale))
        if s > scale:
            code[:off] = encode(VALUES[code[:off]] * (float(scale) / s))
    code[off:off + len(rows)] = encode(rows / s)
    return s


def store(code, scale, rows, slots):
    """kv_evict_cache_store for keys or values: rows [n][H][d] float64; code and scale in place."""
    P, n, t = code.shape[2], len(slots), 0
    while t < n:
        e = t + 1
        if 0 <= slots[t] < len(code) * P:
            while e < n and slots[e] == slots[e - 1] + 1 and slots[e] % P:
                e += 1
            page, off = divmod(int(slots[t]), P)
            for h in range(code.shape[1]):
                scale[page, h] = write_rows(code[page, h], scale[page, h], off, rows[t:e, h])
        t = e


def gather(code, scale, rows, pages):
    """One unit's rows [n][d] float64 into its pages of head h: code [pages][P][d], scale [pages], in place."""
    P = code.shape[1]
    for j in range(-(-len(rows) // P)):
        scale[pages[j]] = write_rows(code[pages[j]], 0.0, 0, rows[j * P:(j + 1) * P])


def pages(lens_from, lens_to, table, free, ring, P, slot_stride=None):
    """kv_evict_cache_pages on host arrays: (table, free, ring, lens, slots, ok)."""
    table, free = table.copy(), free.copy()
    (N, S), M, n = lens_from.shape, table.shape[2], len(free)
    up = lambda x: -(-x // P)  # noqa: E731
    slots = None if slot_stride is None else np.full((N, slot_stride), -1, np.int32)
    cap = M * P
    f, t = lens_from.astype(np.int64), lens_to.astype(np.int64)
    head, count = int(ring[0]), int(ring[1])
    bad = bool((f < 0).any() or (t < 0).any() or (f > cap).any() or (t > cap).any())
    bad |= not 0 <= head < n or not 0 <= count <= n
    grow = np.maximum(t - f, 0).sum(axis=1)
    bad |= slots is not None and bool((grow > slot_stride).any())
    taken = int(np.maximum(up(t) - up(f), 0).sum())
    given = int(np.maximum(up(f) - up(t), 0).sum())
    bad |= count + given > n
    if bad or taken > count:
        return table, free, ring.copy(), lens_from.copy(), slots, "check" if bad else "pages"
    at, tail = 0, count
    for l in range(N):
        c = 0
        for s in range(S):
            a, b = int(f[l, s]), int(t[l, s])
            for j in range(up(a), up(b)):
                table[l, s, j] = free[(head + at) % n]
                at += 1
            for j in range(up(b), up(a)):
                free[(head + tail) % n] = table[l, s, j]
                tail += 1
            for i in range(a, b):
                if slots is not None:
                    page = int(table[l, s, i // P])
                    slots[l, c] = page * P + i % P if 0 <= page < n else -1
                    c += 1
    return table, free, np.array([(head + taken) % n, count - taken + given], np.int32), lens_to.copy(), slots, "ok"


def attend(q, k, ks, v, vs, table, lens, group):
    """Attention of q [n][T][Hq][d] (float64) over sequences given by table [n][M] and lens [n]: (out, lse, mass,
    size), the last two for bounds: the sum of probabilities times magnitudes of v, and the largest
    sum_j |q_j k_ij| / sqrt(d) of a row."""
    n, T, Hq, d = q.shape
    P = k.shape[2]
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    lse, size = np.full(q.shape[:3], -np.inf), np.zeros(q.shape[:3])
    for r in range(n):
        L = int(lens[r])
        pg = table[r, :-(-L // P)].astype(np.int64)
        good = np.repeat((pg >= 0) & (pg < len(k)), P)[:L]
        pg = np.clip(pg, 0, len(k) - 1)
        for h in range(Hq // group):
            kk = (VALUES[k[pg, h]] * ks[pg, h].astype(np.float64)[:, None, None]).reshape(-1, d)[:L]
            vv = (VALUES[v[pg, h]] * vs[pg, h].astype(np.float64)[:, None, None]).reshape(-1, d)[:L]
            for t in range(T):
                m = L - T + t + 1
                if m <= 0:
                    continue
                use = good[:m]
                for g in range(group):
                    x = q[r, t, h * group + g]
                    if not np.isfinite(x).all():
                        out[r, t, h * group + g] = lse[r, t, h * group + g] = np.nan
                        continue
                    if not use.any():
                        continue
                    l = kk[:m][use] @ x / math.sqrt(d)
                    top = l.max()
                    if np.isnan(top):
                        out[r, t, h * group + g] = lse[r, t, h * group + g] = np.nan
                        continue
                    e = np.exp(l - top)
                    lse[r, t, h * group + g] = top + math.log(e.sum())
                    out[r, t, h * group + g] = e @ vv[:m][use] / e.sum()
                    mass[r, t, h * group + g] = e @ np.abs(vv[:m][use]) / e.sum()
                    size[r, t, h * group + g] = (np.abs(kk[:m][use]) @ np.abs(x)).max() / math.sqrt(d)
    return out, lse, mass, size
