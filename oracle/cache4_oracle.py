"""Rotary positions and the paged 4-bit cache in plain numpy, 64 bits.

Written from the definitions in include/kv_evict.h; shares no code with the library. Arrays are the library's layouts
on the host: codes uint8 [pages][H][P][d / 2], numbers of the rows float64 [pages][H][P][2] (s, z)."""

from __future__ import annotations

import math

import numpy as np


def _bf16(x):
    """float32 values rounded to bf16 (nearest, ties to even), as float64."""
    b = np.asarray(x, np.float32).view(np.uint32)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).view(np.float32)
    return np.where(np.isnan(x), np.nan, r).astype(np.float64)


# ------------------------------------------------------------------------------------------------ rotary positions

def frequencies(kind, n, base=10000.0, factor=1.0, original=0.0, low=1.0, high=4.0):
    """(frequencies [n / 2], amplitude), pair by pair."""
    out, amplitude = [], 1.0
    if kind == "ntk":
        base = base * factor ** (n / (n - 2))
    if kind == "yarn":
        amplitude = 0.1 * math.log(factor) + 1
        # the pair whose frequency makes r turns: base^(-2j/n) * original / (2 pi) = r
        pair = lambda r: n / 2 * math.log(original / (2 * math.pi * r)) / math.log(base)  # noqa: E731
        a, b = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), n - 1)
    for j in range(n // 2):
        f = base ** (-2 * j / n)
        if kind == "linear":
            f /= factor
        elif kind == "parts":
            turns = f * original / (2 * math.pi)
            g = min(max((turns - low) / (high - low), 0), 1)
            f = (1 - g) * f / factor + g * f
        elif kind == "yarn":
            g = min(max((j - a) / max(b - a, 0.001), 0), 1)
            f = g * f / factor + (1 - g) * f
        out.append(f)
    return np.array(out), amplitude


def rotate(x, positions, freq, amplitude=1.0, interleaved=False, transpose=False):
    """Rows x [tokens][heads][d] float64 turned by positions."""
    n = 2 * len(freq)
    y = np.array(x, np.float64)
    angle = np.asarray(positions, np.float64)[:, None] * freq
    turn = amplitude * np.exp((-1j if transpose else 1j) * angle)[:, None]
    if interleaved:
        z = (y[..., 0:n:2] + 1j * y[..., 1:n:2]) * turn
        y[..., 0:n:2], y[..., 1:n:2] = z.real, z.imag
    else:
        z = (y[..., :n // 2] + 1j * y[..., n // 2:n]) * turn
        y[..., :n // 2], y[..., n // 2:n] = z.real, z.imag
    return y


# ------------------------------------------------------------------------------------------------ rows in 4 bits

def encode(rows):
    """(codes [...][d] as integers, s and z [...][2]) of bf16 rows [...][d] (float64)."""
    rows = np.asarray(rows, np.float64)
    good = np.isfinite(rows).all(-1)
    x = np.where(good[..., None], rows, 0.0)
    lo, hi = x.min(-1) + 0.0, x.max(-1)
    s = _bf16(np.float32(np.float32(hi / 16 - lo / 16) * np.float32(16 / 15)))
    s = np.where(s >= 2.0 ** -120, s, 0.0)
    unit = np.float32(np.where(s > 0, s, 1.0) / 16)[..., None]
    c = np.minimum(np.rint(np.float32(x / 16 - lo[..., None] / 16) / unit), 15)
    c = np.where((s > 0)[..., None], c, 0).astype(np.uint8)
    param = np.stack([s, lo], -1)
    return c, np.where(good[..., None], param, np.nan)


def pack(c):
    return (c[..., 0::2] | c[..., 1::2] << 4).astype(np.uint8)


def unpack(code):
    return np.stack([code & 15, code >> 4], -1).reshape(*code.shape[:-1], 2 * code.shape[-1])


def values(code, param):
    return unpack(code).astype(np.float64) * param[..., :1] + param[..., 1:]


def store(code, param, rows, slots):
    """kv_evict_cache_store for keys or values: rows [n][H][d] float64; code and param in place."""
    P = code.shape[2]
    for t, slot in enumerate(slots):
        if 0 <= slot < len(code) * P:
            c, f = encode(rows[t])
            code[slot // P, :, slot % P], param[slot // P, :, slot % P] = pack(c), f


def gather(code, param, rows, pages):
    """One unit's rows [n][d] float64 into its pages of head h: code [pages][P][d / 2], param [pages][P][2], in place."""
    P = code.shape[1]
    c, f = encode(rows)
    for i in range(len(rows)):
        code[pages[i // P], i % P], param[pages[i // P], i % P] = pack(c[i]), f[i]


def attend(q, k, kp, v, vp, table, lens, group):
    """Attention of q [n][T][Hq][d] (float64) over sequences given by table [n][M] and lens [n]: (out, lse, and for
    bounds mass, of p (s c + |z|); codes, of p s c; size, the largest sum_j |q_j| (s c_j + |z|) / sqrt(d) of a row; most,
    the largest p s)."""
    n, T, Hq, d = q.shape
    P = k.shape[2]
    out, mass, codes = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
    lse, size, most = np.full(q.shape[:3], -np.inf), np.zeros(q.shape[:3]), np.zeros(q.shape[:3])
    for r in range(n):
        L = int(lens[r])
        pg = table[r, :-(-L // P)].astype(np.int64)
        good = np.repeat((pg >= 0) & (pg < len(k)), P)[:L]
        pg = np.clip(pg, 0, len(k) - 1)
        for h in range(Hq // group):
            ck, cv = (unpack(c[pg, h]).reshape(-1, d)[:L].astype(np.float64) for c in (k, v))
            pk, pv = (f[pg, h].reshape(-1, 2)[:L] for f in (kp, vp))
            for t in range(T):
                m = L - T + t + 1
                if m <= 0:
                    continue
                use = np.flatnonzero(good[:m])
                for g in range(group):
                    at = (r, t, h * group + g)
                    x = q[at]
                    if not len(use) and np.isfinite(x).all():
                        continue
                    kk = ck[use] * pk[use, :1] + pk[use, 1:]
                    with np.errstate(invalid="ignore"):
                        l = kk @ x / math.sqrt(d)
                    if not np.isfinite(x).all() or np.isnan(l).any():
                        out[at] = lse[at] = np.nan
                        continue
                    e = np.exp(l - l.max())
                    p = e / e.sum()
                    lse[at] = l.max() + math.log(e.sum())
                    out[at] = p @ (cv[use] * pv[use, :1] + pv[use, 1:])
                    codes[at] = (p * pv[use, 0]) @ cv[use]
                    mass[at] = codes[at] + p @ np.abs(pv[use, 1])
                    size[at] = ((ck[use] * pk[use, :1] + np.abs(pk[use, 1:])) @ np.abs(x)).max() / math.sqrt(d)
                    most[at] = (p * pv[use, 0]).max()
    return out, lse, mass, codes, size, most
