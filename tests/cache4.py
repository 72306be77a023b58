"""Inputs and checks shared by the tests of rotary positions and of the paged 4-bit cache."""

import numpy as np

from oracle import cache4_oracle as Q
from tests.cache8 import LOGIT_STEP, OUT_STEP, bf16, to_torch

# A weight (probability times s) is rounded to f16, 2^-11 / 2 of itself; its exponential and the log2 of s add 2^-22 of it
# and the fp32 rounding of an exponent of up to 2^7, 2^-17: together below 2^-11 / 2 + 2^-16.
W_STEP = 2.0 ** -12 + 2.0 ** -16
# cos and sin are off by 2^-22 at most, and each result has two products of them; 2^-22 for the fp32 rounding of both
# products and their sum.
TURN_STEP = 2.0 ** -22 + 2.0 ** -22


def rows(rng, shape, spread=1.0):
    gain = np.exp(0.5 * spread * rng.standard_normal(shape[-1]))
    return bf16(rng.standard_normal(shape) * gain)


def pool(rng, pages, heads, P, d=128):
    """Codes and numbers of a written pool."""
    x = rows(rng, (pages, heads, P, d)) * np.exp(0.3 * rng.standard_normal((pages, heads, P, 1)))
    c, f = Q.encode(bf16(x))
    return Q.pack(c), f


def param_torch(f, device="cuda"):
    return to_torch(f, device)


def check_rotation(out, ref, x, amplitude, n, interleaved):
    """out (float64 from bf16) against the rotation ref of rows x; n elements turn."""
    a = np.abs(x[..., :n])
    if interleaved:
        pair = np.repeat(a[..., 0::2] + a[..., 1::2], 2, -1)
    else:
        half = a[..., :n // 2] + a[..., n // 2:]
        pair = np.concatenate([half, half], -1)
    bound = OUT_STEP * np.abs(ref[..., :n]) + (1 + OUT_STEP) * TURN_STEP * abs(amplitude) * pair + 1e-38
    err = np.abs(out[..., :n] - ref[..., :n])
    assert (err <= bound).all(), float((err / bound).max())
    assert np.array_equal(out[..., n:], x[..., n:])


# A weight of less than 2^-14 is off by half of f16's least step, 2^-25. The weight of the largest p s so far is 2^6 at least (a
# reference is 2^6 and never above it), so that is 2^-31 of the largest.
W_LEAST = 2.0 ** -31


def check_attention(out, lse, q, k, kp, v, vp, table, lens, group):
    """out and lse (numpy) against the definition; returns the worst |error| / bound of both."""
    ref, rl, mass, codes, size, most = Q.attend(q, k, kp, v, vp, table, lens, group)
    assert np.array_equal(np.isnan(out), np.isnan(ref))
    n = np.maximum(np.asarray(lens, np.float64), 1)[:, None, None, None]
    bound = (OUT_STEP * np.abs(ref) + W_STEP * codes + 4 * LOGIT_STEP * size[..., None] * mass + 2.0 ** -18 * mass +
             n * W_LEAST * 15 * most[..., None] + n * 2.0 ** -147 + 2.0 ** -133)
    good = ~np.isnan(ref)
    err, bound = np.abs(out[good] - ref[good]), bound[good]
    assert (err <= bound).all(), float((err / bound).max())
    worst = float((err / bound).max()) if err.size else 0.0
    if lse is not None:
        assert np.array_equal(np.isnan(lse), np.isnan(rl)) and np.array_equal(np.isneginf(lse), np.isneginf(rl))
        fine = np.isfinite(rl)
        # 2^-20: the approximate logarithm and exponential (2^-22 each) and the fp32 of the result
        lb = LOGIT_STEP * size[fine] + 2.0 ** -20 * (8 + np.abs(rl[fine]))
        le = np.abs(lse[fine] - rl[fine])
        assert (le <= lb).all(), float((le / lb).max())
        worst = max(worst, float((le / lb).max()) if le.size else 0.0)
    return worst
