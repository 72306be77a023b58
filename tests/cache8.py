"""Inputs and checks shared by the tests of the paged 8-bit cache."""

import numpy as np

from oracle import cache8_oracle as C

# bf16 rounds by at most half a step, 2^-8 of the value. In the attention the probabilities enter the value
# product with at most 2^-11 of their value lost (the kernel's own rounding of them and of its exponential),
# and a logit, a 128-term fp32 sum scaled three times, is off by at most 2^-16 of the sum of its terms'
# magnitudes (128 * 2^-24, and as much for the order of the sum): a relative 2 * that in a probability and in
# the sum they are divided by.
OUT_STEP, P_STEP, LOGIT_STEP = 2.0 ** -8, 2.0 ** -11, 2.0 ** -16


def bf16(x):
    """float64 values rounded to bf16 (nearest, ties to even), as float64."""
    b = np.asarray(x, np.float32).view(np.uint32)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).view(np.float32)
    return np.where(np.isnan(x), np.nan, r).astype(np.float64)


def to_torch(x, device="cuda"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).to(device)


def rows(rng, shape, spread=1.0):
    """bf16 rows with channels that are larger than others."""
    gain = np.exp(0.5 * spread * rng.standard_normal(shape[-1]))
    return bf16(rng.standard_normal(shape) * gain)


def pool(rng, pages, heads, P, d=128):
    """Codes and scales of a written pool; NaN codes in none of them."""
    code = rng.integers(0, 256, (pages, heads, P, d)).astype(np.uint8)
    # values as rows have them: normal, scaled by page
    code[:] = C.encode(np.clip(rng.standard_normal(code.shape) * 100, -448, 448))
    scale = np.ldexp(1.0, rng.integers(-9, -5, (pages, heads))).astype(np.float32)
    return code, scale


def table_for(rng, lens, P, spare=3, max_pages=None):
    """A table [n][M] of shuffled pages for the lengths, -1 behind them, and the number of pages."""
    have = [-(-int(x) // P) for x in lens]
    M = max_pages or max(1, max(have))
    order = rng.permutation(sum(have) + spare)
    table, at = np.full((len(lens), M), -1, np.int32), 0
    for i, n in enumerate(have):
        table[i, :n] = order[at:at + n]
        at += n
    return table, sum(have) + spare


def check_attention(out, lse, q, k, ks, v, vs, table, lens, group):
    """out and lse (numpy) against the definition; returns the worst |error| / bound of both."""
    ref, rl, mass, size = C.attend(q, k, ks, v, vs, table, lens, group)
    assert np.array_equal(np.isnan(out), np.isnan(ref))
    bound = OUT_STEP * np.abs(ref) + (P_STEP + 4 * LOGIT_STEP * size[..., None]) * mass + 1e-37
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
