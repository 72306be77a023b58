"""Angles of rotary positions against rational arithmetic: the table of a handle, and rotations far out."""

import ctypes
import math
import os
from fractions import Fraction

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_30738_gb300", "libkvevict.so")
PI = Fraction("3.141592653589793238462643383279502884197169399375105820974944592307816406286")


def _k():
    if not os.path.exists(LIB):
        pytest.skip("library not built")
    from paper_2609_30738_gb300 import kv_evict as K
    return K


def _turns(angle):
    """Radians (a Fraction) as a fraction of a turn in [-1/2, 1/2)."""
    t = angle / (2 * PI)
    return t - math.floor(t + Fraction(1, 2))


def test_the_table_holds_64_bits_of_a_turn():
    # a handle begins with its pairs' turns a position in units of 2^-64, 32 bits unsigned above 32 signed ones
    K = _k()
    f = [500000.0 ** (-2 * j / 128) for j in range(40)] + [
        0.0, 1.0, -1.0, 2 * math.pi, -2 * math.pi, 3.5, 1e-12, -1e-12, 1e-30, -5e-324, math.pi, 1e6, -1e6 / 3, 2.0 ** 40 + 0.5,
        2.0 ** 61 + 512, -(2.0 ** 62 - 512), 2.0 ** -63, 2.0 ** -64 * 6, 2.0 ** -66, 0.7, 0.1, -0.1, 12345.678, 1e15]
    r = K.Rotary(frequencies=f)
    words = np.ctypeslib.as_array(ctypes.cast(r._h, ctypes.POINTER(ctypes.c_uint32)), (128,)).astype(object)
    for j, x in enumerate(f):
        low = words[2 * j] - (words[2 * j] >> 31 << 32)
        off = (words[2 * j + 1] * 2 ** 32 + low) - Fraction(x) / (2 * PI) * 2 ** 64
        off -= 2 ** 64 * math.floor(off / 2 ** 64 + Fraction(1, 2))
        assert abs(off) <= Fraction(5, 8) + Fraction(1, 1 << 20), (x, float(off))


def test_frequencies_beyond_any_use_are_taken():
    K = _k()
    K.Rotary(frequencies=[1e300, -1e300, 2.0 ** 117, 2.0 ** 116, 2.0 ** 180, 2.0 ** 64, 1.7e308, -2.0 ** 63] * 8)


@pytest.mark.gpu
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("pos", [2 ** 31 - 1, -2 ** 31, 2 ** 27 + 12345, 1 << 24])
def test_angles_far_out(pos, inter):
    # frequencies that come back to within 2^-20 radians of a whole turn at pos. There b of the pair (1, 0) is the small sine itself,
    # which bf16 holds to 2^-8 of itself, and the angle shows to the 2^-31 of a turn that are promised.
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    K = _k()
    rng = np.random.default_rng(abs(pos))
    f = [2 * math.pi * int(k) / pos for k in rng.integers(1, abs(pos) // 7, 64)]
    x = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device="cuda")
    a, b = (slice(0, None, 2), slice(1, None, 2)) if inter else (slice(0, 64), slice(64, None))
    x[..., a] = 1.0
    got = K.Rotary(frequencies=f, interleaved=inter).rotate(x, torch.tensor([pos], dtype=torch.int32, device="cuda"))
    got = got[0, 0, b].double().cpu().tolist()
    worst = 0.0
    for g, w in zip(got, f):
        t = float(2 * PI * _turns(Fraction(w) * pos))
        assert abs(t) < 2.0 ** -20
        worst = max(worst, abs(g - t) / (2 * math.pi * 2.0 ** -31 + (2.0 ** -8 + 2.0 ** -21) * abs(t)))
    assert worst <= 1.0, worst


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("n,inter,P", [(9, False, 16), (700, True, 32), (1500, False, 128)])
def test_far_appends_are_rotate_then_store(bits, n, inter, P):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    K = _k()
    rng = np.random.default_rng(n + bits)
    spec = dict(num_layers=1, num_q_heads=8, num_kv_heads=2, head_dim=128)
    r = K.Rotary(128, 96, interleaved=inter, scaling="ntk", factor=4.0)
    pos = rng.integers(-2 ** 31, 2 ** 31, n)
    pos[:6] = [-1, 2 ** 31 - 1, -2 ** 31, 0, -4000000, 1 << 30]
    pos = torch.from_numpy(pos.astype(np.int32)).cuda()
    x = torch.from_numpy(rng.standard_normal((n, 12, 128)).astype(np.float32)).cuda().to(torch.bfloat16)
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    Cache = K.Cache8 if bits == 8 else K.Cache4
    pages = -(-n // P)
    a, b = (Cache(spec, max_seqs=1, num_pages=pages, max_pages=pages, page_tokens=P) for _ in range(2))
    names = ("k", "v", "k_scale", "v_scale") if bits == 8 else ("k", "v", "k_param", "v_param")
    for name in names:
        getattr(a, name).zero_()
        getattr(b, name).zero_()
    new = lambda t: torch.empty(t.shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    a.store(r.rotate(k, pos, new(k)), v, slots)
    got = b.append(r, pos, k, v, slots, q=q, q_out=new(q))
    assert torch.equal(got, r.rotate(q, pos, new(q)))
    for name in names:
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    assert a.status() == b.status() == K.KVE_OK


@pytest.mark.gpu
@pytest.mark.parametrize("inter", [False, True])
def test_cosines_and_sines_to_2_to_the_minus_23(inter):
    # Pairs (a, b) of bf16 numbers at an angle t that turns them to (nearly) (0, b'): a cos t - b sin t is so small there that bf16 rounds
    # it by 2^-28 at most, and the errors of the two products show. With a cosine and a sine off by E each and the product that
    # is rounded by half an fp32 step, 2^-24 |b sin t|, the result is off by (|a| + |b|) E + 2^-24 |b sin t|; the angle's 2^-31 of a turn
    # move it by 2^-28.3 hypot(a, b) more, and its own roundings are relative to it.
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    K = _k()
    rng = np.random.default_rng(11)
    n = 64 * 256
    small = rng.integers(128, 257, n) * np.exp2(-rng.integers(8, 17, n).astype(float))   # bf16 numbers in [2^-9, 1]
    flip = rng.random(n) < 0.5
    a, b = np.where(flip, small, 1.0) * rng.choice([-1, 1], n), np.where(flip, 1.0, small) * rng.choice([-1, 1], n)
    t = np.arctan2(a, b) + rng.uniform(-2.0 ** -20, 2.0 ** -20, n)
    t += np.pi * rng.integers(-1, 2, n)
    first, second = (slice(0, None, 2), slice(1, None, 2)) if inter else (slice(0, 64), slice(64, None))
    x = torch.zeros(n // 64, 1, 128, dtype=torch.bfloat16)
    x[:, 0, first], x[:, 0, second] = (torch.from_numpy(v.reshape(-1, 64)).to(torch.bfloat16) for v in (a, b))
    assert np.array_equal(x[:, 0, first].double().numpy().reshape(-1), a) and np.array_equal(x[:, 0, second].double().numpy().reshape(-1), b)
    x, one = x.cuda(), torch.ones(1, dtype=torch.int32, device="cuda")
    for i in range(n // 64):
        K.Rotary(frequencies=t[64 * i:64 * i + 64], interleaved=inter).rotate(x[i:i + 1], one)
    got = x[:, 0, first].double().cpu().numpy().reshape(-1)
    want = a * np.cos(t) - b * np.sin(t)
    assert np.abs(want).max() < 2.0 ** -19
    bound = ((np.abs(a) + np.abs(b)) * 2.0 ** -23 + 2.0 ** -24 * np.abs(b * np.sin(t)) + 2.0 ** -28.3 * np.hypot(a, b) +
             2.0 ** -8 * np.abs(want) + 2.0 ** -30)
    err = np.abs(got - want)
    assert (err <= bound).all(), float((err / bound).max())
