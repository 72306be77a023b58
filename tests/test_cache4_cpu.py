"""Rotary positions and the paged 4-bit cache without a GPU: their oracle against hand-computed values, the frequencies,
and the host checks of the calls (they return before any launch, so addresses that are never followed suffice)."""

import ctypes
import math
import os

import numpy as np
import pytest

from oracle import cache4_oracle as Q
from tests import cache4 as F
from tests import cache8 as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_30738_gb300", "libkvevict.so")
FAKE, ODD, SIDE = ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 4), ctypes.c_void_p((1 << 20) + 2)


def _k():
    if not os.path.exists(LIB):
        pytest.skip("library not built")
    from paper_2609_30738_gb300 import kv_evict as K
    return K


# ------------------------------------------------------------------------------------------------ oracle

def test_codes_by_hand():
    x = np.zeros((3, 128))
    x[0, :4] = [-1.0, 14.0, 0.5, 1.5]            # s = 1: ties to the even code
    x[1] = 7.25                                   # no spread
    x[2, 5] = np.inf
    c, f = Q.encode(x)
    assert f[0].tolist() == [1.0, -1.0] and c[0, :5].tolist() == [0, 15, 2, 2, 1]
    assert f[1].tolist() == [0.0, 7.25] and not c[1].any()
    assert np.isnan(f[2]).all() and not c[2].any()
    assert Q.pack(c)[0, :2].tolist() == [0xF0, 0x22]
    assert np.array_equal(Q.unpack(Q.pack(c)), c)


def test_an_element_is_off_by_half_a_step():
    x = F.rows(np.random.default_rng(1), (500, 128), 2.0)
    c, f = Q.encode(x)
    off = np.abs(Q.values(Q.pack(c), f) - x)
    assert (off <= 0.53 * f[:, :1]).all() and c.max() == 15 and c.min() == 0


def test_extreme_rows_have_finite_numbers():
    big = T.bf16(np.full(128, 3.38e38))
    big[::2] *= -1
    c, f = Q.encode(np.stack([big, big * 2.0 ** -250, np.full(128, -0.0)]))
    assert np.isfinite(f).all() and (c[0, 1::2] == 15).all() and f[1, 0] == 0 and not np.signbit(f[2, 1])


def test_attention_oracle_is_a_softmax():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(3)
    table, n = T.table_for(rng, [37, 5], 16)
    k, kp = F.pool(rng, n, 2, 16)
    v, vp = F.pool(rng, n, 2, 16)
    q = F.rows(rng, (2, 3, 4, 128))
    out, lse = Q.attend(q, k, kp, v, vp, table, [37, 5], 2)[:2]
    for r, L in enumerate([37, 5]):
        for t in range(3):
            m = L - 3 + t + 1
            for hq in range(4):
                kk, vv = (np.concatenate([Q.values(c[p, hq // 2], f[p, hq // 2]) for p in table[r] if p >= 0])[:m]
                          for c, f in ((k, kp), (v, vp)))
                a = torch.from_numpy(kk @ q[r, t, hq] / np.sqrt(128.0))
                np.testing.assert_allclose(out[r, t, hq], torch.softmax(a, 0).numpy() @ vv, rtol=1e-12)
                np.testing.assert_allclose(lse[r, t, hq], torch.logsumexp(a, 0).item(), rtol=1e-12)


def test_rotation_keeps_lengths_and_depends_on_differences():
    rng = np.random.default_rng(4)
    f, _ = Q.frequencies("none", 64)
    q, k = rng.standard_normal((1, 1, 128)), rng.standard_normal((1, 1, 128))
    for inter in (False, True):
        at = lambda x, p: Q.rotate(x, [p], f, 1.0, inter)[0, 0]  # noqa: E731
        assert math.isclose(np.linalg.norm(at(q, 1234)), np.linalg.norm(q), rel_tol=1e-12)
        assert math.isclose(at(q, 1000) @ at(k, 990), at(q, 10) @ at(k, 0), rel_tol=1e-9)
        back = Q.rotate(Q.rotate(q, [77], f, 1.0, inter), [77], f, 1.0, inter, True)
        np.testing.assert_allclose(back, q, atol=1e-12)
    quarter = Q.rotate(np.eye(1, 128)[None], [1], np.full(8, math.pi / 2))
    assert abs(quarter[0, 0, 8] - 1) < 1e-12 and abs(quarter[0, 0, 0]) < 1e-12


def test_transpose_is_the_gradient():
    # central differences of sum(g * rotate(x)) against the transposed rotation of g
    rng = np.random.default_rng(5)
    f, amp = Q.frequencies("yarn", 32, 10000.0, 4.0, 2048, 1, 32)
    x, g = rng.standard_normal((2, 1, 128)), rng.standard_normal((2, 1, 128))
    loss = lambda y: (g * Q.rotate(y, [5, 900], f, amp, True)).sum()  # noqa: E731
    grad = Q.rotate(g, [5, 900], f, amp, True, True)
    for i in (0, 1, 17, 31, 32, 127):
        d = np.zeros_like(x)
        d[1, 0, i] = 1e-3
        assert abs((loss(x + d) - loss(x - d)) / 2e-3 - grad[1, 0, i]) < 1e-8


# ------------------------------------------------------------------------------------------------ frequencies

@pytest.mark.parametrize("n", [16, 32, 96, 128])
@pytest.mark.parametrize("kind,over", [("none", {}), ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0)),
                                       ("parts", dict(factor=8.0, original=8192.0)),
                                       ("yarn", dict(factor=16.0, original=4096.0, high=32.0)),
                                       ("yarn", dict(factor=2.0, original=100.0, high=32.0)),
                                       ("yarn", dict(factor=2.0, original=1e9, high=32.0))])
def test_frequencies(n, kind, over):
    K = _k()
    o = dict(base=500000.0, factor=1.0, original=0.0, low=1.0, high=4.0)
    o.update(over)
    want, amp = Q.frequencies(kind, n, **o)
    r = K.Rotary(128, n, base=o["base"], scaling=kind, factor=o["factor"], original_length=o["original"],
                 low_turns=o["low"], high_turns=o["high"])
    np.testing.assert_allclose(r.frequencies, want, rtol=1e-13)
    assert math.isclose(r.amplitude, amp, rel_tol=1e-15) and r.rotary_dim == n


@pytest.mark.parametrize("over", [dict(base=1.0), dict(base=math.nan), dict(scaling="linear", factor=0.5),
                                  dict(scaling="parts", factor=2.0), dict(scaling="ntk", factor=math.inf),
                                  dict(scaling="parts", factor=2.0, original_length=100, low_turns=4.0, high_turns=4.0),
                                  dict(scaling="yarn", factor=2.0, original_length=100, low_turns=0.0),
                                  dict(rotary_dim=8), dict(rotary_dim=24), dict(rotary_dim=144), dict(rotary_dim=0),
                                  dict(head_dim=64), dict(amplitude=math.inf), dict(frequencies=[math.nan] * 64)])
def test_rotary_refuses(over):
    K = _k()
    with pytest.raises(K.KvEvictError):
        K.Rotary(**over)


def test_rotary_refuses_names_and_counts():
    K = _k()
    with pytest.raises(ValueError):
        K.Rotary(scaling="dynamic")
    with pytest.raises(ValueError):
        K.Rotary(frequencies=np.ones(63))


def _rotary(K):
    return K.Rotary()


def test_apply_refuses():
    K = _k()
    r = _rotary(K)
    s = lambda *v: (ctypes.c_int64 * 2)(*v)  # noqa: E731
    good = [r._h, FAKE, None, FAKE, None, 8, FAKE, 16, 0, None]
    apply = K.library().kv_evict_rotary_apply

    def refused(**over):
        a = list(good)
        for i, v in over.items():
            a[int(i[1:])] = v
        return apply(*a) == K.KVE_EINVAL
    assert refused(a0=None) and refused(a1=None) and refused(a3=None) and refused(a6=None)
    assert refused(a1=ODD, a3=ODD) and refused(a3=SIDE) and refused(a6=SIDE)
    assert refused(a5=0) and refused(a7=-1) and refused(a8=2) and refused(a7=1 << 28)
    assert refused(a2=s(1024, 100)) and refused(a2=s(-1024, 128)) and refused(a2=s(1 << 37, 128))
    assert refused(a4=s(1024, 64)) and refused(a4=s(512, 128)) and refused(a4=s(0, 128))
    assert refused(a2=s(2048, 128)) and refused(a4=s(2048, 128))       # in place at other strides
    assert apply(r._h, None, None, None, None, 8, None, 0, 0, None) == K.KVE_OK


# ------------------------------------------------------------------------------------------------ refusals of the cache

def _make4(K, bufs=(FAKE,) * 4, **over):
    c = dict(num_layers=2, num_q_heads=32, num_kv_heads=8, head_dim=128, page_tokens=32, num_pages=100, max_pages=20,
             max_seqs=4)
    c.update(over)
    cfg = K.CacheConfig(*[c[n] for n, _ in K.CacheConfig._fields_])
    h, n = ctypes.c_void_p(), ctypes.c_size_t()
    st = K.library().kv_evict_cache4_create(ctypes.byref(cfg), *bufs, ctypes.byref(h), ctypes.byref(n))
    return st, h, n.value


@pytest.mark.parametrize("over", [dict(head_dim=64), dict(page_tokens=48), dict(page_tokens=8), dict(num_q_heads=30),
                                  dict(num_kv_heads=0), dict(num_layers=0), dict(num_pages=0), dict(max_pages=101),
                                  dict(max_seqs=1025), dict(num_q_heads=2048), dict(num_pages=1 << 23)])
def test_create_refuses(over):
    K = _k()
    st, h, _ = _make4(K, **over)
    assert st == K.KVE_EINVAL and not h.value


def test_create_checks_addresses():
    K = _k()
    for i in range(4):
        for bad in (None, ODD):
            bufs = [FAKE] * 4
            bufs[i] = bad
            assert _make4(K, bufs)[0] == K.KVE_EINVAL
    st, h, n = _make4(K)
    assert st == K.KVE_OK and n > 0
    K.library().kv_evict_cache_destroy(h)


def test_append_refuses():
    K = _k()
    r, lib = _rotary(K), K.library()
    st, h, _ = _make4(K)
    assert st == K.KVE_OK
    ws = ctypes.c_void_p(1 << 20)
    s = lambda *v: (ctypes.c_int64 * 2)(*v)  # noqa: E731
    good = [h, r._h, FAKE, FAKE, None, FAKE, None, FAKE, FAKE, None, None, FAKE, 4, ws, None]

    def refused(**over):
        a = list(good)
        for i, v in over.items():
            a[int(i[1:])] = v
        return lib.kv_evict_cache_append(*a) == K.KVE_EINVAL
    for i in (0, 1, 2, 7, 8, 11, 13):
        assert refused(**{"a%d" % i: None}), i
    assert refused(a3=None) and refused(a5=None)                       # both or neither
    for i, bad in ((2, SIDE), (3, ODD), (5, ODD), (7, ODD), (8, ODD), (11, SIDE), (13, ODD)):
        assert refused(**{"a%d" % i: bad}), i
    assert refused(a12=-1) and refused(a12=1 << 20)
    assert refused(a4=s(4096, 100)) and refused(a6=s(4096, 64)) and refused(a6=s(128, 128)) and refused(a6=s(8192, 128))
    assert refused(a9=s(-8, 128)) and refused(a10=s(1024, 4))
    none = list(good)
    none[12] = 0
    for i in (2, 3, 5, 7, 8, 11):
        none[i] = None
    assert lib.kv_evict_cache_append(*none) == K.KVE_OK
    lib.kv_evict_cache_destroy(h)


def test_attend_and_store_refuse_on_a_4_bit_cache():
    K = _k()
    st, h, _ = _make4(K)
    lib, ws = K.library(), ctypes.c_void_p(1 << 20)
    assert lib.kv_evict_cache_attend(h, 2, 1, 1, FAKE, None, FAKE, FAKE, FAKE, None, None, ws, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_attend(h, 0, 1, 33, FAKE, None, FAKE, FAKE, FAKE, None, None, ws, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_attend(h, 0, 5, 1, FAKE, None, FAKE, FAKE, FAKE, None, None, ws, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_attend(h, 0, 1, 1, ODD, None, FAKE, FAKE, FAKE, None, None, ws, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_store(h, FAKE, ODD, None, None, FAKE, 1, ws, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_attend(h, 0, 0, 1, None, None, FAKE, FAKE, None, None, None, ws, None) == K.KVE_OK
    lib.kv_evict_cache_destroy(h)


def test_bindings_check_their_tensors():
    torch = pytest.importorskip("torch")
    K = _k()
    r = _rotary(K)
    x = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    p = torch.zeros(4, dtype=torch.int32)
    for bad in ((x, p), (x, p.long()), (x, p[:3]), (x[..., :64], p), (x[0], p)):
        with pytest.raises(ValueError):
            r.rotate(*bad)
    with pytest.raises(ValueError):
        K.Cache4(dict(num_layers=1, num_q_heads=8, num_kv_heads=8, head_dim=128), 1, 4, 4, k=torch.zeros(4, 8, 64, 64, dtype=torch.uint8),
                 v=torch.zeros(4, 8, 64, 64, dtype=torch.uint8), k_param=torch.zeros(4, 8, 64, 2), v_param=torch.zeros(4, 8, 64, 2))
