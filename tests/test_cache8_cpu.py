"""The paged 8-bit cache without a GPU: its oracle against hand-computed values and library routines, and the
host checks of its calls (they return before any launch, so addresses that are never followed suffice)."""

import ctypes
import os

import numpy as np
import pytest

from oracle import cache8_oracle as C
from tests import cache8 as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_30738_gb300", "libkvevict.so")


def test_codes_are_e4m3():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(1)
    mid = (C.VALUES[:126] + C.VALUES[1:127]) / 2                    # the ties
    x = np.concatenate([rng.standard_normal(20000) * 10 ** rng.uniform(-4, 2, 20000), C.VALUES[:127], mid])
    x = np.clip(np.concatenate([x, -x]), -448, 448).astype(np.float32)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(C.encode(x.astype(np.float64)), ref)
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(C.VALUES, every.astype(np.float64))
    assert C.encode(np.array([1e9, -np.inf, np.nan])).tolist()[:2] == [126, 254]


def test_scale_is_the_smallest_power():
    assert C.need(np.array([448.0])) == 1.0 and C.need(np.array([449.0])) == 2.0
    assert C.need(np.array([1.75])) == 2.0 ** -8 and C.need(np.array([1.7578125])) == 2.0 ** -7
    assert C.need(np.zeros(4)) == 2.0 ** -126
    assert C.need(np.array([np.inf, np.nan, -3.5])) == 2.0 ** -7


def test_growing_scale_keeps_older_codes():
    # a later row eight times larger: the older codes are those that a common scale gives (normal ones)
    rng = np.random.default_rng(2)
    a, b = T.bf16(rng.uniform(0.5, 1, (5, 128))), T.bf16(rng.uniform(4, 8, (2, 128)))
    code, scale = np.zeros((1, 1, 16, 128), np.uint8), np.zeros((1, 1))
    C.store(code, scale, a[:, None], list(range(5)))
    C.store(code, scale, b[:, None], [5, 6])
    both = np.concatenate([a, b])
    assert np.array_equal(code[0, 0, :7], C.encode(both / scale[0, 0]))
    once = code.copy()
    C.store(code, scale, b[:, None], [5, 6])
    assert np.array_equal(code, once)


def test_pages_oracle_by_hand():
    f, t = np.array([[17, 0, 40]], np.int32), np.array([[33, 16, 0]], np.int32)
    table = np.array([[[3, 1, -1], [-1, -1, -1], [0, 6, 2]]], np.int32)
    free = np.array([9, 4, 5, 7, 8, -5, -5, -5, -5, -5], np.int32)
    tab, fr, ring, lens, slots, ok = C.pages(f, t, table, free, np.array([1, 4]), 16, 34)
    assert ok == "ok" and tab.tolist() == [[[3, 1, 4], [5, -1, -1], [0, 6, 2]]]
    assert fr.tolist() == [9, 4, 5, 7, 8, 0, 6, 2, -5, -5] and ring.tolist() == [3, 5]
    assert slots[0].tolist() == [17 + i for i in range(15)] + [64] + [80 + i for i in range(16)] + [-1, -1]
    assert C.pages(f, t, table, free, np.array([1, 1]), 16, 34)[5] == "pages"
    assert C.pages(f, t, table, free, np.array([1, 4]), 16, 31)[5] == "check"


def test_attention_oracle_is_a_softmax():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(3)
    table, n = T.table_for(rng, [37, 5], 16)
    k, ks = T.pool(rng, n, 2, 16)
    v, vs = T.pool(rng, n, 2, 16)
    q = T.rows(rng, (2, 3, 4, 128))
    out, lse, _, _ = C.attend(q, k, ks, v, vs, table, [37, 5], 2)
    for r, L in enumerate([37, 5]):
        for t in range(3):
            m = L - 3 + t + 1
            for hq in range(4):
                kk, vv = (np.concatenate([C.VALUES[c[p, hq // 2]] * s[p, hq // 2] for p in table[r] if p >= 0])[:m]
                          for c, s in ((k, ks), (v, vs)))
                a = torch.from_numpy(kk @ q[r, t, hq] / np.sqrt(128.0))
                np.testing.assert_allclose(out[r, t, hq], torch.softmax(a, 0).numpy() @ vv, rtol=1e-12)
                np.testing.assert_allclose(lse[r, t, hq], torch.logsumexp(a, 0).item(), rtol=1e-12)


# ------------------------------------------------------------------------------------------------ refusals

FAKE, ODD = ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 4)
SIDE = ctypes.c_void_p((1 << 20) + 2)


def _k():
    if not os.path.exists(LIB):
        pytest.skip("library not built")
    from paper_2609_30738_gb300 import kv_evict as K
    return K


def _cfg(K, **over):
    c = dict(num_layers=2, num_q_heads=32, num_kv_heads=8, head_dim=128, page_tokens=32, num_pages=100, max_pages=20,
             max_seqs=4)
    c.update(over)
    return K.CacheConfig(*[c[n] for n, _ in K.CacheConfig._fields_])


def _make(K, cfg, bufs=(FAKE,) * 4):
    h, n = ctypes.c_void_p(), ctypes.c_size_t()
    st = K.library().kv_evict_cache_create(ctypes.byref(cfg), *bufs, ctypes.byref(h), ctypes.byref(n))
    return st, h, n.value


@pytest.mark.parametrize("over", [dict(head_dim=64), dict(page_tokens=48), dict(page_tokens=8), dict(page_tokens=256),
                                  dict(num_q_heads=30), dict(num_q_heads=4), dict(num_kv_heads=0), dict(num_layers=0),
                                  dict(num_layers=257), dict(num_pages=0), dict(max_pages=0), dict(max_pages=101),
                                  dict(max_seqs=0), dict(max_seqs=1025), dict(num_q_heads=2048, num_kv_heads=8),
                                  dict(num_pages=1 << 23, num_kv_heads=8), dict(num_kv_heads=1025, num_q_heads=1025)])
def test_create_refuses(over):
    K = _k()
    st, h, _ = _make(K, _cfg(K, **over))
    assert st == K.KVE_EINVAL and not h.value


def test_create_and_its_workspace():
    K = _k()
    st, h, n = _make(K, _cfg(K))
    assert st == K.KVE_OK and n > 0 and n % 256 == 0
    K.library().kv_evict_cache_destroy(h)
    K.library().kv_evict_cache_destroy(None)
    for bad in range(4):
        for p in (None, ODD):
            st, h, _ = _make(K, _cfg(K), tuple(p if i == bad else FAKE for i in range(4)))
            assert st == K.KVE_EINVAL and not h.value
    assert K.library().kv_evict_strerror(K.KVE_EPAGES) == b"too few free pages"


def test_calls_refuse():
    K = _k()
    lib, (st, h, _) = K.library(), _make(K, _cfg(K))
    i64 = ctypes.c_int64
    pair = lambda a, b: (i64 * 2)(a, b)  # noqa: E731
    assert st == K.KVE_OK
    # pages: lens_from, lens_to, table, free, ring_in, ring_out, lens_out, slots, stride, ws
    ok = [FAKE] * 8 + [10, FAKE]
    for i in range(7):
        for bad in (None, SIDE):
            assert lib.kv_evict_cache_pages(h, *[bad if j == i else x for j, x in enumerate(ok)], None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_pages(h, *ok[:8], -1, FAKE, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_pages(h, *ok[:8], 1 << 31, FAKE, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_pages(h, *ok[:7], SIDE, 10, FAKE, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_pages(h, *ok[:9], ODD, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_pages(None, *ok, None) == K.KVE_EINVAL
    # store: k, v, k_strides, v_strides, slots, n, ws
    good = [FAKE, FAKE, None, None, FAKE, 5, FAKE]
    assert lib.kv_evict_cache_store(h, *good[:5], 0, FAKE, None) == K.KVE_OK      # nothing to do
    assert lib.kv_evict_cache_store(h, None, None, None, None, None, 0, FAKE, None) == K.KVE_OK
    for i, bad in [(0, None), (0, ODD), (1, None), (1, ODD), (2, pair(1024, 4)), (2, pair(-8, 128)), (3, pair(1 << 37, 8)),
                   (4, None), (4, SIDE), (5, -1), (5, 1 << 20), (6, None), (6, ODD)]:
        assert lib.kv_evict_cache_store(h, *[bad if j == i else x for j, x in enumerate(good)], None) == K.KVE_EINVAL, i
    # attend: layer, n_seq, q_tokens, q, q_strides, table, lens, out, out_strides, lse, ws
    good = [1, 4, 1, FAKE, None, FAKE, FAKE, FAKE, None, None, FAKE]
    assert lib.kv_evict_cache_attend(h, *[0 if j == 1 else x for j, x in enumerate(good)], None) == K.KVE_OK
    assert lib.kv_evict_cache_attend(h, 1, 0, 1, None, None, FAKE, FAKE, None, None, None, FAKE, None) == K.KVE_OK
    for i, bad in [(0, -1), (0, 2), (1, -1), (1, 5), (2, 0), (2, 33), (3, None), (3, ODD), (4, pair(4096, 4)),
                   (5, None), (5, SIDE), (6, None), (6, SIDE), (7, None), (7, ODD), (8, pair(64, 128)), (8, pair(4096, 64)),
                   (8, pair(0, 128)), (8, pair(2048, 128)), (9, SIDE), (10, None), (10, ODD)]:
        assert lib.kv_evict_cache_attend(h, *[bad if j == i else x for j, x in enumerate(good)], None) == K.KVE_EINVAL, (i, bad)
    # gather: the plan's layers, heads, requests and rows against the cache's
    spec = dict(num_layers=2, num_q_heads=32, num_kv_heads=8, head_dim=128, window=8, budget=64)
    fits = K.Plan(spec, [300, 200])
    wrong = [(K.Plan(dict(spec, num_layers=1), [300]), 0), (K.Plan(spec, [300], per_query_head=True), 0),
             (K.Plan(dict(spec, num_kv_heads=16), [300]), 0), (fits, -1), (fits, 3),
             (K.Plan(spec, [300] * 5), 0),
             (K.Plan(dict(spec, num_q_heads=8, budget=640 - 7, candidate_factor=0), [2000]), 0)]
    for plan, first in wrong:
        assert lib.kv_evict_cache_gather(h, plan._h, FAKE, FAKE, FAKE, first, FAKE, FAKE, None) == K.KVE_EINVAL
    for i in (0, 1, 2, 4, 5):
        args = [FAKE, FAKE, FAKE, 0, FAKE, FAKE]
        for bad in (None, SIDE):
            assert lib.kv_evict_cache_gather(h, fits._h, *[bad if j == i else x for j, x in enumerate(args)],
                                             None) == K.KVE_EINVAL
    # reset: the ring whole or not at all
    assert lib.kv_evict_cache_reset(h, FAKE, None, FAKE, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_reset(h, None, FAKE, FAKE, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_reset(h, None, None, ODD, None) == K.KVE_EINVAL
    assert lib.kv_evict_cache_status(None, FAKE, None) == K.KVE_EINVAL
    lib.kv_evict_cache_destroy(h)


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    K = _k()
    q = torch.zeros((3, 2, 8, 128), dtype=torch.bfloat16)
    assert K._row_strides(q, 8, "q") is None
    wide = torch.zeros((3, 2, 12, 128), dtype=torch.bfloat16)[:, :, 2:10]
    assert list(K._row_strides(wide, 8, "q")) == [12 * 128, 128]
    one = torch.zeros((3, 1, 12, 128), dtype=torch.bfloat16)[:, :, 2:10]      # a token in each: theirs is the stride
    assert list(K._row_strides(one, 8, "q")) == [12 * 128, 128]
    assert list(K._row_strides(wide[:, 0], 8, "q")) == [24 * 128, 128]
    for bad in (q.float(), q[..., ::2], q.transpose(0, 1), q[:, :, :4]):
        with pytest.raises(ValueError):
            K._row_strides(bad, 8, "q")
    with pytest.raises(ValueError):                                           # pages in host memory
        K.Cache8(dict(num_layers=1, num_q_heads=8, num_kv_heads=2, head_dim=128), 2, 8, 4, 16, device="cpu")


def test_pool_tensors_are_on_one_device():
    torch = pytest.importorskip("torch")
    K = _k()
    here, there = torch.empty(2), torch.empty(2, device="meta")
    assert K.Cache8._one_device([], "cuda") == "cuda"
    assert K.Cache8._one_device([there, there], "cuda") == there.device
    for given in ([here, there], [there, there, here]):
        with pytest.raises(ValueError):
            K.Cache8._one_device(given, "cuda")


def test_sources_of_a_gather_hold_the_plans_rows():
    torch = pytest.importorskip("torch")
    K = _k()
    spec = dict(num_layers=2, num_q_heads=8, num_kv_heads=2, head_dim=128, window=8, budget=16)
    bf = dict(dtype=torch.bfloat16)
    plan = K.Plan(spec, [40, 21])
    for t in (torch.empty((2, 2, 61, 128), **bf), torch.empty(2 * 2 * 61 * 128 + 8, **bf)):
        plan._check_source("k", t)
    for t in (torch.empty((2, 2, 60, 128), **bf), torch.empty((2, 2, 61, 128)), torch.empty((2, 2, 61, 128), dtype=torch.float16),
              torch.empty(0, **bf), torch.empty((2, 61, 2, 128), **bf).transpose(1, 2),
              torch.empty((2, 2, 61, 256), **bf)[..., :128]):
        with pytest.raises(ValueError):
            plan._check_source("v", t)
    # queries' heads own the units, the rows are the KV heads'
    K.Plan(spec, [40, 21], per_query_head=True)._check_source("k", torch.empty((2, 2, 61, 128), **bf))
    # token-major keys: the tensor as it lies, its view, and one token too few; the values are dense
    plan.set_kv_strides((61 * 256, 128, 256), None)
    whole = torch.empty((2, 61, 2, 128), **bf)
    plan._check_source("k", whole)
    plan._check_source("k", whole.transpose(1, 2))
    for name, t in (("k", whole[:, :60].contiguous()), ("k", whole[:1]), ("v", whole.transpose(1, 2))):
        with pytest.raises(ValueError):
            plan._check_source(name, t)
    plan.set_kv_strides(None, None)
    plan._check_source("k", torch.empty((2, 2, 61, 128), **bf))


def test_kept_lens_of_a_plan():
    torch = pytest.importorskip("torch")
    from paper_2609_30738_gb300 import kv_evict as K
    from paper_2609_30738_gb300.workloads import WORKLOADS, scaled
    spec = scaled(WORKLOADS["mistral-1layer-L2048"], num_layers=2, seq_lens=[700, 90], budget=70)
    plan = K.Plan(spec, [700, 90], layer_budgets=[70, 25])
    W = spec["window"]
    lens = torch.tensor([[1, 2, 3, 4], [5, 6, 7, 8]], dtype=torch.int32)
    want = [[1, 70 + W, min(70, 90 - W) + W, 4], [5, 25 + W, 25 + W, 8]]
    assert plan.kept_lens(lens, 1).tolist() == want and lens.tolist() == [[1, 2, 3, 4], [5, 6, 7, 8]]
    for first in (-1, -2, 3):
        with pytest.raises(ValueError):
            plan.kept_lens(lens, first)
