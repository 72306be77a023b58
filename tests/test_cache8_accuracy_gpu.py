"""Attention over the paged 8-bit cache where the tokens with the largest probabilities are not those that the output
is made of: every term keeps its accuracy against the largest of its own tile, not against the row's.

The bound of a row is that of tests/cache8.py and one term more, the step in which a tile's terms are held: a token's
probability times its page's value scale is a multiple of 2^-25 of the largest such product among the tokens of its tile
(128 positions) that the row sees, so it is off by at most half of that. (Rounding to f16 before, in steps of 2^-32,
adds 2^-33.)"""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import cache8_oracle as C
from tests import cache8 as T

pytestmark = pytest.mark.gpu
DEV = "cuda"
TILE, FLOOR = 128, 2.0 ** -26 + 2.0 ** -33


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_30738_gb300 import kv_evict
    kv_evict.library()
    return kv_evict


def _dev(x):
    return torch.from_numpy(np.array(x)).to(DEV)


def _floor(q, k, ks, v, vs, table, lens, group):
    """Of every output element: the sum over its tiles of half a step times the largest probability times value
    scale, times the codes' magnitudes."""
    n, t, hq, d = q.shape
    P = k.shape[2]
    out = np.zeros(q.shape)
    for r in range(n):
        L = int(lens[r])
        pg = table[r, :-(-L // P)].astype(np.int64)
        for h in range(hq // group):
            kk = (C.VALUES[k[pg, h]] * ks[pg, h].astype(np.float64)[:, None, None]).reshape(-1, d)[:L]
            cc = np.abs(C.VALUES[v[pg, h]]).reshape(-1, d)[:L]
            sc = np.repeat(vs[pg, h].astype(np.float64), P)[:L]
            for i in range(t):
                m = L - t + i + 1
                for g in range(group):
                    l = kk[:m] @ q[r, i, h * group + g] / math.sqrt(d)
                    p = np.exp(l - l.max())
                    p = p / p.sum() * sc[:m]
                    for a in range(0, m, TILE):
                        out[r, i, h * group + g] += FLOOR * p[a:a + TILE].max() * cc[a:min(a + TILE, m)].sum(axis=0)
    return out


def _check(K, q, k, ks, v, vs, table, lens, group):
    n, t, hq, d = q.shape
    spec = dict(num_layers=1, num_q_heads=hq, num_kv_heads=hq // group, head_dim=d)
    c = K.Cache8(spec, n, len(k), table.shape[1], k.shape[2], k=_dev(k), k_scale=_dev(ks.astype(np.float32)), v=_dev(v),
                 v_scale=_dev(vs.astype(np.float32)))
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full(q.shape[:3], 7.0, device=DEV)
    c.attend(T.to_torch(q), _dev(table), _dev(np.array(lens, np.int32)), 0, out, lse)
    assert c.status() == K.KVE_OK
    ref, rl, mass, size = C.attend(q, k, ks, v, vs, table, lens, group)
    got, gl = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    bound = (T.OUT_STEP * np.abs(ref) + (T.P_STEP + 4 * T.LOGIT_STEP * size[..., None]) * mass +
             _floor(q, k, ks, v, vs, table, lens, group) + 1e-37)
    err = np.abs(got - ref)
    assert np.isfinite(got).all() and (err <= bound).all(), float((err / bound)[np.isfinite(err)].max())
    assert (np.abs(gl - rl) <= T.LOGIT_STEP * size + 2.0 ** -20 * (8 + np.abs(rl))).all()


@pytest.mark.parametrize("P,G,t", [(16, 4, 1), (64, 8, 1), (128, 4, 4), (32, 4, 9), (64, 2, 1)])
@pytest.mark.parametrize("n,share", [(96, 0.99), (96, 1 - 2e-6), (700, 0.9993), (4096, 0.998), (4096, 0.9994), (4096, 0.9999),
                                     (16384, 0.987), (1100, 1 - 1e-9)])
@pytest.mark.parametrize("flat", [True, False])
def test_one_token_has_the_probability_and_no_value(K, P, G, t, n, share, flat):
    """Token 0 takes `share` of the probability or so and its values are zeros: the output is the others'."""
    rng = np.random.default_rng(n + P + G + t)
    table, pages = T.table_for(rng, [n], P)
    k, ks = T.pool(rng, pages, 1, P)
    v, vs = T.pool(rng, pages, 1, P)
    ks[:], vs[:] = 2.0 ** -6, 2.0 ** -5
    sign = rng.choice([-1.0, 1.0], 128)
    k[:] = 0 if flat else C.encode(rng.standard_normal(k.shape))
    k[table[0, 0], 0, 0] = C.encode(64.0 * sign)
    if flat:
        v[:] = C.encode(np.array(1.5))
    v[table[0, 0], 0, 0] = 0
    logit = math.log(share / (1 - share) * (n - 1))
    a = logit / (128 * 64.0 * 2.0 ** -6 / math.sqrt(128.0))
    q = T.bf16(a * sign * np.linspace(0.97, 1.0, t * G).reshape(1, t, G, 1))
    _check(K, q, k, ks, v, vs, table, [n], G)


@pytest.mark.parametrize("P,G,t", [(16, 1, 4), (32, 2, 4), (64, 4, 4), (16, 4, 12), (64, 1, 2)])
@pytest.mark.parametrize("up", [3, 20, 28, 36, 60, 100])
def test_a_large_value_page_that_earlier_queries_do_not_see(K, P, G, t, up):
    """The newest draft begins a page whose values are 2^up times the others'."""
    rng = np.random.default_rng(P + up)
    lens = [2 * P + 1, 128 + P + 1, 1025]
    table, pages = T.table_for(rng, lens, P)
    k, ks = T.pool(rng, pages, 1, P)
    v, vs = T.pool(rng, pages, 1, P)
    for r, n in enumerate(lens):
        vs[table[r, n // P], 0] = 2.0 ** (up - 7)
    q = T.rows(rng, (3, t, G, 128))
    _check(K, q, k, ks, v, vs, table, lens, G)


@pytest.mark.parametrize("P,G,t", [(16, 1, 4), (32, 2, 4), (64, 4, 4)])
@pytest.mark.parametrize("low,high", [(-10, 119), (-30, 119), (-70, 119), (-126, 40), (-60, 0)])
def test_values_at_both_ends_of_the_range_in_a_tile(K, P, G, t, low, high):
    """Pages of scale 2^low that every query sees, and one of 2^high that only the newest does."""
    rng = np.random.default_rng(P - low)
    lens = [2 * P + 1, 128 + P + 1, 1025]
    table, pages = T.table_for(rng, lens, P)
    k, ks = T.pool(rng, pages, 1, P)
    v, vs = T.pool(rng, pages, 1, P)
    vs[:] = 2.0 ** low
    for r, n in enumerate(lens):
        vs[table[r, n // P], 0] = 2.0 ** high
    q = T.rows(rng, (3, t, G, 128))
    _check(K, q, k, ks, v, vs, table, lens, G)


@pytest.mark.parametrize("P,G,t", [(16, 4, 1), (32, 4, 2), (64, 4, 4), (16, 1, 1)])
@pytest.mark.parametrize("up,down", [(20, 10), (40, 40), (40, 60), (60, 30), (100, 110), (2, 30)])
def test_a_large_value_page_with_small_probabilities(K, P, G, t, up, down):
    """Pages whose values are 2^up times the others' and whose probabilities 2^-down of theirs."""
    rng = np.random.default_rng(up + down)
    n = 700
    table, pages = T.table_for(rng, [n], P)
    k, ks = T.pool(rng, pages, 1, P)
    v, vs = T.pool(rng, pages, 1, P)
    ks[:], vs[:] = 2.0 ** -6, 2.0 ** -7
    sign = rng.choice([-1.0, 1.0], 128)
    k[:] = C.encode(rng.standard_normal(k.shape))
    a = down * math.log(2.0) / (128 * 64.0 * 2.0 ** -6 / math.sqrt(128.0))
    for j in (1, 3, 700 // P - 1):
        k[table[0, j], 0] = C.encode(-64.0 * sign)
        vs[table[0, j], 0] = 2.0 ** (up - 7)
    q = T.bf16(a * sign * np.linspace(0.97, 1.0, t * G).reshape(1, t, G, 1))
    _check(K, q, k, ks, v, vs, table, [n], G)


@pytest.mark.parametrize("P,G,t", [(16, 4, 1), (64, 8, 1), (128, 4, 4)])
@pytest.mark.parametrize("n", [1, 96, 3000, 20011])
def test_values_near_the_largest_that_bf16_holds(K, P, G, t, n):
    """An average of values of 2e38 and more is one of them, whatever its unnormalised sum would be."""
    rng = np.random.default_rng(n + P)
    table, pages = T.table_for(rng, [n], P)
    k, ks = T.pool(rng, pages, 1, P)
    v, vs = T.pool(rng, pages, 1, P)
    v[:] = C.encode(rng.uniform(320, 416, v.shape))
    vs[:] = 2.0 ** 119
    q = T.rows(rng, (1, t, G, 128))
    if t > 1 and n < t:
        q = q[:, :1]
    _check(K, q, k, ks, v, vs, table, [n], G)
