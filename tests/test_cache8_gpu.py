"""The paged 8-bit cache on the GPU, through the C ABI, against its 64-bit oracle: tables and codes exactly,
the attention within the bounds of tests/cache8.py."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import cache8_oracle as C
from oracle import kv_evict_oracle as O
from paper_2609_30738_gb300 import synth
from paper_2609_30738_gb300.workloads import WORKLOADS, scaled
from tests import cache8 as T
from tests import parity as PT

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_30738_gb300 import kv_evict
    kv_evict.library()
    return kv_evict


def _dev(x):
    return torch.from_numpy(np.array(x)).to(DEV)


def _cache(K, hq, heads, P, num_pages, max_pages, max_seqs, layers=1, pool=None):
    spec = dict(num_layers=layers, num_q_heads=hq, num_kv_heads=heads, head_dim=128)
    bufs = {} if pool is None else dict(zip(("k", "k_scale", "v", "v_scale"), (_dev(x) for x in pool)))
    return K.Cache8(spec, max_seqs, num_pages, max_pages, P, **bufs)


# ------------------------------------------------------------------------------------------------ tables

def _pages_case(rng, layers, seqs, P, hi, kind):
    cap_pages = -(-hi // P)
    f = rng.integers(0, hi + 1, (layers, seqs)).astype(np.int32)
    if kind == "fresh":
        t, f = f, np.zeros_like(f)
    elif kind == "decode":
        f = np.minimum(f, hi - 1)
        t = f + 1
        t[:, rng.random(seqs) < 0.2] = 0
    else:
        t = rng.integers(0, hi + 1, (layers, seqs)).astype(np.int32)
    have = -(-f // P)
    need = -(-t // P)
    total = int(have.sum() + np.maximum(need - have, 0).sum()) + int(rng.integers(0, 9))
    total = max(total, cap_pages)
    order = rng.permutation(total).astype(np.int32)
    table = np.full((layers, seqs, cap_pages), -1, np.int32)
    at = 0
    for l in range(layers):
        for s in range(seqs):
            table[l, s, :have[l, s]] = order[at:at + have[l, s]]
            at += have[l, s]
    head = int(rng.integers(0, total))
    free = np.roll(np.concatenate([order[at:], order[:at]]), head)
    return f, t, table, free, np.array([head, total - at], np.int32)


def _run_pages(c, f, t, table, free, ring, stride, alias=False):
    d = [_dev(x) for x in (f, t, table, free, ring)]
    out_ring = d[4] if alias else torch.full((2,), -9, dtype=torch.int32, device=DEV)
    lens = d[0] if alias else torch.full_like(d[0], -9)
    slots = None if stride is None else torch.full((f.shape[0], stride), -9, dtype=torch.int32, device=DEV)
    c.pages(d[0], d[1], d[2], d[3], d[4], out_ring, lens, slots)
    return [x.cpu().numpy() for x in (d[2], d[3], out_ring, lens)] + [None if slots is None else slots.cpu().numpy()]


@pytest.mark.parametrize("layers,seqs,P,hi,kind", [
    (1, 1, 16, 1, "fresh"), (1, 1, 128, 5000, "fresh"), (3, 5, 32, 70, "any"), (32, 16, 32, 200, "decode"),
    (2, 1024, 16, 40, "any"), (7, 33, 64, 900, "fresh"), (32, 3, 16, 2500, "fresh"), (1, 9, 16, 30011, "any"),
    (256, 64, 16, 33, "decode"), (5, 8, 128, 1, "decode")])
@pytest.mark.parametrize("alias", [False, True])
def test_pages(K, layers, seqs, P, hi, kind, alias):
    rng = np.random.default_rng(layers * 1000 + seqs * 10 + hi)
    f, t, table, free, ring = _pages_case(rng, layers, seqs, P, hi, kind)
    grow = int(np.maximum(t - f, 0).sum(axis=1).max())
    c = _cache(K, 1, 1, P, len(free), table.shape[2], seqs, layers)
    for stride in (grow, grow + 61, None):
        want = C.pages(f, t, table, free, ring, P, stride)
        assert want[5] == "ok"
        got = _run_pages(c, f, t, table, free, ring, stride, alias)
        assert c.status() == K.KVE_OK
        for a, b in zip(got, want):
            assert a is None and b is None or np.array_equal(a, b)


@pytest.mark.parametrize("layers,seqs,kind", [(256, 100, "decode"), (40, 1024, "any"), (200, 200, "fresh")])
@pytest.mark.parametrize("alias", [False, True])
def test_pages_of_more_sequences_than_one_round(K, layers, seqs, kind, alias):
    """More (layer, sequence) pairs than the launch has warps: a CTA has several groups of them."""
    rng = np.random.default_rng(layers + seqs)
    f, t, table, free, ring = _pages_case(rng, layers, seqs, 16, 70, kind)
    grow = int(np.maximum(t - f, 0).sum(axis=1).max())
    c = _cache(K, 1, 1, 16, len(free), table.shape[2], seqs, layers)
    for stride, short in ((grow + 9, 0), (None, 0), (grow, 1)):
        r = ring.copy()
        if short:
            r[1] = max(0, int(np.maximum(-(-t // 16) - -(-f // 16), 0).sum()) - 1)
        want = C.pages(f, t, table, free, r, 16, stride)
        got = _run_pages(c, f, t, table, free, r, stride, alias)
        assert c.status() == {"ok": K.KVE_OK, "pages": K.KVE_EPAGES}[want[5]] and want[5] == ("pages" if short else "ok")
        for a, b in zip(got, want):
            assert a is None and b is None or np.array_equal(a, b)


def test_pages_all_or_nothing(K):
    rng = np.random.default_rng(5)
    f, t, table, free, ring = _pages_case(rng, 4, 6, 16, 300, "any")
    c = _cache(K, 1, 1, 16, len(free), table.shape[2], 6, 4)
    grow = int(np.maximum(t - f, 0).sum(axis=1).max())
    cap = table.shape[2] * 16
    taken = int(np.maximum(-(-t // 16) - -(-f // 16), 0).sum())
    cases = [(f, t, [ring[0], taken - 1], grow, K.KVE_EPAGES), (f, t, [ring[0], taken], grow, K.KVE_OK),
             (f, t, ring, grow - 1, K.KVE_ECUDA), (f, t, [len(free), 1], grow, K.KVE_ECUDA),
             (f, t, [-1, 1], grow, K.KVE_ECUDA), (f, t, [0, len(free) + 1], grow, K.KVE_ECUDA)]
    for value in (-1, cap + 1, -2 ** 31, 2 ** 31 - 1):
        for which in (0, 1):
            x = [f.copy(), t.copy()]
            x[which][2, 3] = value
            cases.append((x[0], x[1], ring, grow, K.KVE_ECUDA))
    for a, b, r, stride, status in cases:
        r = np.array(r, np.int32)
        want = C.pages(a, b, table, free, r, 16, stride)
        assert want[5] == {K.KVE_OK: "ok", K.KVE_EPAGES: "pages", K.KVE_ECUDA: "check"}[status]
        got = _run_pages(c, a, b, table, free, r, stride)
        assert c.status() == status and c.status() == K.KVE_OK
        for x, y in zip(got, want):
            assert np.array_equal(x, y)


@pytest.mark.parametrize("P", [16, 128])
def test_pages_outside_the_pool_give_no_slots(K, P):
    """A ring entry, and the table entry of a page that is filled further, outside the pool: their tokens have no
    slot, the others theirs, the table and the ring move as ever, and the status tells."""
    f = np.array([[P // 2 + 1, 0, 3]], np.int32)
    t = np.array([[P + P // 2, 3 * P - 5, 40 * P]], np.int32)
    n = 60
    for row, entries in ((0, {}), (1, {}), (-7, {}), (0, {2: n}), (0, {0: -1, 30: 2 ** 31 - 1, 36: -2 ** 31})):
        free = np.arange(n, dtype=np.int32)[::-1].copy()
        for i, x in entries.items():
            free[i] = x
        table = np.full((1, 3, 50), -1, np.int32)
        table[0, 0, 0], table[0, 2, 0] = 55 if row < 0 else row, n + 5 if row < 0 else 7
        ring = np.array([0, 50], np.int32)
        want = C.pages(f, t, table, free, ring, P)
        new = [x[:] for x in want[0][0]]
        slots, at = np.full((1, 45 * P), -1, np.int64), 0
        for s in range(3):
            for i in range(f[0, s], t[0, s]):
                page = int(new[s][i // P])
                slots[0, at] = page * P + i % P if 0 <= page < n else -1
                at += 1
        c = _cache(K, 1, 1, P, n, 50, 3)
        for with_slots in (True, False):
            got = _run_pages(c, f, t, table, free, ring, 45 * P if with_slots else None)
            assert c.status() == (K.KVE_ECUDA if row < 0 or entries else K.KVE_OK) and c.status() == K.KVE_OK
            for a, b in zip(got[:4], want[:4]):
                assert np.array_equal(a, b)
            assert got[4] is None or np.array_equal(got[4], slots)


# ------------------------------------------------------------------------------------------------ writers

def _same_pool(c, want):
    for name, t, w in zip(("k", "k_scale", "v", "v_scale"), (c.k, c.k_scale, c.v, c.v_scale), want):
        got = t.cpu().numpy()
        # (a scale that no call has set keeps what its memory held: NaN there is the same on both sides)
        differs = (got != w) & ~(np.isnan(got) & np.isnan(w)) if got.shape == w.shape else got.shape != w.shape
        if np.any(differs):
            at = np.argwhere(differs)
            raise AssertionError(f"{name}: {len(at)} values differ, first at {at[0]}: {got[tuple(at[0])]} {w[tuple(at[0])]}")


def _store_slots(rng, lens, new, P, table):
    out = []
    for i, (a, b) in enumerate(zip(lens, new)):
        pos = np.arange(a, a + b)
        out.append(table[i, pos // P] * P + pos % P if b else np.array([-1]))
    return np.concatenate(out).astype(np.int32)


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("lens,new,heads", [
    ([0], [1], 1), ([5], [1], 8), ([15, 16, 31, 32, 63, 64, 127, 128], [1] * 8, 3), ([0, 0], [300, 129], 2),
    ([7, 130, 0, 3], [200, 1, 0, 125], 4), ([0], [4500], 2), ([3], [4999], 1)])
def test_store(K, P, lens, new, heads):
    rng = np.random.default_rng(P + sum(new))
    table, pages = T.table_for(rng, [a + b for a, b in zip(lens, new)], P)
    k, ks = T.pool(rng, pages, heads, P)
    v, vs = T.pool(rng, pages, heads, P)
    slots = _store_slots(rng, lens, new, P, table)
    n = len(slots)
    kn, vn = T.rows(rng, (n, heads, 128)), T.rows(rng, (n, heads, 128), 2.0)
    kn[rng.random(n) < 0.3] *= 64          # pages whose scale has to grow
    c = _cache(K, heads, heads, P, pages, table.shape[1], len(lens), pool=(k, ks, v, vs))
    for _ in range(2):                     # the same call again changes nothing
        c.store(T.to_torch(kn), T.to_torch(vn), _dev(slots))
        assert c.status() == K.KVE_OK
    ks, vs = ks.astype(np.float64), vs.astype(np.float64)
    C.store(k, ks, kn, slots)
    C.store(v, vs, vn, slots)
    _same_pool(c, (k, ks, v, vs))


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("times", [1, 12])
def test_store_long_and_short_runs_in_one_call(K, P, times):
    """Runs of 1 to 130 rows side by side, padded tokens between them, in calls of both block sizes."""
    rng = np.random.default_rng(P * times)
    new = [1, 9, 8, 1, 130, 7, 0, 2, 10, 1, 16, 17, 1, 33, 3, 65, 1, 1, 8, 9] * times
    lens = [int(x) for x in rng.integers(0, 70, len(new))]
    heads = 2
    table, pages = T.table_for(rng, [a + b for a, b in zip(lens, new)], P)
    k, ks = T.pool(rng, pages, heads, P)
    v, vs = T.pool(rng, pages, heads, P)
    slots = _store_slots(rng, lens, new, P, table)
    n = len(slots)
    assert (n > 1024) == (times > 1)
    kn, vn = T.rows(rng, (n, heads, 128)), T.rows(rng, (n, heads, 128))
    kn[rng.random(n) < 0.1] *= 64
    vn[rng.random(n) < 0.1] *= 16
    c = _cache(K, heads, heads, P, pages, table.shape[1], len(lens), pool=(k, ks, v, vs))
    for _ in range(2):
        c.store(T.to_torch(kn), T.to_torch(vn), _dev(slots))
        assert c.status() == K.KVE_OK
    ks, vs = ks.astype(np.float64), vs.astype(np.float64)
    C.store(k, ks, kn, slots)
    C.store(v, vs, vn, slots)
    _same_pool(c, (k, ks, v, vs))


def test_store_values_that_bf16_can_hold(K):
    rng = np.random.default_rng(9)
    for P in (16, 64):
        k, ks = T.pool(rng, 3, 2, P)
        v, vs = T.pool(rng, 3, 2, P)
        kn, vn = T.rows(rng, (7, 2, 128)), T.rows(rng, (7, 2, 128))
        kn[0, 0, :4] = [np.inf, -np.inf, np.nan, -0.0]
        kn[1, 1] = np.nan
        kn[2] = np.inf
        kn[3] = 0.0
        kn[4] = T.bf16(2.0 ** -133 * rng.integers(0, 200, (2, 128)))      # subnormal
        kn[5] = T.bf16(3e38 * rng.uniform(-1, 1, (2, 128)))
        vn[:, :, ::2] = 0.0
        vn[:, :, 1::2] = -0.0
        for slots in ([0, 1, 2, 3, 4, 5, 6], [P + 3, 1, 2 * P, 5, 2, 2 * P + 9, P - 1]):
            c = _cache(K, 2, 2, P, 3, 1, 3, pool=(k, ks, v, vs))
            a, b = [k.copy(), ks.astype(np.float64)], [v.copy(), vs.astype(np.float64)]
            if len(set(s // P for s in slots)) > 1:
                slots = [slots[0], -1, slots[2], -7, slots[6], -1, -1]    # a page each
            c.store(T.to_torch(kn), T.to_torch(vn), _dev(np.array(slots, np.int32)))
            assert c.status() == K.KVE_OK
            C.store(*a, kn, slots)
            C.store(*b, vn, slots)
            got = c.k.cpu().numpy()
            nan = C.VALUES[a[0]] != C.VALUES[a[0]]
            assert np.array_equal(np.isnan(C.VALUES[got]), nan)
            got[nan] = a[0][nan]           # a NaN has two codes
            c.k.copy_(_dev(got))
            _same_pool(c, (*a, *b))


def test_store_strides_and_slots_outside_the_pool(K):
    rng = np.random.default_rng(11)
    P, heads = 32, 3
    k, ks = T.pool(rng, 4, heads, P)
    v, vs = T.pool(rng, 4, heads, P)
    c = _cache(K, heads, heads, P, 4, 2, 2, pool=(k, ks, v, vs))
    x = T.rows(rng, (9, 2 * heads + 1, 128))
    slots = np.array([30, 31, 32, -1, 128, 2 ** 31 - 1, 100, 101, -2 ** 31], np.int32)
    d = T.to_torch(x)
    c.store(d[:, 1:1 + heads], d[:, 1 + heads:], _dev(slots))
    assert c.status() == K.KVE_ECUDA and c.status() == K.KVE_OK
    ks, vs = ks.astype(np.float64), vs.astype(np.float64)
    C.store(k, ks, x[:, 1:1 + heads], slots)
    C.store(v, vs, x[:, 1 + heads:], slots)
    _same_pool(c, (k, ks, v, vs))


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("perq,major,pinned", [(False, False, False), (True, False, False), (False, True, False),
                                               (False, False, True)])
def test_gather(K, P, perq, major, pinned):
    rng = np.random.default_rng(P)
    layers, hkv, hq, W = 3, 2, 4, 8
    lens, budgets = [400, 33, 150], [70, 41, 1]
    spec = dict(num_layers=layers, num_q_heads=hq, num_kv_heads=hkv, head_dim=128, window=W, budget=70, pool_kernel=1,
                candidate_factor=1, norm_eps=1e-12)
    SL, H = sum(lens), hq if perq else hkv
    k, v = T.rows(rng, (layers, hkv, SL, 128)), T.rows(rng, (layers, hkv, SL, 128))
    idx = np.full((3, layers, H, 70), -1, np.int32)
    for r, L in enumerate(lens):
        for l in range(layers):
            m = min(budgets[l], L - W)
            for h in range(H):
                idx[r, l, h, :m] = np.sort(rng.permutation(L - W)[:m])
    first, S = 2, 6
    rows = np.zeros((layers, S), np.int64)
    for l in range(layers):
        for r, L in enumerate(lens):
            rows[l, first + r] = min(budgets[l], L - W) + W
    table, pages = T.table_for(rng, rows.reshape(-1), P)
    table = table.reshape(layers, S, -1)
    ck, cks = T.pool(rng, pages, H, P)
    cv, cvs = T.pool(rng, pages, H, P)
    c = _cache(K, hq, H, P, pages, table.shape[2], S, layers, (ck, cks, cv, cvs))
    kt, vt, strides = T.to_torch(k, "cpu"), T.to_torch(v, "cpu"), None
    if major:
        kt, vt = (x.permute(0, 2, 1, 3).contiguous() for x in (kt, vt))
        strides = (SL * hkv * 128, 128, hkv * 128)
    kt, vt = (x.pin_memory() if pinned else x.to(DEV) for x in (kt, vt))
    plan = K.Plan(spec, lens, budgets, perq, strides, strides)
    c.gather(plan, kt, vt, _dev(idx), _dev(table), first)
    assert c.status() == K.KVE_OK
    cks, cvs = cks.astype(np.float64), cvs.astype(np.float64)
    off = 0
    for r, L in enumerate(lens):
        for l in range(layers):
            for h in range(H):
                m = min(budgets[l], L - W)
                at = off + np.concatenate([idx[r, l, h, :m], np.arange(L - W, L)])
                kvh = h // (hq // hkv) if perq else h
                for code, scale, src in ((ck, cks, k), (cv, cvs, v)):
                    one, s = code[:, h].copy(), scale[:, h].copy()
                    C.gather(one, s, src[l, kvh, at], table[l, first + r])
                    code[:, h], scale[:, h] = one, s
        off += L
    _same_pool(c, (ck, cks, cv, cvs))


def test_gather_leaves_bad_pages_out(K):
    rng = np.random.default_rng(3)
    spec = dict(num_layers=1, num_q_heads=1, num_kv_heads=1, head_dim=128, window=4, budget=60, pool_kernel=1,
                candidate_factor=1, norm_eps=1e-12)
    pool = T.pool(rng, 4, 1, 16) + T.pool(rng, 4, 1, 16)
    c = _cache(K, 1, 1, 16, 4, 4, 1, pool=pool)
    k = T.rows(rng, (1, 1, 64, 128))
    idx = np.arange(60, dtype=np.int32)[None]
    for table, good in (([3, -1, 4, 1], [3, None, None, 1]), ([2 ** 31 - 1, 0, -2 ** 31, 2], [None, 0, None, 2])):
        c.k.copy_(_dev(pool[0]))
        c.k_scale.copy_(_dev(pool[1]))
        c.gather(K.Plan(spec, [64]), T.to_torch(k), T.to_torch(k), _dev(idx), _dev(np.array(table, np.int32)))
        assert c.status() == K.KVE_ECUDA and c.status() == K.KVE_OK
        want, s = pool[0].copy(), pool[1].astype(np.float64)
        for j, p in enumerate(good):
            if p is not None:
                s[p, 0] = C.write_rows(want[p, 0], 0.0, 0, k[0, 0, 16 * j:16 * j + 16])
        assert np.array_equal(c.k.cpu().numpy(), want) and np.array_equal(c.k_scale.cpu().numpy(), s)


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("bad", [-1, 60, 61, 2 ** 31 - 1, -2 ** 31])
def test_gather_reports_indices_outside_the_candidates(K, P, bad):
    """A kept index outside the candidates is a row of zeros and an error; the others are written as ever."""
    rng = np.random.default_rng(P)
    spec = dict(num_layers=1, num_q_heads=2, num_kv_heads=2, head_dim=128, window=4, budget=20, pool_kernel=1,
                candidate_factor=1, norm_eps=1e-12)
    pages = -(-24 // P)
    pool = T.pool(rng, pages, 2, P) + T.pool(rng, pages, 2, P)
    c = _cache(K, 2, 2, P, pages, pages, 1, pool=pool)
    k = T.rows(rng, (1, 2, 64, 128))
    table = np.arange(pages, dtype=np.int32)
    for at in ([], [7], [0, 19]):
        idx = np.stack([np.sort(rng.permutation(60)[:20]) for _ in range(2)]).astype(np.int32)
        idx[1, at] = bad
        c.k.copy_(_dev(pool[0]))
        c.k_scale.copy_(_dev(pool[1]))
        c.gather(K.Plan(spec, [64]), T.to_torch(k), T.to_torch(k), _dev(idx), _dev(table))
        assert c.status() == (K.KVE_ECUDA if at else K.KVE_OK) and c.status() == K.KVE_OK
        want, s = pool[0].copy(), pool[1].astype(np.float64)
        for h in range(2):
            rows = np.concatenate([k[0, h, np.clip(idx[h], 0, 63)], k[0, h, 60:]])
            if h == 1:
                rows[at] = 0.0
            one, sc = want[:, h].copy(), s[:, h].copy()
            C.gather(one, sc, rows, table)
            want[:, h], s[:, h] = one, sc
        assert np.array_equal(c.k.cpu().numpy(), want) and np.array_equal(c.k_scale.cpu().numpy(), s)


# ------------------------------------------------------------------------------------------------ attention

def _attend(c, q, table, lens, layer=0, lse=True, fill=7.0, stream=None):
    n, t, hq, d = q.shape
    out = torch.full((n, t, hq, d), fill, dtype=torch.bfloat16, device=DEV)
    lt = torch.full((n, t, hq), fill, device=DEV) if lse else None
    c.attend(T.to_torch(q), _dev(table), _dev(lens), layer, out, lt, stream)
    return out.float().cpu().numpy().astype(np.float64), None if lt is None else lt.cpu().numpy().astype(np.float64)


def _attention_case(K, rng, P, G, heads, t, lens, max_pages=None, nan_behind=True, peaked=1.0):
    table, pages = T.table_for(rng, lens, P, max_pages=max_pages)
    k, ks = T.pool(rng, pages, heads, P)
    v, vs = T.pool(rng, pages, heads, P)
    if nan_behind:         # what pages hold behind a sequence must not matter, and is not touched
        for r, L in enumerate(lens):
            if L % P:
                for x in (k, v):
                    x[table[r, L // P], :, L % P:] = 127
    q = T.rows(rng, (len(lens), t, G * heads, 128)) * peaked
    c = _cache(K, G * heads, heads, P, pages, table.shape[1], len(lens), pool=(k, ks, v, vs))
    return c, q, k, ks, v, vs, table, np.array(lens, np.int32)


LENS = [0, 1, 2, 15, 16, 17, 31, 33, 96, 127, 128, 129, 255, 256, 257, 511, 700, 1025]


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("G,heads,t", [(1, 3, 1), (4, 2, 1), (3, 1, 1), (8, 1, 1), (4, 1, 4), (5, 2, 3), (1, 2, 9),
                                       (16, 1, 1), (12, 1, 2), (2, 1, 16), (4, 1, 13), (16, 1, 4), (1, 1, 128),
                                       (128, 1, 1), (7, 1, 18)])
def test_attend(K, P, G, heads, t):
    rng = np.random.default_rng(P * 100 + G * 10 + t)
    c, q, k, ks, v, vs, table, lens = _attention_case(K, rng, P, G, heads, t, LENS)
    out, lse = _attend(c, q, table, lens)
    assert c.status() == K.KVE_OK
    worst = T.check_attention(out, lse, q, k, ks, v, vs, table, lens, G)
    again, lse2 = _attend(c, q, table, lens)
    assert np.array_equal(out, again) and np.array_equal(lse, lse2)      # and no order of arrival in it
    print(f"worst {worst:.3f}")


@pytest.mark.parametrize("lens,G,heads,t", [([20011], 4, 2, 1), ([1, 9000, 0, 4099], 8, 1, 1), ([6000] * 3, 4, 2, 5),
                                            ([130] * 300, 2, 1, 1), ([3] * 1024, 1, 1, 1), ([40000], 1, 1, 1)])
def test_attend_long_and_many(K, lens, G, heads, t):
    rng = np.random.default_rng(len(lens) + lens[0])
    c, q, k, ks, v, vs, table, lens = _attention_case(K, rng, 64, G, heads, t, lens)
    out, lse = _attend(c, q, table, lens)
    assert c.status() == K.KVE_OK
    T.check_attention(out, lse, q, k, ks, v, vs, table, lens, G)


@pytest.mark.parametrize("peaked", [0.0, 1e-3, 8.0, 300.0])
def test_attend_flat_and_peaked(K, peaked):
    rng = np.random.default_rng(int(peaked) + 1)
    c, q, k, ks, v, vs, table, lens = _attention_case(K, rng, 32, 4, 2, 1, [700, 5, 3000], peaked=peaked)
    q = T.bf16(q)
    out, lse = _attend(c, q, table, lens)
    T.check_attention(out, lse, q, k, ks, v, vs, table, lens, 4)


def test_attend_scales_far_apart(K):
    """Pages whose scales differ by many binades, in keys and in values."""
    rng = np.random.default_rng(21)
    for P in (16, 64):
        c, q, k, ks, v, vs, table, lens = _attention_case(K, rng, P, 4, 1, 1, [900, 77])
        ks = np.ldexp(1.0, rng.integers(-20, -5, ks.shape)).astype(np.float32)
        vs = np.ldexp(1.0, rng.integers(-60, 60, vs.shape)).astype(np.float32)
        vs[::3] = 2.0 ** -126
        c.k_scale.copy_(_dev(ks))
        c.v_scale.copy_(_dev(vs))
        out, lse = _attend(c, q, table, lens)
        T.check_attention(out, lse, q, k, ks, v, vs, table, lens, 4)


def test_attend_query_values(K):
    """Rows with tiny, huge and non-finite queries; the other rows are as they were without them."""
    rng = np.random.default_rng(22)
    c, q, k, ks, v, vs, table, lens = _attention_case(K, rng, 32, 4, 2, 2, [300, 0, 1, 64])
    q[0, 0, 1, 5], q[0, 1, 6, 0], q[2, 1, 0, 127], q[1, 0, 0, 0] = np.inf, np.nan, -np.inf, np.nan
    q[3, 1, 3] = 0.0
    q[0, 0, 2] = T.bf16(q[0, 0, 2] * 1e-38)
    q[0, 0, 3, 1:] = T.bf16(q[0, 0, 3, 1:] * 2.0 ** -12)       # one element far above the others
    q[3, 0, 5] = T.bf16(q[3, 0, 5] * 1e4)
    out, lse = _attend(c, q, table, lens)
    T.check_attention(out, lse, q, k, ks, v, vs, table, lens, 4)
    assert np.isnan(out[0, 0, 1]).all() and not np.isnan(out[0, 0, 0]).any()


def test_attend_nan_that_only_later_queries_see(K):
    """A NaN among the newest values reaches the rows that see it and no other; a NaN key likewise."""
    rng = np.random.default_rng(23)
    for G, t in ((4, 4), (2, 20), (1, 128)):
        c, q, k, ks, v, vs, table, lens = _attention_case(K, rng, 16, G, 1, t, [150, 300, 129])
        for r, pos, dim in ((0, 150 - 2, 17), (1, 299, 100), (1, 300 - t + 1, 101), (2, 128, 3)):
            v[table[r, pos // 16], 0, pos % 16, dim] = 255
        k[table[0, 149 // 16], 0, 149 % 16, 9] = 127
        c.v.copy_(_dev(v))
        c.k.copy_(_dev(k))
        out, lse = _attend(c, q, table, lens)
        assert np.isnan(out[0, t - 1]).all() and not np.isnan(out[0, 0]).any()
        T.check_attention(out, lse, q, k, ks, v, vs, table, lens, G)


def test_attend_bad_pages_and_lengths(K):
    rng = np.random.default_rng(24)
    c, q, k, ks, v, vs, table, lens = _attention_case(K, rng, 32, 4, 2, 1, [300, 64, 500], max_pages=17)
    table[0, 3], table[0, 0], table[1, :2], table[2, 15] = -1, len(k), 2 ** 31 - 1, -2 ** 31
    out, lse = _attend(c, q, table, lens)
    assert c.status() == K.KVE_ECUDA and c.status() == K.KVE_OK
    T.check_attention(out, lse, q, k, ks, v, vs, table, lens, 4)
    table, pages = T.table_for(rng, [17 * 32, 1, 500], 32, spare=0)
    table %= len(k)
    for bad, as_if in ((17 * 32 + 1, 17 * 32), (2 ** 31 - 1, 17 * 32), (-1, 0), (-2 ** 31, 0)):
        lens = np.array([bad, 1, 500], np.int32)
        out, lse = _attend(c, q, table, lens)
        assert c.status() == K.KVE_ECUDA
        T.check_attention(out, lse, q, k, ks, v, vs, table, [as_if, 1, 500], 4)


def test_attend_layers_strides_and_rows_behind(K):
    rng = np.random.default_rng(25)
    P, heads, G, t, S, layers = 32, 2, 4, 2, 5, 3
    lens = rng.integers(0, 200, (layers, S)).astype(np.int32)
    table, pages = T.table_for(rng, lens.reshape(-1), P)
    table = table.reshape(layers, S, -1)
    k, ks = T.pool(rng, pages, heads, P)
    v, vs = T.pool(rng, pages, heads, P)
    c = _cache(K, G * heads, heads, P, pages, table.shape[2], S, layers, (k, ks, v, vs))
    n = 3
    x = T.rows(rng, (n, t, G * heads + 3, 128))
    qd = T.to_torch(x)[:, :, 2:2 + G * heads]
    big = torch.full((n, t, 2 * G * heads, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((S, t, G * heads), 7.0, device=DEV)
    c.attend(qd, _dev(table), _dev(lens), 1, big[:, :, ::2], lse[:n])
    assert c.status() == K.KVE_OK
    T.check_attention(big[:, :, ::2].float().cpu().numpy().astype(np.float64), lse[:n].cpu().numpy().astype(np.float64),
                      x[:, :, 2:2 + G * heads], k, ks, v, vs, table[1, :n], lens[1, :n], G)
    assert (big[:, :, 1::2] == 7).all() and (lse[n:] == 7).all()
    # heads outside tokens
    turned = torch.full((G * heads, n, t, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    c.attend(qd, _dev(table), _dev(lens), 2, turned.permute(1, 2, 0, 3))
    T.check_attention(turned.permute(1, 2, 0, 3).float().cpu().numpy().astype(np.float64), None,
                      x[:, :, 2:2 + G * heads], k, ks, v, vs, table[2, :n], lens[2, :n], G)


def test_pool_beyond_32_bit_offsets(K):
    """Pages whose bytes lie beyond 2^32 of the pool's start, written and read."""
    rng = np.random.default_rng(26)
    P, heads, G = 128, 8, 4
    pages = 40000                                      # 5.2 GB of keys
    c = _cache(K, G * heads, heads, P, pages, 8, 2)
    ids = np.array([[pages - 1, 3, 37777, 33000], [39998, 1, 32768, 16384]], np.int32)
    table = np.concatenate([ids, np.full((2, 4), -1, np.int32)], 1)
    lens = np.array([400, 512], np.int32)
    pos = [np.arange(400), np.arange(512)]
    slots = np.concatenate([ids[r, p // P].astype(np.int64) * P + p % P for r, p in enumerate(pos)]).astype(np.int32)
    kn, vn = T.rows(rng, (len(slots), heads, 128)), T.rows(rng, (len(slots), heads, 128))
    c.store(T.to_torch(kn), T.to_torch(vn), _dev(slots))
    q = T.rows(rng, (2, 1, G * heads, 128))
    out, lse = _attend(c, q, table, lens)
    assert c.status() == K.KVE_OK
    order = np.sort(ids.reshape(-1))
    at = torch.from_numpy(order.astype(np.int64)).to(DEV)
    small = {p: i for i, p in enumerate(order)}
    t2 = np.array([[small[p] for p in row] for row in ids], np.int32)
    k, ks, v, vs = (x[at].cpu().numpy() for x in (c.k, c.k_scale, c.v, c.v_scale))
    for r in range(2):
        for h in (0, heads - 1):
            a = np.concatenate([C.VALUES[k[p, h]] * ks[p, h] for p in t2[r]])[:lens[r]]
            rows = kn[sum(lens[:r]):sum(lens[:r + 1]), h]
            for j in range(0, lens[r], P):             # the definition of a page's rows
                s = C.need(rows[j:j + P])
                assert np.array_equal(a[j:j + P], C.VALUES[C.encode(rows[j:j + P] / s)] * s)
    T.check_attention(out, lse, q, k, ks, v, vs, t2, lens, G)


def test_calls_on_another_stream_and_captured(K):
    """Decode steps as a program captures them: one graph that advances lengths, pages and slots in place,
    stores the new rows and attends, replayed; and the same calls on a side stream."""
    rng = np.random.default_rng(27)
    P, heads, G, S, layers = 16, 2, 4, 6, 2
    spec = dict(num_layers=layers, num_q_heads=G * heads, num_kv_heads=heads, head_dim=128)
    c = K.Cache8(spec, S, 64, 5, P)
    table, lens, free, ring = c.state()
    start = np.array([[3, 15, 16, 0, 31, 1], [7, 15, 1, 0, 30, 2]], np.int32)
    slots0 = torch.full((layers, 128), -1, dtype=torch.int32, device=DEV)
    c.pages(lens, _dev(start), table, free, ring, ring, lens, slots0)
    rows = {}
    for l in range(layers):
        n = int(start[l].sum())
        kn, vn = T.rows(rng, (128, heads, 128)), T.rows(rng, (128, heads, 128))
        c.store(T.to_torch(kn), T.to_torch(vn), slots0[l])
        rows[l] = (kn[:n], vn[:n])
    assert c.status() == K.KVE_OK
    to, slots = torch.zeros_like(lens), torch.zeros((layers, S), dtype=torch.int32, device=DEV)
    kd, vd = (torch.zeros((layers, S, heads, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.zeros((layers, S, 1, G * heads, 128), dtype=torch.bfloat16, device=DEV)
    out = torch.zeros_like(q)
    lse = torch.zeros((layers, S, 1, G * heads), device=DEV)

    def step():
        torch.add(lens, 1, out=to)
        c.pages(lens, to, table, free, ring, ring, lens, slots)
        for l in range(layers):
            c.store(kd[l], vd[l], slots[l])
            c.attend(q[l], table, lens, l, out[l], lse[l])

    saved = [x.clone() for x in (lens, table, free, ring)] + [x.clone() for x in (c.k, c.v, c.k_scale, c.v_scale)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert c.status() == K.KVE_OK
    for x, y in zip((lens, table, free, ring, c.k, c.v, c.k_scale, c.v_scale), saved):
        x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, y in zip((lens, table, free, ring, c.k, c.v, c.k_scale, c.v_scale), saved):
        x.copy_(y)
    want = [x.cpu().numpy() for x in (c.k, c.k_scale, c.v, c.v_scale)]
    want[1], want[3] = want[1].astype(np.float64), want[3].astype(np.float64)
    f, tab, fr, rg = (x.cpu().numpy() for x in (lens, table, free, ring))
    for _ in range(20):
        new = [T.rows(rng, (layers, S, heads, 128)) for _ in range(2)]
        qn = T.rows(rng, (layers, S, 1, G * heads, 128))
        kd.copy_(T.to_torch(new[0]))
        vd.copy_(T.to_torch(new[1]))
        q.copy_(T.to_torch(qn))
        graph.replay()
        tab, fr, rg, f, sl, ok = C.pages(f, f + 1, tab, fr, rg, P, S)
        assert ok == "ok" and c.status() == K.KVE_OK
        assert np.array_equal(lens.cpu().numpy(), f) and np.array_equal(table.cpu().numpy(), tab)
        assert np.array_equal(ring.cpu().numpy(), rg) and np.array_equal(slots.cpu().numpy(), sl)
        for l in range(layers):
            C.store(want[0], want[1], new[0][l], sl[l])
            C.store(want[2], want[3], new[1][l], sl[l])
        _same_pool(c, want)
        for l in range(layers):
            T.check_attention(out[l].float().cpu().numpy().astype(np.float64), lse[l].cpu().numpy().astype(np.float64),
                              qn[l], want[0], want[1], want[2], want[3], tab[l], f[l], G)


def test_out_may_be_the_queries(K):
    rng = np.random.default_rng(30)
    for G, t in ((4, 1), (4, 5)):
        c, q, k, ks, v, vs, table, lens = _attention_case(K, rng, 32, G, 2, t, [3000, 5, 0, 700])
        x = T.to_torch(q)
        c.attend(x, _dev(table), _dev(lens), 0, x)
        T.check_attention(x.float().cpu().numpy().astype(np.float64), None, q, k, ks, v, vs, table, lens, G)


def test_binding_checks_what_it_is_given(K):
    c = _cache(K, 8, 2, 16, 8, 4, 3)
    table, lens, free, ring = c.state()
    q = torch.zeros((3, 1, 8, 128), dtype=torch.bfloat16, device=DEV)
    rows = torch.zeros((5, 2, 128), dtype=torch.bfloat16, device=DEV)
    slots = torch.full((5,), -1, dtype=torch.int32, device=DEV)
    bad = [lambda: c.attend(q, table[:, :2], lens, 0, q.clone()), lambda: c.attend(q, table, lens[:, :2], 0, q.clone()),
           lambda: c.attend(q, table, lens, 0, q[:2].clone()), lambda: c.attend(q[0], table, lens, 0, q[0].clone()),
           lambda: c.attend(q, table, lens, 0, q.clone(), torch.zeros((3, 8), device=DEV)),
           lambda: c.store(rows, rows[:4], slots), lambda: c.store(rows, rows, slots[:4]),
           lambda: c.pages(lens, lens, table, free[:7], ring, ring, lens),
           lambda: c.pages(lens[:, :2], lens, table, free, ring, ring, lens),
           lambda: c.pages(lens, lens, table, free, ring, ring, lens, slots),
           lambda: c.pages(lens, lens.long(), table, free, ring, ring, lens),
           lambda: c.pages(lens, lens.cpu(), table, free, ring, ring, lens),
           lambda: c.pages(lens, lens, table, free, ring, ring, lens, slots.reshape(1, 5).long()),
           lambda: c.attend(q, table.long(), lens, 0, q.clone()), lambda: c.attend(q, table, lens.long(), 0, q.clone()),
           lambda: c.attend(q, table, lens, 0, q.clone(), torch.zeros((3, 1, 8), dtype=torch.bfloat16, device=DEV)),
           lambda: c.attend(q, table, lens, 0, q.clone(), torch.zeros((3, 1, 8))),
           lambda: c.attend(q.cpu(), table, lens, 0, q.clone()), lambda: c.attend(q, table, lens, 0, q.cpu()),
           lambda: c.store(rows, rows, slots.long()), lambda: c.store(rows.cpu(), rows, slots),
           lambda: c.store(rows, rows, slots.cpu()), lambda: c.reset(free[:7], ring), lambda: c.reset(free, ring.long())]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(K.KvEvictError):
        c.attend(q, table, lens, 1, q.clone())
    with pytest.raises(K.KvEvictError):
        c.attend(torch.zeros((4, 1, 8, 128), dtype=torch.bfloat16, device=DEV), table, lens, 0, torch.zeros_like(q).repeat(2, 1, 1, 1)[:4])


def test_gather_checks_its_sources(K):
    spec = dict(num_layers=1, num_q_heads=8, num_kv_heads=2, head_dim=128, window=8, budget=16)
    plan, c = K.Plan(spec, [61]), _cache(K, 8, 2, 16, 8, 4, 3)
    table, idx = c.state()[0], torch.zeros((2, 16), dtype=torch.int32, device=DEV)
    good = torch.zeros((1, 2, 61, 128), dtype=torch.bfloat16, device=DEV)
    for bad in (good.float(), good[:, :, :60].contiguous(), good.cpu(), good.view(torch.int16)):
        for k, v in ((bad, good), (good, bad)):
            with pytest.raises(ValueError):
                c.gather(plan, k, v, idx, table)


def test_pool_in_host_memory_is_refused(K):
    """Any of the four tensors on the host, pinned or not, through the binding and through the C call."""
    import ctypes
    spec = dict(num_layers=1, num_q_heads=8, num_kv_heads=2, head_dim=128)
    make = lambda: dict(k=torch.zeros((8, 2, 16, 128), dtype=torch.uint8, device=DEV),  # noqa: E731
                        v=torch.zeros((8, 2, 16, 128), dtype=torch.uint8, device=DEV),
                        k_scale=torch.zeros((8, 2), device=DEV), v_scale=torch.zeros((8, 2), device=DEV))
    cfg = K.CacheConfig(1, 8, 2, 128, 16, 8, 4, 3)

    def create(bufs):
        h, n = ctypes.c_void_p(), ctypes.c_size_t()
        st = K.library().kv_evict_cache_create(ctypes.byref(cfg), *[bufs[x].data_ptr() for x in ("k", "v", "k_scale", "v_scale")],
                                               ctypes.byref(h), ctypes.byref(n))
        K.library().kv_evict_cache_destroy(h)
        return st

    assert create(make()) == K.KVE_OK
    for name in make():
        for pin in (False, True):
            bufs = make()
            host = bufs[name].cpu()
            if pin:
                host = host.pin_memory()
            host = host if host.data_ptr() % 128 == 0 else None
            if host is not None:
                bufs[name] = host
                assert create(bufs) == K.KVE_EINVAL
                with pytest.raises(ValueError):
                    K.Cache8(spec, 3, 8, 4, 16, **bufs)


@pytest.mark.parametrize("G,heads,t,lens", [(4, 2, 1, [5000, 0, 3, 129]), (4, 1, 9, [40, 0, 20000, 5]), (1, 3, 2, [700] * 9)])
def test_attend_over_its_own_queries(K, G, heads, t, lens):
    """out may be q: blocks that several CTAs share have read their queries before one of them writes."""
    rng = np.random.default_rng(31)
    c, q, k, ks, v, vs, table, lens = _attention_case(K, rng, 32, G, heads, t, lens)
    alone = _attend(c, q, table, lens)
    wide = torch.full((q.shape[0], t, G * heads + 3, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    for x in (T.to_torch(q), wide[:, :, 1:1 + G * heads]):
        for _ in range(5):
            x.copy_(T.to_torch(q))
            lse = torch.zeros(q.shape[:3], device=DEV)
            c.attend(x, _dev(table), _dev(lens), 0, x, lse)
            assert c.status() == K.KVE_OK
            assert np.array_equal(x.float().cpu().numpy(), alone[0]) and np.array_equal(lse.cpu().numpy(), alone[1])
    assert bool((wide[:, :, :1] == 7).all()) and bool((wide[:, :, 1 + G * heads:] == 7).all())


def test_empty_batches(K):
    c = _cache(K, 8, 2, 16, 8, 4, 3)
    table, lens, free, ring = c.state()
    none = dict(dtype=torch.bfloat16, device=DEV)
    c.store(torch.empty((0, 2, 128), **none), torch.empty((0, 2, 128), **none), lens[0, :0])
    c.attend(torch.empty((0, 2, 8, 128), **none), table, lens, 0, torch.empty((0, 2, 8, 128), **none),
             torch.empty((0, 2, 8), device=DEV))
    no_slots = torch.empty((1, 0), dtype=torch.int32, device=DEV)
    c.pages(lens, lens.clone(), table, free, ring, ring, lens, no_slots)
    assert c.status() == K.KVE_OK and ring.tolist() == [0, 8]
    c.pages(lens, lens + 1, table, free, ring, ring, lens, no_slots)      # tokens, and room for none
    assert c.status() == K.KVE_ECUDA and ring.tolist() == [0, 8] and lens.tolist() == [[0, 0, 0]]


def test_two_caches_at_once(K):
    """Two caches, each with its own workspace, on two streams at once."""
    rng = np.random.default_rng(28)
    cases = [_attention_case(K, rng, 64, 4, 2, 1, [5000, 300]), _attention_case(K, rng, 32, 8, 1, 2, [7000, 1, 90])]
    alone = [_attend(x[0], x[1], x[6], x[7]) for x in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ins = [(T.to_torch(x[1]), _dev(x[6]), _dev(x[7])) for x in cases]
    outs = [torch.zeros_like(q) for q, _, _ in ins]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, s, (q, table, lens), o in zip(cases, streams, ins, outs):
            x[0].attend(q, table, lens, 0, o, None, s)
    torch.cuda.synchronize()
    for (a, _), o, x in zip(alone, outs, cases):
        assert x[0].status() == K.KVE_OK
        assert np.array_equal(a, o.float().cpu().numpy().astype(np.float64))


def test_eviction_that_finds_too_few_pages_writes_none(K):
    """A sequence's old table entries name pages that others hold by now: where the new pages are refused, the rows
    go nowhere; the next call that is served writes them. On a stream that is not the current one."""
    spec = scaled(WORKLOADS["mistral-1layer-L2048"], num_layers=1, seq_lens=[200], num_kv_heads=2, num_q_heads=8,
                  budget=40)
    batch = synth.make_batch(spec, seed=3)
    plan = K.Plan(spec, batch["seq_lens"])
    bufs = K.Buffers(plan)
    c = K.Cache8(spec, max_seqs=2, num_pages=6, max_pages=6, page_tokens=16)
    table, lens, free, ring = c.state()
    q, k, v = (batch[x].to(DEV) for x in ("q_win", "k", "v"))
    lam = np.full(1, 0.5, np.float32)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        t.zero_()
    for to in ([40, 0], [0, 0], [0, 60]):      # sequence 0 leaves its entries behind, sequence 1 takes pages
        c.pages(lens, _dev(np.array([to], np.int32)), table, free, ring, ring, lens)
    before = [t.cpu().numpy() for t in (c.k, c.k_scale, c.v, c.v_scale)], lens.tolist(), ring.tolist()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        K.run_step_cache8(plan, bufs, c, q, k, v, lam, -lam, table, lens, free, ring, stream=stream)
        assert plan.status(bufs.ws, stream) == K.KVE_OK and c.status(stream) == K.KVE_EPAGES
        _same_pool(c, before[0])
        assert lens.tolist() == before[1] and ring.tolist() == before[2]
        c.gather(plan, k, v, bufs.indices, table, 0, side)      # nor does one behind the status call
        assert c.status(side) == K.KVE_OK
        _same_pool(c, before[0])
    # the same with the pages given back first
    c.pages(lens, torch.zeros_like(lens), table, free, ring, ring, lens)
    torch.cuda.synchronize()
    K.run_step_cache8(plan, bufs, c, q, k, v, lam, -lam, table, lens, free, ring, stream=side)
    assert c.status(side) == K.KVE_OK and lens.tolist() == [[40 + spec["window"], 0]]
    assert all(bool((t != 0).any()) for t in (c.k, c.k_scale, c.v, c.v_scale))


def test_captured_eviction_into_the_cache(K):
    """The step behind its first call: no wait for the device, and captured, replayed on other prompts, what it gives
    eagerly."""
    spec = scaled(WORKLOADS["mistral-1layer-L2048"], num_layers=2, seq_lens=[300, 133], num_kv_heads=2, num_q_heads=8,
                  budget=40)
    plan = K.Plan(spec, [300, 133], layer_budgets=[40, 25])
    bufs = K.Buffers(plan)
    c = K.Cache8(spec, max_seqs=3, num_pages=40, max_pages=6, page_tokens=16)
    table, lens, free, ring = c.state()
    start = [x.clone() for x in (table, lens, free, ring)]
    data = [[synth.make_batch(spec, seed=s)[x].to(DEV) for x in ("q_win", "k", "v")] for s in (4, 5)]
    q, k, v = (x.clone() for x in data[0])
    lam = np.full(2, 0.5, np.float32)

    def step(stream=None):
        K.run_step_cache8(plan, bufs, c, q, k, v, lam, -lam, table, lens, free, ring, first_seq=1, stream=stream)

    def fresh(i):
        for x, y in zip((table, lens, free, ring, q, k, v), start + data[i]):
            x.copy_(y)
        for t in (c.k, c.v, c.k_scale, c.v_scale):
            t.zero_()

    def result():
        assert plan.status(bufs.ws) == K.KVE_OK and c.status() == K.KVE_OK
        return [x.clone() for x in (table, lens, free, ring, c.k, c.v, c.k_scale, c.v_scale)]

    want = []
    for i in (0, 1):
        fresh(i)
        step()
        want.append(result())
    assert want[0][1].tolist() == [[0, 40 + spec["window"], 40 + spec["window"]],
                                   [0, 25 + spec["window"], 25 + spec["window"]]]
    assert not torch.equal(want[0][4], want[1][4])
    fresh(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (1, 0, 1):
        fresh(i)
        graph.replay()
        for a, b in zip(result(), want[i]):
            assert torch.equal(a, b)
    # on a stream behind a long kernel the call returns before that has ended
    side = torch.cuda.Stream()
    fresh(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)      # 0.1 s
        ran = torch.cuda.Event()
        ran.record()
    step(side)
    assert not ran.query()
    side.synchronize()
    for a, b in zip(result(), want[0]):
        assert torch.equal(a, b)


def test_eviction_into_the_cache_then_decode(K):
    """The whole path: score, select, pages and gather of a ragged batch into the cache, then answers that grow it,
    against the oracles of both."""
    spec = scaled(WORKLOADS["mistral-1layer-L2048"], num_layers=2, seq_lens=[700, 433], num_kv_heads=2, num_q_heads=8,
                  budget=40)
    batch = synth.make_batch(spec, seed=8)
    plan = K.Plan(spec, batch["seq_lens"], layer_budgets=[40, 25])
    bufs = K.Buffers(plan)
    c = K.Cache8(spec, max_seqs=4, num_pages=64, max_pages=6, page_tokens=16)
    table, lens, free, ring = c.state()
    q, k, v = (batch[x].to(DEV) for x in ("q_win", "k", "v"))
    lam = np.full(2, 0.5, np.float32)
    K.run_step_cache8(plan, bufs, c, q, k, v, lam, -lam, table, lens, free, ring, first_seq=1)
    assert plan.status(bufs.ws) == K.KVE_OK and c.status() == K.KVE_OK
    W = spec["window"]
    assert lens.cpu().tolist() == [[0, 40 + W, 40 + W, 0], [0, 25 + W, 25 + W, 0]]
    # the rows that the bf16 compact cache would hold, in 8 bits
    plan.gather(k, v, bufs.indices, bufs.k_out, bufs.v_out)
    ko, vo = (x.float().cpu().numpy().astype(np.float64).reshape(2, 2, 2, -1, 128) for x in (bufs.k_out, bufs.v_out))
    want = [x.cpu().numpy() for x in (c.k, c.k_scale, c.v, c.v_scale)]
    want[1], want[3] = want[1].astype(np.float64), want[3].astype(np.float64)
    tab = table.cpu().numpy()
    for r in range(2):
        for l in range(2):
            for h in range(2):
                n = int(lens[l, 1 + r])
                for (code, scale), rows in (((want[0], want[1]), ko), ((want[2], want[3]), vo)):
                    one, s = code[:, h].copy(), scale[:, h].copy()
                    C.gather(one, s, rows[r, l, h, :n], tab[l, 1 + r])
                    code[:, h], scale[:, h] = one, s
    _same_pool(c, want)
    rng = np.random.default_rng(29)
    for _ in range(3):
        to = torch.where(lens > 0, lens + 1, lens)
        slots = torch.zeros((2, 4), dtype=torch.int32, device=DEV)
        c.pages(lens, to, table, free, ring, ring, lens, slots)
        assert int((slots >= 0).sum()) == 4
        for l in range(2):
            kn, vn, qn = T.rows(rng, (4, 2, 128)), T.rows(rng, (4, 2, 128)), T.rows(rng, (4, 1, 8, 128))
            c.store(T.to_torch(kn), T.to_torch(vn), slots[l])
            C.store(want[0], want[1], kn, slots[l].cpu().numpy())
            C.store(want[2], want[3], vn, slots[l].cpu().numpy())
            out, lse = _attend(c, qn, table.cpu().numpy(), lens.cpu().numpy(), l)
            T.check_attention(out, lse, qn, *want, table.cpu().numpy()[l], lens.cpu().numpy()[l], 4)
            assert (out[[0, 3]] == 0).all() and np.isneginf(lse[[0, 3]]).all()
    _same_pool(c, want)
    assert c.status() == K.KVE_OK
