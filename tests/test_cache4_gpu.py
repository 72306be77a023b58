"""The paged 4-bit cache and the rotating append on the GPU, against their definitions in 64 bits."""

import math

import numpy as np
import pytest

from oracle import cache4_oracle as Q
from tests import cache4 as F
from tests import cache8 as T

pytestmark = pytest.mark.gpu


def _k():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_30738_gb300 import kv_evict as K
    return torch, K


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _spec(layers=1, hq=8, hkv=2, window=4, budget=8):
    return dict(num_layers=layers, num_q_heads=hq, num_kv_heads=hkv, head_dim=128, window=window, budget=budget,
                pool_kernel=1, candidate_factor=4 if budget <= 128 else 1)


def _i32(x, device="cuda"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(device)


class Pool:
    """A written 4-bit pool on both sides."""

    def __init__(self, K, rng, spec, pages, P, max_seqs=4, max_pages=None, **kw):
        import torch
        h = spec["num_kv_heads"]
        self.host = [*F.pool(rng, pages, h, P), *F.pool(rng, pages, h, P)]
        k, kp, v, vp = self.host
        dev = [torch.from_numpy(k.copy()).cuda(), F.param_torch(kp), torch.from_numpy(v.copy()).cuda(), F.param_torch(vp)]
        self.cache = K.Cache4(spec, max_seqs=max_seqs, num_pages=pages, max_pages=max_pages or pages, page_tokens=P,
                              k=dev[0], k_param=dev[1], v=dev[2], v_param=dev[3], **kw)

    def check(self):
        c = self.cache
        for got, want in zip((c.k, c.k_param, c.v, c.v_param), self.host):
            got = got.cpu().numpy() if got.dtype.itemsize == 1 else _np(got)
            np.testing.assert_array_equal(got, want)


# ------------------------------------------------------------------------------------------------ rows by slot

SLOT_CASES = [(16, 1, 8, 2), (32, 5, 8, 1), (64, 77, 4, 4), (128, 300, 16, 2), (16, 2000, 8, 8)]


@pytest.mark.parametrize("P,n,hq,hkv", SLOT_CASES)
def test_store(P, n, hq, hkv):
    torch, K = _k()
    rng = np.random.default_rng(P + n)
    spec = _spec(hq=hq, hkv=hkv)
    pages = -(-n // P) + 3
    pool = Pool(K, rng, spec, pages, P)
    slots = rng.permutation(pages * P)[:n]
    slots[rng.random(n) < 0.1] = -1
    k, v = F.rows(rng, (n, hkv, 128)), F.rows(rng, (n, hkv, 128))
    k[0, 0], v[-1, -1, :64] = 3.0, 0.0
    for i in range(2):   # (the second call changes nothing)
        pool.cache.store(T.to_torch(k), T.to_torch(v), _i32(slots))
    Q.store(pool.host[0], pool.host[1], k, slots)
    Q.store(pool.host[2], pool.host[3], v, slots)
    pool.check()
    assert pool.cache.status() == K.KVE_OK


def test_store_of_special_rows():
    torch, K = _k()
    rng = np.random.default_rng(9)
    pool = Pool(K, rng, _spec(hq=2, hkv=1), 3, 16)
    k = F.rows(rng, (12, 1, 128))
    k[0, 0, 7], k[1, 0, 127], k[2, 0, 0] = math.nan, math.inf, -math.inf
    k[3], k[4], k[5] = 0.0, -5.5, T.bf16(np.array(2.0 ** -130))
    k[6, 0, ::2], k[6, 0, 1::2] = 3.3e38, -3.3e38
    k[6] = T.bf16(k[6])
    k[7] = T.bf16(100 + np.arange(128) / 64.0)
    k[8, 0, 3] = T.bf16(np.array(1e30))
    k[9] = T.bf16(k[9] * 1e-37)
    k[10] = -np.abs(k[10])
    k[11] = T.bf16(np.arange(128) * 0.125)        # many ties
    v = k[::-1].copy()
    slots = rng.permutation(48)[:12]
    pool.cache.store(T.to_torch(k), T.to_torch(v), _i32(slots))
    Q.store(pool.host[0], pool.host[1], k, slots)
    Q.store(pool.host[2], pool.host[3], v, slots)
    pool.check()


def test_slots_outside_the_pool_are_left_out():
    torch, K = _k()
    rng = np.random.default_rng(10)
    pool = Pool(K, rng, _spec(), 4, 16)
    k, v = F.rows(rng, (4, 2, 128)), F.rows(rng, (4, 2, 128))
    slots = [64, 3, 2 ** 31 - 1, -(2 ** 31)]
    q = T.to_torch(F.rows(rng, (4, 8, 128)))
    pool.cache.store(T.to_torch(k), T.to_torch(v), _i32(slots))
    Q.store(pool.host[0], pool.host[1], k, slots)
    Q.store(pool.host[2], pool.host[3], v, slots)
    pool.check()
    assert pool.cache.status() == K.KVE_ECUDA and pool.cache.status() == K.KVE_OK
    r, pos = K.Rotary(), _i32([0, 0, 0, 0])
    pool.cache.append(r, pos, T.to_torch(k), T.to_torch(v), _i32(slots), q=q, q_out=torch.empty_like(q))
    pool.check()
    assert pool.cache.status() == K.KVE_ECUDA


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("P,n,hq,hkv,rd,inter,fused", [
    (16, 1, 8, 2, 128, False, True), (16, 9, 2, 2, 64, True, True), (32, 40, 24, 2, 96, False, False),
    (64, 33, 40, 8, 32, False, True), (64, 300, 8, 1, 128, True, False), (128, 1, 1, 1, 16, False, False),
    (128, 1500, 32, 8, 128, False, True), (32, 1100, 4, 4, 80, True, True), (16, 1200, 4, 2, 112, False, True)])
def test_append_is_rotate_then_store(bits, P, n, hq, hkv, rd, inter, fused):
    # bit for bit, from slices of a projection and into runs of every kind; queries too
    torch, K = _k()
    rng = np.random.default_rng(P + n + rd)
    spec = _spec(hq=hq, hkv=hkv)
    r = K.Rotary(128, rd, interleaved=inter, scaling="yarn", factor=4.0, original_length=4096)
    pages = -(-n // P) + 8
    Cache = K.Cache8 if bits == 8 else K.Cache4
    a, b = (Cache(spec, max_seqs=4, num_pages=pages, max_pages=pages, page_tokens=P) for _ in range(2))
    beside = ("k", "v", "k_scale", "v_scale") if bits == 8 else ("k", "v", "k_param", "v_param")
    for name in beside:
        getattr(a, name).fill_(1)
        getattr(b, name).copy_(getattr(a, name))
    # runs: half of the tokens one prompt from the middle of a page on, the others a few each
    order = rng.permutation(pages)
    slots = []
    for i, page in enumerate(order):
        off = int(rng.integers(P)) if i % 2 else 0
        m = P - off if i % 3 else int(rng.integers(1, P - off + 1))
        slots += [int(page) * P + off + j for j in range(m)]
    slots = np.array((slots + [-1] * n)[:n])
    if n > 20:   # (the first of a run: in 8 bits a call writes a page from one place)
        starts = np.append(np.flatnonzero(np.diff(slots) != 1) + 1, 0)
        slots[starts[rng.integers(len(starts))]] = -1
    pos = _i32(rng.integers(0, 200000) + np.arange(n))
    if fused:
        x = T.to_torch(F.rows(rng, (n, hq + 2 * hkv, 128)))
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    else:
        q, k, v = (T.to_torch(F.rows(rng, (n, h, 128))) for h in (hq, hkv, hkv))
    want_q = r.rotate(q, pos, torch.empty(n, hq, 128, dtype=torch.bfloat16, device="cuda"))
    turned = r.rotate(k, pos, torch.empty(n, hkv, 128, dtype=torch.bfloat16, device="cuda"))
    a.store(turned, v, _i32(slots))
    got_q = torch.empty_like(want_q)
    assert b.append(r, pos, k, v, _i32(slots), q=q, q_out=got_q) is got_q
    assert torch.equal(got_q, want_q)
    for name in beside:
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    # without queries, and with them turned in place
    for name in beside:
        getattr(b, name).fill_(1)
    b.append(r, pos, k, v, _i32(slots))
    for name in beside:
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    assert b.append(r, pos, k, v, _i32(slots), q=q) is q and torch.equal(q, want_q)
    assert a.status() == b.status() == K.KVE_OK


def test_append_checks_its_tensors():
    torch, K = _k()
    cache = K.Cache4(_spec(), max_seqs=2, num_pages=4, max_pages=4, page_tokens=16)
    r = K.Rotary()
    k = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda")
    s = p = _i32([0, 1, 2])
    for bad in (dict(positions=p[:2]), dict(positions=p.long()), dict(positions=p.cpu()), dict(q=q[:2]),
                dict(q=q.float()), dict(q_out=q), dict(q=q, q_out=q[:, :4]), dict(k_new=k[:2]), dict(v_new=k.float()),
                dict(k_new=k.cpu()), dict(slots=s.long()), dict(q=q.cpu()), dict(q=q, q_out=q.cpu().pin_memory())):
        a = dict(positions=p, k_new=k, v_new=k, slots=s)
        a.update(bad)
        with pytest.raises(ValueError):
            cache.append(r, a.pop("positions"), a.pop("k_new"), a.pop("v_new"), a.pop("slots"), **a)
    assert cache.append(r, p[:0], k[:0], k[:0], s[:0], q=q[:0]) is not None and cache.status() == K.KVE_OK


# ------------------------------------------------------------------------------------------------ gather

@pytest.mark.parametrize("P,lens,layers,hkv,budget,window,first", [
    (16, [40, 9, 300], 2, 2, 21, 8, 1), (32, [97], 3, 1, 64, 32, 0), (64, [700, 60], 1, 4, 509, 4, 2),
    (128, [33, 34, 35, 36], 1, 2, 1, 1, 0), (16, [2000], 1, 1, 512, 1, 0)])
def test_gather(P, lens, layers, hkv, budget, window, first):
    torch, K = _k()
    rng = np.random.default_rng(P + budget)
    spec = _spec(layers, 2 * hkv, hkv, window, budget)
    plan = K.Plan(spec, lens)
    kept = [min(budget, L - window) for L in lens]
    M = -(-(budget + window) // P)
    seqs = first + len(lens) + 1
    need = [-(-(m + window) // P) for m in kept]
    pages = layers * sum(need) + 3
    pool = Pool(K, rng, spec, pages, P, max_seqs=seqs, max_pages=M)
    order, at = rng.permutation(pages), 0
    table = np.full((layers, seqs, M), -1)
    for l in range(layers):
        for r in range(len(lens)):
            table[l, first + r, :need[r]] = order[at:at + need[r]]
            at += need[r]
    k, v = (F.rows(rng, (layers, hkv, sum(lens), 128)) for _ in range(2))
    idx = np.full((len(lens), layers, hkv, budget), -1)
    off = 0
    for r, L in enumerate(lens):
        for l in range(layers):
            for h in range(hkv):
                pick = np.sort(rng.permutation(L - window)[:kept[r]])
                idx[r, l, h, :kept[r]] = pick
                rows = np.concatenate([pick, np.arange(L - window, L)]) + off
                pg = table[l, first + r]
                for x, (c, f) in ((k, (0, 1)), (v, (2, 3))):
                    Q.gather(pool.host[c][:, h], pool.host[f][:, h], x[l, h, rows], pg)
        off += L
    pool.cache.gather(plan, T.to_torch(k), T.to_torch(v), _i32(idx).view(-1, budget), _i32(table), first_seq=first)
    pool.check()
    assert pool.cache.status() == K.KVE_OK


def test_gather_reports_what_it_cannot_follow():
    torch, K = _k()
    rng = np.random.default_rng(12)
    spec = _spec(1, 2, 1, 2, 4)
    plan = K.Plan(spec, [30])
    pool = Pool(K, rng, spec, 3, 16, max_seqs=1, max_pages=1)
    k = F.rows(rng, (1, 1, 30, 128))
    idx = np.array([[3, -1, 28, 5]])              # -1 and 28 are no candidates
    rows = np.stack([k[0, 0, 3], np.zeros(128), np.zeros(128), k[0, 0, 5], k[0, 0, 28], k[0, 0, 29]])
    pool.cache.gather(plan, T.to_torch(k), T.to_torch(k), _i32(idx), _i32([[[2]]]))
    for c, f in ((0, 1), (2, 3)):
        Q.gather(pool.host[c][:, 0], pool.host[f][:, 0], rows, [2])
    pool.check()
    assert pool.cache.status() == K.KVE_ECUDA
    for page in (3, -1):                          # no such page: nothing written
        pool.cache.gather(plan, T.to_torch(k), T.to_torch(k), _i32([[3, 4, 5, 6]]), _i32([[[page]]]))
        pool.check()
        assert pool.cache.status() == K.KVE_ECUDA


def test_refused_pages_keep_the_gather_from_writing():
    torch, K = _k()
    rng = np.random.default_rng(13)
    spec = _spec(1, 2, 1, 2, 30)
    plan = K.Plan(spec, [64])
    pool = Pool(K, rng, spec, 1, 16, max_seqs=1, max_pages=1)
    _, lens, free, ring = pool.cache.state()
    table = _i32([[[0]]])
    ring.zero_()                                  # none is free
    pool.cache.pages(lens, _i32([[10]]), table, free, ring, ring, lens)
    plan2 = K.Plan(_spec(1, 2, 1, 2, 8), [64])
    k = T.to_torch(F.rows(rng, (1, 1, 64, 128)))
    pool.cache.gather(plan2, k, k, _i32([np.arange(8)]), table)
    pool.check()
    assert pool.cache.status() == K.KVE_EPAGES
    with pytest.raises(K.KvEvictError):
        pool.cache.gather(plan, k, k, _i32([np.arange(30)]), table)


# ------------------------------------------------------------------------------------------------ attention

def _attend(K, rng, lens, P, hq, hkv, t, layers=1, fused=False, shake=None, n_seq=None, check=True):
    """One call over a pool that `shake(k, kp, v, vp, table)` may change; checked against the definition."""
    import torch
    n = len(lens)
    spec = _spec(layers, hq, hkv)
    tables, pages = T.table_for(rng, list(lens) * layers, P)
    M = tables.shape[1]
    tables = tables.reshape(layers, n, M)
    host = [*F.pool(rng, pages, hkv, P), *F.pool(rng, pages, hkv, P)]
    q = F.rows(rng, (n, t, hq, 128), 0.5)
    if shake:
        shake(*host, tables, q)
    k, kp, v, vp = host
    cache = K.Cache4(spec, max_seqs=n, num_pages=pages, max_pages=M, page_tokens=P, k=torch.from_numpy(k).cuda(),
                     k_param=F.param_torch(kp), v=torch.from_numpy(v).cuda(), v_param=F.param_torch(vp))
    lens_t = _i32([lens] * layers)
    if fused:
        wide = torch.zeros(n, t, hq + 2 * hkv, 128, dtype=torch.bfloat16, device="cuda")
        wide[:, :, :hq] = T.to_torch(q)
        qt = wide[:, :, :hq]
    else:
        qt = T.to_torch(q)
    out = torch.full((n, t, hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, t, hq), 7.0, device="cuda")
    layer, s = layers - 1, n if n_seq is None else n_seq
    cache.attend(qt[:s], _i32(tables), lens_t, layer, out[:s], lse[:s])
    assert (out[s:] == 7.0).all() and (lse[s:] == 7.0).all()
    worst = None
    if check:
        worst = F.check_attention(_np(out[:s]), lse[:s].cpu().numpy().astype(np.float64), q[:s], k, kp, v, vp,
                                  tables[layer, :s], np.array(lens[:s]), hq // hkv)
    return cache, out, lse, (qt, _i32(tables), lens_t, layer), worst


@pytest.mark.parametrize("lens,P,hq,hkv,t", [
    ([1], 16, 1, 1, 1), ([1, 2, 15, 16, 17, 31, 32, 33], 16, 4, 2, 1), ([127, 128, 129, 0, 255], 32, 8, 2, 1),
    ([96, 700, 300], 32, 32, 8, 1), ([4000], 64, 8, 1, 1), ([1000, 3], 128, 16, 2, 2), ([500, 64, 77], 16, 32, 8, 4),
    ([333], 64, 24, 2, 1), ([600, 40], 32, 24, 2, 3), ([90, 1], 128, 40, 8, 5), ([257, 256], 64, 8, 8, 8),
    ([300], 16, 64, 1, 2), ([50, 20000], 64, 8, 2, 1), ([3, 2, 1, 0], 16, 8, 2, 4), ([8192] * 2, 16, 4, 4, 1)])
def test_attention(lens, P, hq, hkv, t):
    torch, K = _k()
    cache = _attend(K, np.random.default_rng(sum(lens) + P), lens, P, hq, hkv, t, layers=2, fused=hq > 8)[0]
    assert cache.status() == K.KVE_OK


def test_attention_of_many_sequences_and_of_one_long():
    torch, K = _k()
    rng = np.random.default_rng(20)
    lens = [int(x) for x in rng.integers(0, 400, 200)]
    _attend(K, rng, lens, 16, 4, 1, 1)
    _attend(K, rng, [70001], 128, 4, 1, 1)
    _attend(K, rng, [40000], 32, 16, 1, 1)


@pytest.mark.parametrize("n,longest,P,hq,hkv,t,last", [
    (40, 300, 32, 8, 8, 1, 9000), (40, 300, 16, 32, 8, 2, 4500), (310, 90, 16, 16, 8, 1, 700), (620, 40, 32, 4, 4, 2, 3000),
    (700, 3, 16, 32, 4, 1, 4096), (40, 200, 16, 32, 8, 4, 2500), (62, 200, 64, 32, 8, 4, 3000), (470, 70, 32, 16, 1, 1, 900), (1024, 30, 16, 4, 4, 1, 500)])
def test_attention_of_many_blocks(n, longest, P, hq, hkv, t, last):
    torch, K = _k()
    rng = np.random.default_rng(n + P)
    lens = [int(x) for x in rng.integers(0, longest, n - 1)] + [last]
    cache = _attend(K, rng, lens, P, hq, hkv, t, fused=True)[0]
    assert cache.status() == K.KVE_OK


def test_rows_behind_n_seq_stay_and_empty_batches_are_served():
    torch, K = _k()
    cache, out, _, args, _ = _attend(K, np.random.default_rng(21), [40, 50, 60], 16, 8, 2, 2, n_seq=2)
    before = out.clone()
    cache.attend(args[0][:0], *args[1:], out[:0])
    torch.cuda.synchronize()
    assert torch.equal(out, before) and cache.status() == K.KVE_OK


def test_in_place_and_without_lse():
    torch, K = _k()
    cache, out, _, (q, table, lens, layer), _ = _attend(K, np.random.default_rng(22), [900, 30], 32, 8, 2, 2, fused=True)
    cache.attend(q, table, lens, layer, q)
    assert torch.equal(q, out)


def test_repeats_bit_for_bit():
    torch, K = _k()
    cache, out, lse, args, _ = _attend(K, np.random.default_rng(23), [9000, 100, 12345, 0, 77], 64, 8, 2, 1)
    for _ in range(3):
        again, l2 = torch.empty_like(out), torch.empty_like(lse)
        cache.attend(*args, again, l2)
        assert torch.equal(again, out) and torch.equal(l2, lse)


def test_nan_behind_a_sequence_and_among_its_newest():
    # behind the length nothing counts; a NaN row counts for the queries that see it, and for no other
    torch, K = _k()

    def shake(k, kp, v, vp, tables, q):
        for s, L in enumerate((41, 70)):
            page, off = tables[0, s, L // 16], L % 16
            kp[page, :, off:], vp[page, :, off:] = np.nan, np.nan
        page, off = tables[0, 0, 39 // 16], 39 % 16     # the last but one of sequence 0: its last two drafts see it
        vp[page, 0, off] = np.nan
        page, off = tables[0, 1, 69 // 16], 69 % 16     # the last of sequence 1, a key
        kp[page, 1, off] = np.nan
    _, out, lse, _, _ = _attend(K, np.random.default_rng(24), [41, 70], 16, 8, 2, 4, shake=shake)
    bad = torch.isnan(out).any(-1).cpu()
    assert bad[0, 2:, :4].all() and not bad[0, :2].any() and not bad[0, :, 4:].any()
    assert bad[1, 3, 4:].all() and not bad[1, :3].any() and not bad[1, :, :4].any()


def test_pages_outside_the_pool_are_left_out():
    torch, K = _k()
    for P in (16, 64):
        def shake(k, kp, v, vp, tables, q):
            tables[0, 0, 1], tables[0, 1, 0], tables[0, 2, :] = len(k), -5, 1 << 30
        cache = _attend(K, np.random.default_rng(25), [200, 2 * P - 3, P, 30], P, 8, 2, 2, shake=shake)[0]
        assert cache.status() == K.KVE_ECUDA and cache.status() == K.KVE_OK


def test_a_length_outside_the_table_is_reported():
    torch, K = _k()
    cache, _, _, (q, table, lens, layer), _ = _attend(K, np.random.default_rng(26), [40, 20], 16, 8, 2, 1)
    out = torch.empty_like(q)
    for bad in (-1, 49, 2 ** 31 - 1):
        lens[0, 1] = bad
        cache.attend(q, table, lens, layer, out)
        assert cache.status() == K.KVE_ECUDA


def test_query_rows_that_are_not_finite_or_too_large():
    torch, K = _k()

    def shake(k, kp, v, vp, tables, q):
        q[0, 0, 0, 5], q[0, 0, 3, 127], q[0, 0, 5, 0] = np.nan, np.inf, -np.inf
        q[0, 0, 6] = 0.0
        q[0, 0, 7] = T.bf16(q[0, 0, 7] * 1e-38)
    _attend(K, np.random.default_rng(27), [300], 16, 8, 2, 1, shake=shake)
    _, out, _, _, _ = _attend(K, np.random.default_rng(28), [30], 16, 8, 2, 1, check=False,
                              shake=lambda k, kp, v, vp, tables, q: q.__setitem__((0, 0, 1, 9), 2.0 ** 112))
    bad = torch.isnan(out[0, 0]).all(-1).cpu()
    assert bad.tolist() == [False, True] + [False] * 6


def test_queries_of_widely_different_elements():
    torch, K = _k()

    def shake(k, kp, v, vp, tables, q):
        q[0, 0] *= 2.0 ** -rng.integers(0, 30, q[0, 0].shape)
        q[1, 0] = T.bf16(q[1, 0] * 1e-6)
        kp[tables[0, 1, :2]] = T.bf16(kp[tables[0, 1, :2]] * 1e6)
    rng = np.random.default_rng(29)
    _attend(K, rng, [300, 32], 16, 8, 2, 1, shake=shake)


@pytest.mark.parametrize("hq,hkv,t", [(4, 1, 1), (8, 1, 2)])
def test_values_of_very_different_scales(hq, hkv, t):
    # rows of far larger values that a query does not see, or that hardly count, cost the others nothing; rows without a
    # spread, and values at both ends of bf16's range
    torch, K = _k()
    rng = np.random.default_rng(30)

    def far(k, kp, v, vp, tables, q):
        last = tables[0, 0, 299 // 16], slice(None), 299 % 16
        vp[last] *= 2.0 ** 90
        page, off = tables[0, 1, 3], 5
        vp[page, :, off] *= 2.0 ** 40
        kp[page, :, off, 0] = 0.0
        q[1] = np.abs(q[1])
        kp[page, :, off, 1] = -20.0          # a probability near 0
        vp[tables[0, 2]] *= np.exp2(rng.integers(-100, 20, vp[tables[0, 2]].shape[:-1]))[..., None]
        vp[tables[0, 3], ..., 0] = 0.0       # constant rows
        vp[tables[0, 4]] = T.bf16(vp[tables[0, 4]] * 2.0 ** -118)
    _attend(K, rng, [300, 200, 150, 100, 64], 16, hq, hkv, t, shake=far)

    def large(k, kp, v, vp, tables, q):
        c, f = Q.encode(T.bf16(np.where(rng.random((*v.shape[:3], 128)) < 0.5, 3.3e38, -3.3e38)))
        v[:], vp[:] = Q.pack(c), f
        c, f = Q.encode(T.bf16(np.full((*v.shape[1:3], 128), 3.3e38)))
        v[tables[0, 1]], vp[tables[0, 1]] = Q.pack(c), f
    _, out, _, _, _ = _attend(K, rng, [300, 77], 16, hq, hkv, t, shake=large)
    assert torch.isfinite(out).all()


def test_a_dominating_token():
    torch, K = _k()

    def shake(k, kp, v, vp, tables, q):
        q[:] = np.abs(q)
        kp[tables[0, 0, 2], :, 3] = [0.0, 3.0]    # one key far along every query
        vp[tables[0, 0, 2], :, 3] = 0.0           # without a value
    _attend(K, np.random.default_rng(31), [700], 16, 4, 1, 1, shake=shake)


def test_a_pool_beyond_32_bits():
    # codes from 4 GB on: pages in the last part of a pool of 2^26 rows and more
    torch, K = _k()
    rng = np.random.default_rng(32)
    P, h, pages = 128, 8, (1 << 26) // (128 * 8) + 16
    spec = _spec(1, 8, h)
    cache = K.Cache4(spec, max_seqs=1, num_pages=pages, max_pages=4, page_tokens=P)
    ids = [pages - 1, pages - 5, pages - 9]
    slots = np.concatenate([np.arange(P) + p * P for p in ids])[:300]
    k, v, q = (F.rows(rng, (n, h, 128)) for n in (300, 300, 1))
    cache.store(T.to_torch(k), T.to_torch(v), _i32(slots))
    out = torch.empty(1, 1, 8, 128, dtype=torch.bfloat16, device="cuda")
    cache.attend(T.to_torch(q)[None], _i32([[ids + [-1]]]), _i32([[300]]), 0, out)
    host = []
    for x in (k, v):
        code, f = np.zeros((3, h, P, 64), np.uint8), np.zeros((3, h, P, 2))
        Q.store(code, f, x, np.arange(300))
        host += [code, f]
    F.check_attention(_np(out), None, q[None], *host, np.array([[0, 1, 2]]), [300], 1)
    assert torch.equal(cache.k[pages - 5].cpu(), torch.from_numpy(host[0][1])) and cache.status() == K.KVE_OK


# ------------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("bits", [8, 4])
def test_eviction_then_answers(bits):
    """Rotated prompt -> eviction step into the paged cache -> captured decode steps (pages, append, attend) whose lengths,
    positions and ring move on the GPU; against the definition over what the cache holds."""
    torch, K = _k()
    rng = np.random.default_rng(40)
    Lr, spec = [150, 90], _spec(2, 8, 2, 8, 24)
    r = K.Rotary(128, 64, base=500000.0, scaling="parts", factor=4.0, original_length=128)
    plan = K.Plan(spec, Lr)
    bufs = K.Buffers(plan)
    SL = sum(Lr)
    k = T.to_torch(F.rows(rng, (2, 2, SL, 128)))
    v = T.to_torch(F.rows(rng, (2, 2, SL, 128)))
    q = T.to_torch(F.rows(rng, (2, 2, 8, 8, 128)))           # [layers][requests][heads][window]
    pos = _i32(np.concatenate([np.arange(L) for L in Lr]))
    raw = k.clone()
    r.rotate(k.view(4, SL, 128).transpose(0, 1), pos)        # every layer and head at once
    F.check_rotation(_np(k[1, 1])[:, None], Q.rotate(_np(raw[1, 1])[:, None], pos.cpu().numpy(), r.frequencies), _np(raw[1, 1])[:, None],
                     1.0, 64, False)
    for i, L in enumerate(Lr):
        for l in range(2):
            r.rotate(q[l, i].transpose(0, 1), _i32(np.arange(L - 8, L)))
    Cache = K.Cache8 if bits == 8 else K.Cache4
    cache = Cache(spec, max_seqs=3, num_pages=40, max_pages=5, page_tokens=16)
    table, lens, free, ring = cache.state()
    K.run_step_cache8(plan, bufs, cache, q, k, v, np.full(2, 0.5), np.full(2, -0.5), table, lens, free, ring)
    assert plan.status(bufs.ws) == K.KVE_OK and cache.status() == K.KVE_OK
    assert lens[:, :2].tolist() == [[32, 32], [32, 32]]
    if bits == 4:
        idx = bufs.indices.view(2, 2, 2, 24).cpu().numpy()   # [request][layer][head]
        rows = np.concatenate([idx[1, 1, 0], np.arange(82, 90)]) + 150
        c, f = Q.encode(_np(k[1, 0])[rows])
        pg = table[1, 1, :2].tolist()
        assert np.array_equal(Q.unpack(cache.k[pg, 0].cpu().numpy()).reshape(32, 128), c)
        assert np.array_equal(_np(cache.k_param[pg, 0]).reshape(32, 2), f)
    # one decode step of both sequences, the third stays empty
    x = T.to_torch(F.rows(rng, (2, 3, 12, 128)))             # [layer][sequence][heads of q, k, v]
    at = _i32([150, 90, 0])
    slots = torch.empty(2, 3, dtype=torch.int32, device="cuda")
    to, one = torch.empty_like(lens), _i32([[1, 1, 0]] * 2)
    qr = torch.empty(2, 3, 8, 128, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty(2, 3, 1, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 3, 1, 8, device="cuda")

    def step():
        torch.add(lens, one, out=to)
        cache.pages(lens, to, table, free, ring, ring, lens, slots)
        for l in range(2):
            cache.append(r, at, x[l, :, 8:10], x[l, :, 10:], slots[l], q=x[l, :, :8], q_out=qr[l])
            cache.attend(qr[l].view(3, 1, 8, 128), table, lens, l, out[l], lse[l])
        at.add_(one[0])
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(3):
        x.copy_(T.to_torch(F.rows(rng, (2, 3, 12, 128))))
        graph.replay()
    torch.cuda.synchronize()
    assert cache.status() == K.KVE_OK and lens[:, :2].tolist() == [[36, 36], [36, 36]] and at.tolist() == [154, 94, 0]
    tab, ln = table.cpu().numpy(), lens.cpu().numpy()
    want = Q.rotate(_np(x[1, :, :8]), [153, 93, 0], r.frequencies)
    F.check_rotation(_np(qr[1]), want, _np(x[1, :, :8]), 1.0, 64, False)
    for l in range(2):
        qs = _np(qr[l])[:, None]
        if bits == 4:
            F.check_attention(_np(out[l]), lse[l].cpu().numpy().astype(np.float64), qs, cache.k.cpu().numpy(), _np(cache.k_param),
                              cache.v.cpu().numpy(), _np(cache.v_param), tab[l], ln[l], 4)
        else:
            T.check_attention(_np(out[l]), lse[l].cpu().numpy().astype(np.float64), qs, cache.k.cpu().numpy(), cache.k_scale.cpu().numpy(),
                              cache.v.cpu().numpy(), cache.v_scale.cpu().numpy(), tab[l], ln[l], 4)
    assert not out[:, 2].any() and torch.isneginf(lse[:, 2]).all()


def test_two_caches_on_two_streams():
    torch, K = _k()
    rng = np.random.default_rng(41)
    made = [_attend(K, rng, [3000, 500], 32, 8, 2, 1) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(m[1]) for m in made]
    torch.cuda.synchronize()
    for _ in range(20):
        for m, s, o in zip(made, streams, outs):
            m[0].attend(*m[3], o, None, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, m[1]) for m, o in zip(made, outs))


def test_per_query_head_cache():
    torch, K = _k()
    rng = np.random.default_rng(42)
    spec = _spec(1, 4, 2)
    cache = K.Cache4(spec, max_seqs=1, num_pages=4, max_pages=2, page_tokens=16, per_query_head=True)
    k = F.rows(rng, (20, 4, 128))
    cache.store(T.to_torch(k), T.to_torch(k), _i32(np.arange(20)))
    host = [np.zeros((4, 4, 16, 64), np.uint8), np.zeros((4, 4, 16, 2))]
    Q.store(*host, k, np.arange(20))
    q, out = F.rows(rng, (1, 1, 4, 128)), torch.empty(1, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    cache.attend(T.to_torch(q), _i32([[[0, 1]]]), _i32([[20]]), 0, out)
    F.check_attention(_np(out), None, q, *host, *host, np.array([[0, 1]]), [20], 1)
