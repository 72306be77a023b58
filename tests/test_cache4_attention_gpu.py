"""Attention over the paged 4-bit cache where its sums come near the ends of fp32, and where its blocks are cut."""

import numpy as np
import pytest

from oracle import cache4_oracle as Q
from tests import cache4 as F
from tests import cache8 as T
from tests.test_cache4_gpu import _attend, _k, _np, _spec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,hq,hkv,t", [([5000, 9000, 300], 4, 1, 1), ([70001], 8, 1, 2), ([3000] * 40, 8, 8, 1)])
def test_small_values_of_long_sequences(lens, hq, hkv, t):
    # s of about 2^-119, the least that a row is written with: none of its bits may go with the length
    torch, K = _k()

    def small(k, kp, v, vp, tables, q):
        vp[:] = T.bf16(vp * 2.0 ** -118)
    cache = _attend(K, np.random.default_rng(sum(lens)), lens, 32, hq, hkv, t, shake=small)[0]
    assert cache.status() == K.KVE_OK


def _one_far(z, codes, size, rest):
    """q = 1/2 everywhere and keys of zeros but one, whose logit is 64 z / sqrt(d): a token of given probability, with values
    of `size`, among some of size `rest`."""
    def shake(k, kp, v, vp, tables, q):
        q[:] = 0.5
        kp[...] = 0.0
        page, off = tables[0, 0, 5], 7
        kp[page, :, off, 1] = z
        vp[:] = T.bf16(vp * rest)
        v[page, :, off] = codes
        vp[page, :, off] = [size, -8 * size]
    return shake


@pytest.mark.parametrize("P,lens,hq,hkv,t", [(128, [9000], 4, 1, 1), (16, [2000], 8, 1, 2)])
@pytest.mark.parametrize("size", [2.0 ** 90, 2.0 ** 100])
def test_far_values_that_hardly_count(P, lens, hq, hkv, t, size):
    # 64 z / sqrt(128) = -83.44: a probability of 2^-120.4 of the others', by values that much larger than theirs. Both parts of
    # such a token's values count, s c and z, which nearly cancel where c is 8.
    torch, K = _k()
    rng = np.random.default_rng(5)
    for codes in (0x88, rng.integers(0, 256, 64)):
        shake = _one_far(-14.75, codes, size, size * 2.0 ** -138)
        cache = _attend(K, np.random.default_rng(lens[0]), lens, P, hq, hkv, t, shake=shake)[0]
        assert cache.status() == K.KVE_OK


def test_the_largest_values_among_small_ones():
    # rows of bf16's largest values behind thousands of small ones and in front of them, at every length's unit
    torch, K = _k()
    rng = np.random.default_rng(6)

    def large(k, kp, v, vp, tables, q):
        c, f = Q.encode(T.bf16(np.where(rng.random((len(lens), v.shape[1], 128)) < 0.5, 3.3e38, -3.3e38)))
        for s, n in enumerate(lens):
            for i in {0, n // 2, n - 1}:
                page, off = tables[0, s, i // 64], i % 64
                v[page, :, off], vp[page, :, off] = Q.pack(c[s]), f[s]
    lens = [5000, 1, 3, 700, 2500]
    _, out, _, _, _ = _attend(K, rng, lens, 64, 8, 2, 1, shake=large)
    assert torch.isfinite(out).all()


def _split_blocks(lens, heads, row_blocks, tile, ctas, part=3):
    """How many blocks of rows fall to two CTAs or more, by the rule of the line: a block counts as its tiles and `part`
    more, all is dealt evenly, and no cut leaves fewer than `least` tiles of a block on one of its sides."""
    blocks = [-(-n // tile) for n in lens if n > 0 for _ in range(heads * row_blocks)]
    units = sum(blocks) + part * len(blocks)
    ctas = max(min(max(units // 4, len(blocks)), ctas), 1)
    least = 4 if units // ctas <= 8 else 2
    cuts = np.array([units * w // ctas for w in range(1, ctas)])
    first = np.cumsum([0] + [n + part for n in blocks])[:-1] + part
    return sum(bool(((cuts - a >= least) & (cuts - a <= n - least)).any()) for a, n in zip(first, blocks))


# a table of at most 2048 tokens and no more blocks than SMs: 8 warps a CTA, tiles of 256 tokens. The rows of a block are dealt
# to 8, 4, 2 (with and without idle warps) or one team of warps at the join, and 9 rows or more take the 16-row kernel
@pytest.mark.parametrize("n,length,P,hq,hkv,t", [
    (16, 2000, 32, 8, 8, 1), (16, 2000, 16, 24, 8, 1), (16, 2000, 64, 32, 8, 1), (16, 2000, 128, 64, 8, 1), (8, 1900, 64, 8, 8, 2),
    (8, 1900, 32, 24, 8, 1), (8, 1900, 16, 40, 8, 1), (8, 1900, 128, 8, 8, 7), (16, 2000, 32, 128, 8, 1), (8, 1900, 64, 24, 8, 4),
    (5, 2000, 32, 32, 8, 4), (4, 2000, 64, 64, 8, 3)])
def test_blocks_of_eight_warps_are_joined(n, length, P, hq, hkv, t):
    torch, K = _k()
    lens = [length - i % 3 for i in range(n)]
    rows, sms = t * hq // hkv, torch.cuda.get_device_properties(0).multi_processor_count
    row_blocks = -(-rows // 16) if rows > 8 else 1
    assert n * hkv * row_blocks <= sms and -(-length // P) * P <= 2048
    if sms == 152:
        assert _split_blocks(lens, hkv, row_blocks, 256, sms) > 0
    cache, out, lse, args, _ = _attend(K, np.random.default_rng(n + hq + t), lens, P, hq, hkv, t, fused=True)
    assert cache.status() == K.KVE_OK
    for _ in range(3):
        again, l2 = torch.empty_like(out), torch.empty_like(lse)
        cache.attend(*args, again, l2)
        assert torch.equal(again, out) and torch.equal(l2, lse)


@pytest.mark.parametrize("lens,P,hq,hkv,t", [([96 + 40 * i for i in range(16)], 32, 32, 8, 1), ([300, 0, 5, 2000], 128, 8, 2, 4),
                                             ([700] * 9, 16, 8, 1, 1)])
def test_a_table_wider_than_its_sequences(lens, P, hq, hkv, t):
    # the width of a table chooses between kernels, not between results
    torch, K = _k()
    rng = np.random.default_rng(sum(lens))
    cache, _, _, (q, table, lens_t, layer), _ = _attend(K, rng, lens, P, hq, hkv, t, check=False)
    spare = max(0, 2049 // P + 1 - cache.num_pages)   # (a table is no wider than the pool)
    grown = [torch.cat([x, x[:1].expand(spare, *x.shape[1:])]) for x in (cache.k, cache.k_param, cache.v, cache.v_param)]
    pages = len(grown[0])
    wide = K.Cache4(_spec(1, hq, hkv), max_seqs=len(lens), num_pages=pages, max_pages=pages, page_tokens=P, k=grown[0],
                    k_param=grown[1], v=grown[2], v_param=grown[3])
    assert pages * P > 2048
    to = torch.full((1, len(lens), pages), -1, dtype=torch.int32, device="cuda")
    to[:, :, :table.shape[2]] = table
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    wide.attend(q, to, lens_t, layer, out, lse)
    F.check_attention(_np(out), lse.cpu().numpy().astype(np.float64), _np(q), cache.k.cpu().numpy(), _np(cache.k_param),
                      cache.v.cpu().numpy(), _np(cache.v_param), table[0].cpu().numpy(), np.array(lens), hq // hkv)
    assert wide.status() == K.KVE_OK
