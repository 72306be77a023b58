"""Rows of the paged 4-bit cache where its formulas' roundings show, by hand."""

import numpy as np
import pytest

from oracle import cache4_oracle as Q
from tests import cache8 as T


def _rows():
    """Rows [n][128] of bf16 numbers, their s, and the code of their element 0."""
    x, s, c = np.zeros((5, 128)), [], []

    def row(low, high, first, step, code):
        i = len(s)
        x[i], x[i, 1], x[i, 2], x[i, 0] = high, low, high, first
        s.append(step)
        c.append(code)
    # (22.5 + 15 / 256) / 15 = 1.50390625 and 22.79296875 / 15 = 1.51953125, between two bf16 numbers: fl(16 / 15) is above 16 / 15
    # by 5.6e-8, and fl(fl(d / 16) * that) by an fp32 step above the middle
    row(-15 / 256, 22.5, 22.5, 1.5078125, 15)
    row(-22.125, 0.66796875, -22.125, 1.5234375, 0)
    # 3855 / 15 = 257 exactly: that product is 257 again (half an fp32 step is more than it is off there), a tie to the even 256
    row(-15.0, 3840.0, -15.0, 256.0, 0)
    # s = RN_bf16(662.125 / 15) = 44.25 and fl(2^-20 + 22.125) = 22.125, half of it: to the even code; 2^-18 more is above the half
    row(-22.125, 640.0, 2.0 ** -20, 44.25, 0)
    row(-22.125, 640.0, 2.0 ** -18, 44.25, 1)
    assert np.array_equal(T.bf16(x), x)
    return x, s, c


def test_the_definition():
    x, s, c = _rows()
    code, param = Q.encode(x)
    assert param[:, 0].tolist() == s and code[:, 0].tolist() == c
    assert param[:, 1].tolist() == x[:, 1].tolist() and (code[:, 2] == 15).all() and not code[:, 1].any()


@pytest.mark.gpu
def test_the_kernel():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_30738_gb300 import kv_evict as K
    x, s, c = _rows()
    n = len(x)
    spec = dict(num_layers=1, num_q_heads=1, num_kv_heads=1, head_dim=128, window=1, budget=n - 1, pool_kernel=1, candidate_factor=1)
    rows, slots = T.to_torch(x)[:, None], torch.arange(n, dtype=torch.int32, device="cuda")
    zero = torch.zeros(n, dtype=torch.int32, device="cuda")
    plan = K.Plan(spec, [n])
    keep = torch.arange(n - 1, dtype=torch.int32, device="cuda")[None]
    write = dict(store=lambda k: k.store(rows, rows, slots),
                 append=lambda k: k.append(K.Rotary(), zero, rows, rows, slots),   # (position 0 turns nothing)
                 gather=lambda k: k.gather(plan, rows.view(1, 1, n, 128), rows.view(1, 1, n, 128), keep, zero[:1].view(1, 1, 1)))
    for name, call in write.items():
        cache = K.Cache4(spec, max_seqs=1, num_pages=1, max_pages=1, page_tokens=16)
        call(cache)
        for code, param in ((cache.k, cache.k_param), (cache.v, cache.v_param)):
            got = Q.unpack(code[0, 0, :n].cpu().numpy())
            assert param[0, 0, :n, 0].tolist() == s and param[0, 0, :n, 1].tolist() == x[:, 1].tolist(), name
            assert got[:, 0].tolist() == c and (got[:, 2] == 15).all() and not got[:, 1].any(), name
        assert cache.status() == K.KVE_OK
