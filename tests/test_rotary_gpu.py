"""Rotary positions on the GPU against their definition in 64 bits."""

import math

import numpy as np
import pytest

from oracle import cache4_oracle as Q
from tests import cache4 as F
from tests.cache8 import to_torch

pytestmark = pytest.mark.gpu


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _k():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_30738_gb300 import kv_evict as K
    return torch, K


CASES = [(128, False, "none", 1, 1, 0), (128, False, "none", 7, 3, 0), (128, True, "linear", 40, 5, 100000),
         (64, False, "parts", 33, 40, 4000000), (64, True, "yarn", 129, 2, 31), (96, False, "ntk", 16, 8, 1 << 30),
         (32, True, "none", 1, 1024, 5), (16, False, "none", 1000, 1, 12345), (112, True, "parts", 2, 9, 7),
         (80, False, "yarn", 300, 12, 262144)]


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("n,inter,kind,tokens,heads,start", CASES)
def test_rotate(n, inter, kind, tokens, heads, start, transpose):
    torch, K = _k()
    rng = np.random.default_rng(n + tokens)
    r = K.Rotary(128, n, base=500000.0, interleaved=inter, scaling=kind, factor=8.0, original_length=4096)
    f, amp = Q.frequencies(kind, n, 500000.0, 8.0, 4096, 1.0, 32.0 if kind == "yarn" else 4.0)
    x = F.rows(rng, (tokens, heads, 128))
    pos = start + rng.permutation(tokens)
    p = torch.from_numpy(pos.astype(np.int32)).cuda()
    out = r.rotate(to_torch(x), p, torch.empty(tokens, heads, 128, dtype=torch.bfloat16, device="cuda"), transpose)
    F.check_rotation(_np(out), Q.rotate(x, pos, f, amp, inter, transpose), x, amp, n, inter)


@pytest.mark.parametrize("inter", [False, True])
def test_far_and_negative_positions(inter):
    torch, K = _k()
    rng = np.random.default_rng(3)
    pos = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, -123456, 2 ** 30 + 1, 1 << 24])
    x = F.rows(rng, (len(pos), 2, 128))
    r = K.Rotary(interleaved=inter)
    out = r.rotate(to_torch(x), torch.tensor(pos, dtype=torch.int32, device="cuda"))
    # angles of up to 2^31 radians: their 64-bit products are off by 2^-22 of a radian
    f, _ = Q.frequencies("none", 128)
    ref = Q.rotate(x, pos, f, 1.0, inter)
    pair = np.abs(x).max() * 2 * 2.0 ** -21
    F.check_rotation(np.where(np.abs(_np(out) - ref) <= pair, ref, _np(out)), ref, x, 1.0, 128, inter)


@pytest.mark.parametrize("inter", [False, True])
def test_layouts_and_what_lies_between(inter):
    # rows by head, slices of a wider projection, rows that lie apart: the same rows, and nothing else written
    torch, K = _k()
    rng = np.random.default_rng(5)
    x = to_torch(F.rows(rng, (37, 6, 128)))
    pos = torch.from_numpy(rng.integers(0, 100000, 37).astype(np.int32)).cuda()
    r = K.Rotary(128, 96, interleaved=inter)
    want = r.rotate(x, pos, torch.empty_like(x))
    wide = torch.full((37, 11, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    view = wide[:, 2:8, :128]
    view.copy_(x)
    assert r.rotate(view, pos) is view and torch.equal(view, want)
    rest = wide.clone()
    rest[:, 2:8, :128] = 7.0
    assert (rest == 7.0).all()
    by_head = x.transpose(0, 1).contiguous()
    assert torch.equal(r.rotate(by_head.transpose(0, 1), pos), want)
    four = x.view(1, 37, 6, 128)
    assert torch.equal(r.rotate(four, pos, torch.empty_like(four))[0], want)
    one = x[:, :1].expand(37, 6, 128)   # the same row for every head
    assert torch.equal(r.rotate(one, pos, torch.empty_like(x))[:, 3], want[:, 0])
    assert r.rotate(x[:0], pos[:0]).numel() == 0


def test_gradient_against_differences():
    # d/dx of sum(g rotate(x)) by central differences in exact arithmetic of the rounded rotation's definition: the
    # transposed rotation of g
    torch, K = _k()
    rng = np.random.default_rng(6)
    f, amp = Q.frequencies("yarn", 64, 10000.0, 4.0, 4096, 1.0, 32.0)
    r = K.Rotary(128, 64, interleaved=True, scaling="yarn", factor=4.0, original_length=4096)
    x, g = F.rows(rng, (9, 2, 128)), F.rows(rng, (9, 2, 128))
    pos = rng.integers(0, 32768, 9)
    grad = _np(r.rotate(to_torch(g), torch.from_numpy(pos.astype(np.int32)).cuda(), transpose=True))
    for _ in range(40):
        i = (rng.integers(9), rng.integers(2), rng.integers(128))
        d = np.zeros_like(x)
        d[i] = 2.0 ** -10
        diff = (g * (Q.rotate(x + d, pos, f, amp, True) - Q.rotate(x - d, pos, f, amp, True))).sum() / 2.0 ** -9
        assert abs(grad[i] - diff) <= 2.0 ** -8 * abs(diff) + 2 * F.TURN_STEP * amp * np.abs(g[i[:2]]).max() * 2
    # taken out again: two roundings, the first one turned back
    y = r.rotate(to_torch(x), torch.from_numpy(pos.astype(np.int32)).cuda())
    back = _np(K.Rotary(128, 64, interleaved=True, frequencies=r.frequencies, amplitude=1 / r.amplitude).rotate(
        y, torch.from_numpy(pos.astype(np.int32)).cuda(), transpose=True))
    assert np.abs(back - x).max() <= 2.0 ** -7 * 2 * np.abs(x).max()


def test_special_values_stay_in_their_pairs():
    torch, K = _k()
    x = torch.ones(2, 1, 128, dtype=torch.bfloat16, device="cuda")
    x[0, 0, 3], x[1, 0, 100] = math.nan, math.inf
    y = K.Rotary(128, 64).rotate(x, torch.tensor([0, 9], dtype=torch.int32, device="cuda"))
    bad = ~torch.isfinite(y)
    assert bad[0, 0].nonzero().view(-1).tolist() == [3, 35] and bad[1, 0].nonzero().view(-1).tolist() == [100]
    small = torch.full((1, 1, 128), 1e-38, dtype=torch.bfloat16, device="cuda")
    assert (K.Rotary().rotate(small, torch.zeros(1, dtype=torch.int32, device="cuda")) == small).all()


def test_positions_are_read_at_replay_and_on_other_streams():
    torch, K = _k()
    rng = np.random.default_rng(7)
    x = to_torch(F.rows(rng, (5, 8, 128)))
    pos, out, r = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.empty_like(x), K.Rotary()
    r.rotate(x, pos, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.rotate(x, pos, out)
    pos.copy_(torch.tensor([3, 1, 4, 1, 5], dtype=torch.int32))
    want = r.rotate(x, pos, torch.empty_like(x))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = r.rotate(x, pos, torch.empty_like(x), stream=side)
    with torch.cuda.stream(side):
        b = r.rotate(x, pos, torch.empty_like(x))
    side.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)
