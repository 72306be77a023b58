"""Calls of the rotation with tensors that autograd knows of, or that lie in pinned memory."""

import os

import numpy as np
import pytest

from tests import cache4 as F
from tests.cache8 import to_torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_30738_gb300", "libkvevict.so")


def _k(gpu=False):
    torch = pytest.importorskip("torch")
    if gpu and not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    if not os.path.exists(LIB):
        pytest.skip("library not built")
    from paper_2609_30738_gb300 import kv_evict as K
    return torch, K


def test_a_gradient_that_would_be_lost_is_refused():
    torch, K = _k()
    x = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    grad = x.clone().requires_grad_()
    p, r = torch.zeros(4, dtype=torch.int32), K.Rotary()
    for a in (dict(x=grad), dict(x=grad, out=x), dict(x=x, out=grad), dict(x=grad * 2.0)):
        with pytest.raises(ValueError, match="no gradient"):
            r.rotate(positions=p, **a)
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA device"):
        r.rotate(grad, p)


@pytest.mark.gpu
def test_gradients_through_a_function_of_the_callers():
    torch, K = _k(True)
    rng = np.random.default_rng(1)
    r = K.Rotary(128, 64, interleaved=True)

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, pos):
            ctx.save_for_backward(pos)
            return r.rotate(x, pos, torch.empty_like(x))

        @staticmethod
        def backward(ctx, g):
            return r.rotate(g, ctx.saved_tensors[0], torch.empty_like(g), transpose=True), None

    x, g = (to_torch(F.rows(rng, (5, 8, 128))) for _ in range(2))
    pos = torch.tensor([3, 1, 4, 1, 5], dtype=torch.int32, device="cuda")
    leaf = x.clone().requires_grad_()
    Turn.apply(leaf, pos).backward(g)
    assert torch.equal(leaf.grad, r.rotate(g, pos, torch.empty_like(g), transpose=True))
    for a in (dict(x=leaf), dict(x=leaf * 1.0), dict(x=x, out=leaf)):
        with pytest.raises(ValueError, match="no gradient"):
            r.rotate(positions=pos, **a)
    assert torch.equal(leaf, x)
    with torch.no_grad():
        want = r.rotate(leaf, pos, torch.empty_like(x))
    for Cache in (K.Cache8, K.Cache4):
        cache = Cache(dict(num_layers=1, num_q_heads=8, num_kv_heads=2, head_dim=128), max_seqs=1, num_pages=2, max_pages=1,
                      page_tokens=16)
        k = x[:, :2].contiguous()
        slots = torch.arange(5, dtype=torch.int32, device="cuda")
        for a in (dict(q=leaf), dict(q=leaf, q_out=torch.empty_like(x)), dict(q=x, q_out=leaf)):
            with pytest.raises(ValueError, match="no gradient"):
                cache.append(r, pos, k, k, slots, **a)
        assert torch.equal(leaf, x)
        with torch.no_grad():
            assert torch.equal(cache.append(r, pos, k, k, slots, q=leaf, q_out=torch.empty_like(x)), want)
        assert cache.status() == K.KVE_OK


@pytest.mark.gpu
def test_what_is_read_may_lie_in_pinned_memory():
    # as in append: what is turned and the positions, but not what is written
    torch, K = _k(True)
    rng = np.random.default_rng(2)
    r = K.Rotary(interleaved=True)
    x = to_torch(F.rows(rng, (37, 8, 128)))
    pos = torch.from_numpy(rng.integers(0, 100000, 37).astype(np.int32)).cuda()
    want = r.rotate(x, pos, torch.empty_like(x))
    near, at = x.cpu().pin_memory(), pos.cpu().pin_memory()
    for a, p in ((x, at), (near, pos), (near, at)):
        assert torch.equal(r.rotate(a, p, torch.empty_like(x)), want)
    for bad in ((near, pos), (x, pos, near), (x.cpu(), pos, torch.empty_like(x)), (x, pos.cpu())):
        with pytest.raises(ValueError, match="CUDA device"):
            r.rotate(*bad)
    assert torch.equal(near, x.cpu())
    k = x[:, :2].contiguous()
    slots = torch.arange(37, dtype=torch.int32, device="cuda")
    for Cache in (K.Cache8, K.Cache4):
        made = []
        for p in (pos, at):
            cache = Cache(dict(num_layers=1, num_q_heads=8, num_kv_heads=2, head_dim=128), max_seqs=1, num_pages=3, max_pages=3,
                          page_tokens=16)
            cache.k.zero_()
            q = cache.append(r, p, k, k, slots, q=x if p is pos else near, q_out=torch.empty_like(x))
            assert torch.equal(q, want) and cache.status() == K.KVE_OK
            made.append(cache.k)
        assert torch.equal(*made)
