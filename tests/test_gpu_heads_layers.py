"""The head norm as a layer with compressed contexts, the cache as an object, and the example that runs them together."""
import os
import sys

import pytest
import torch

import _heads as H
from paper_2104_14129_amd import layers as L
from paper_2104_14129_amd.cache import PagedCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(autouse=True)
def _config():
    before = dict(vars(L.config))
    yield
    vars(L.config).update(before)


def _case(dtype, tokens=50, q_heads=4, k_heads=2, dim=64):
    g = torch.Generator().manual_seed(3)
    q, k = (torch.randn((tokens, h, dim), generator=g).to(dtype) for h in (q_heads, k_heads))
    angle = torch.rand((tokens, dim // 2), generator=g)
    return q, k, torch.arange(tokens, dtype=torch.int32), torch.cos(angle), torch.sin(angle)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("level", ["L2", "L4"])
def test_layer_gradients_at_eight_bits(dtype, level):
    """The outputs are those without training.  At eight bits an element of the context is off by at most a 255th of its group's
    range, 8 here; a gradient is smooth in x on that scale, and its error is below 5 % of its size (bfloat16 contexts are exact)."""
    L.set_optimization_level(level, bits=8)
    L.config.mixed = False
    q, k, positions, cos, sin = _case(dtype)
    table = positions.to(DEV), cos.to(DEV), sin.to(DEV)
    layer = L.QHeadNorm(64).to(DEV)
    with torch.no_grad():
        layer.q_weight.mul_(1.5)
        plain = layer(q.to(DEV), k.to(DEV), *table)
    dq, dk = q.to(DEV).requires_grad_(), k.to(DEV).requires_grad_()
    out = layer(dq, dk, *table)
    assert torch.equal(out[0], plain[0]) and torch.equal(out[1], plain[1])
    gq, gk = (torch.randn(t.shape, generator=torch.Generator().manual_seed(s)).to(dtype) for s, t in ((1, q), (2, k)))
    (out[0].float() * gq.to(DEV).float()).sum().add((out[1].float() * gk.to(DEV).float()).sum()).backward()
    for x, g, w, dx, dw in ((q, gq, 1.5, dq.grad, layer.q_weight.grad), (k, gk, 1.0, dk.grad, layer.k_weight.grad)):
        want_x, want_w, _ = H.norm_rotate_backward(g, x, torch.full((64,), w), positions, cos, sin, 1e-6, False)
        assert dx.dtype == dtype and float((dx.cpu().double() - want_x).norm() / want_x.norm()) < 0.05
        assert float((dw.cpu().double() - want_w).norm() / want_w.norm()) < 0.05


def test_layer_without_gradients_of_weights_and_with_an_expanded_gradient():
    q, k, positions, cos, sin = _case(torch.float32)
    layer = L.QHeadNorm(64).to(DEV).requires_grad_(False)
    dq = q.to(DEV).requires_grad_()
    out, _ = layer(dq, k.to(DEV), positions.to(DEV), cos.to(DEV), sin.to(DEV))
    out.sum().backward()
    assert dq.grad.shape == q.shape and layer.q_weight.grad is None


def test_layer_of_no_tokens():
    q, k, positions, cos, sin = _case(torch.float16)
    layer = L.QHeadNorm(64, dtype=torch.float16).to(DEV)
    out = layer(q[:0].to(DEV).requires_grad_(), k[:0].to(DEV), positions[:0].to(DEV), cos.to(DEV), sin.to(DEV))
    (out[0].sum() + out[1].sum()).backward()
    assert (layer.q_weight.grad == 0).all()


@pytest.mark.parametrize("key_bits, value_bits", [(8, 8), (8, 4)])
def test_cache_object(key_bits, value_bits):
    """What is read back is the written value to within half a step of its group's range (5 to 8 here for 64 normal numbers), and the binary16 rounding."""
    cache = PagedCache(8, 16, 2, 64, key_bits, value_bits, device=DEV)
    assert cache.nbytes() == 8 * 2 * 16 * (8 * (key_bits + value_bits) + 16)
    k, v = (torch.randn((20, 2, 64), generator=torch.Generator().manual_seed(s)).half().to(DEV) for s in (1, 2))
    table = torch.tensor([[5, 2]], dtype=torch.int32, device=DEV)
    position = torch.arange(20, device=DEV)
    slots = cache.slots(table, torch.zeros_like(position), position)
    assert slots.tolist() == [5 * 16 + i for i in range(16)] + [2 * 16 + i for i in range(4)]
    cache.write(k, v, slots)
    for x, y, bits in zip((k, v), cache.read(slots, torch.float16), (key_bits, value_bits)):
        extent = (x.amax(-1, keepdim=True) - x.amin(-1, keepdim=True)).float()
        assert ((x.float() - y.float()).abs() <= 0.501 * extent / (2 ** bits - 1) + 2.0 ** -9).all()


def test_the_example():
    """Training lowers the loss; answers from a cache of 8 bits differ by what rounding keys and values to a 255th of their range does."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import cached_attention
    finally:
        sys.path.pop(0)
    result = cached_attention.main(steps=5)
    assert result["losses"][-1] < result["losses"][0] and result["off"] < 0.02
