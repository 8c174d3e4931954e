"""What automatic differentiation may ask of QHeadNorm: tangents, graphs that are kept, mixed types, derivatives of derivatives."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

import _heads as H
from paper_2104_14129_amd import layers as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def _config():
    before = dict(vars(L.config))
    L.set_optimization_level("L2", bits=8)
    yield
    vars(L.config).update(before)


def _case(dtype=torch.float32):
    g = torch.Generator().manual_seed(5)
    q, k = (torch.randn((30, h, 64), generator=g).to(dtype).to(DEV) for h in (4, 2))
    angle = torch.rand((30, 32), generator=g).to(DEV)
    return q, k, torch.arange(30, dtype=torch.int32, device=DEV), torch.cos(angle), torch.sin(angle)


@pytest.mark.parametrize("of", ["q", "k", "q_weight", "k_weight"])
@pytest.mark.parametrize("mode", ["no_grad", "nothing requires a gradient", "training"])   # inference mode makes no tangents
def test_tangents_are_refused_and_not_dropped(of, mode):
    q, k, *table = _case()
    layer = L.QHeadNorm(64).to(DEV).requires_grad_(mode == "training")
    with torch.set_grad_enabled(mode != "no_grad"), forward_ad.dual_level():
        if of in ("q", "k"):
            q, k = (forward_ad.make_dual(t, torch.ones_like(t)) if of == name else t for name, t in (("q", q), ("k", k)))
            call = lambda: layer(q, k, *table)   # noqa: E731
        else:
            w = {of: forward_ad.make_dual(getattr(layer, of).detach(), torch.ones(64, device=DEV))}
            call = lambda: torch.func.functional_call(layer, w, (q, k, *table))   # noqa: E731
        with pytest.raises((NotImplementedError, RuntimeError), match="forward"):
            call()


def test_without_tangents_a_dual_level_changes_nothing():
    q, k, *table = _case()
    layer = L.QHeadNorm(64).to(DEV)
    with torch.no_grad():
        want = layer(q, k, *table)
        with forward_ad.dual_level():
            got = layer(q, k, *table)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_tangents_of_the_outputs_gradients_are_refused():
    q, k, *table = _case()
    q.requires_grad_()
    y, _ = L.QHeadNorm(64).to(DEV)(q, k, *table)
    with forward_ad.dual_level(), pytest.raises((NotImplementedError, RuntimeError), match="forward"):
        torch.autograd.grad(y, q, forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y)))


def test_a_kept_graph_gives_the_same_gradients_again():
    q, k, *table = _case()
    q.requires_grad_(), k.requires_grad_()
    layer = L.QHeadNorm(64).to(DEV)
    out = layer(q, k, *table)
    wanted = [q, k, layer.q_weight, layer.k_weight]
    first = torch.autograd.grad(out, wanted, [torch.ones_like(t) for t in out], retain_graph=True)
    again = torch.autograd.grad(out, wanted, [torch.ones_like(t) for t in out])
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_under_autocast(dtype):
    """A projection in the narrow type, binary32 weights of the norm: outputs in the narrow type as without gradients, gradients of the parameters' types and within
    5 % of the definition's, as for eight-bit contexts elsewhere."""
    x, _, *table = _case()
    x = x.reshape(30, 256)
    project, layer = torch.nn.Linear(256, 384).to(DEV), L.QHeadNorm(64).to(DEV)
    with torch.autocast("cuda", dtype=dtype):
        z = project(x).view(30, 6, 64)
        q, k = z[:, :4], z[:, 4:]
        out = layer(q, k, *table)
        with torch.no_grad():
            plain = layer(q, k, *table)
        g = [torch.randn(t.shape, generator=torch.Generator().manual_seed(s)).to(dtype).to(DEV) for s, t in enumerate(out)]
        loss = sum((t.float() * r.float()).sum() for t, r in zip(out, g))
    assert all(o.dtype == dtype and torch.equal(o, p) for o, p in zip(out, plain))
    z.retain_grad()
    loss.backward()
    assert project.weight.grad.dtype == torch.float32 and layer.q_weight.grad.dtype == torch.float32
    for x1, r, w, grad in ((q, g[0], layer.q_weight, z.grad[:, :4]), (k, g[1], layer.k_weight, z.grad[:, 4:])):
        want, want_w, _ = H.norm_rotate_backward(r.float().cpu(), x1.detach().float().cpu(), w.detach().cpu(), *(t.cpu() for t in table), 1e-6, False)
        assert float((grad.cpu().double() - want).norm() / want.norm()) < 0.05
        assert float((w.grad.cpu().double() - want_w).norm() / want_w.norm()) < 0.05


@pytest.mark.parametrize("linear", [True, False])
@pytest.mark.parametrize("of", [0, 1, 2, 3])
def test_second_derivatives_are_refused_and_not_taken_for_zeros(of, linear):
    q, k, *table = _case()
    q.requires_grad_(), k.requires_grad_()
    layer = L.QHeadNorm(64).to(DEV)
    inputs = [q, k, layer.q_weight, layer.k_weight]
    loss = sum(t.sum() if linear else t.square().sum() for t in layer(q, k, *table))
    plain = torch.autograd.grad(loss, inputs, retain_graph=True)
    graph = torch.autograd.grad(loss, inputs, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(plain, graph))
    again = graph[of].square().sum() + q.sum()
    with pytest.raises(NotImplementedError, match="second derivative"):
        torch.autograd.grad(again, layer.k_weight, retain_graph=True)
    with pytest.raises(NotImplementedError, match="second derivative"):
        again.backward()
