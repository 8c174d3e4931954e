"""The norms around a block and the linear layer with 4-bit weights as modules, and a layer that trains and answers with them."""
import pytest
import torch
import torch.nn as nn
from torch.autograd import forward_ad

import _layer as Y
from paper_2104_14129_amd import binding as B
from paper_2104_14129_amd import layers as L
from paper_2104_14129_amd.cache import PagedCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def _config():
    before = dict(vars(L.config))
    yield
    vars(L.config).update(before)


def _randn(*shape, seed, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("level", ["L2", "L4"])
@pytest.mark.parametrize("gate", ["none", "learned", "token"])
def test_block_norm_gradients_at_eight_bits(dtype, level, gate):
    """The outputs are those without training.  At eight bits an element of a context is off by at most a 255th of its group's range, 8 here; gradients are
    smooth on that scale, and their errors below 5 % of their size (bfloat16 contexts are exact)."""
    L.set_optimization_level(level, bits=8)
    L.config.mixed = False
    layer = L.QBlockNorm(96, gate=gate == "learned", scale=0.5, dtype=dtype).to(DEV)
    with torch.no_grad():
        layer.weight.mul_(1.5)
        if layer.gate is not None:
            layer.gate.mul_(0.7)
    shape = (3, 17, 96)
    x, h, g, gr, gy = (_randn(*shape, seed=s, dtype=dtype) for s in range(5))
    inputs = [t.to(DEV).requires_grad_() for t in ((x, h, g) if gate == "token" else (x, h))]
    with torch.no_grad():
        plain = layer(*inputs)
    out = layer(*inputs)
    assert torch.equal(out[0], plain[0]) and torch.equal(out[1], plain[1]) and out[0].shape == shape
    (out[0].float() * gr.to(DEV).float()).sum().add((out[1].float() * gy.to(DEV).float()).sum()).backward()
    flat = [t.view(-1, 96) for t in (x, h, g, gr, gy)]
    used = {"none": None, "learned": torch.full((96,), 0.7).to(dtype), "token": flat[2]}[gate]
    r, _, _ = Y.block_norm(flat[0], flat[1], used, torch.full((96,), 1.5), torch.ones(96), 0.5, 1e-6)
    want = Y.block_norm_backward(flat[3], flat[4], r, flat[1], used, torch.full((96,), 1.5), torch.ones(96), 0.5, 1e-6)
    got = {"x": inputs[0].grad, "h": inputs[1].grad, "weight": layer.weight.grad, "post": layer.post_weight.grad}
    if gate != "none":
        got["gate"] = inputs[2].grad if gate == "token" else layer.gate.grad
    assert set(got) == set(want)
    for name, (value, _) in want.items():
        assert got[name].dtype == dtype
        assert float((got[name].cpu().double().view(value.shape) - value).norm() / value.norm()) < 0.05, name


def test_block_norm_alone_frozen_and_with_one_gradient():
    layer = L.QBlockNorm(64, post=False).to(DEV)
    x, h = _randn(5, 64, seed=1).to(DEV).requires_grad_(), _randn(5, 64, seed=2).to(DEV)
    r, y = layer(x)
    assert r.data_ptr() == x.data_ptr()
    y.sum().backward()
    assert x.grad.shape == x.shape and layer.weight.grad is not None
    x.grad = None
    layer.requires_grad_(False)
    r, y = layer(x, h)
    r.sum().backward()   # y has none: an expanded gradient of r alone
    assert torch.equal(x.grad, torch.ones_like(x))
    with torch.no_grad():
        none = layer(x[:0], h[:0])
    assert none[1].shape == (0, 64)
    with pytest.raises(ValueError, match="gate"):
        layer(x, None, h)
    with pytest.raises(ValueError, match="gate"):
        L.QBlockNorm(64, gate=True).to(DEV)(x, h, h)


@pytest.mark.parametrize("make", [lambda: L.QBlockNorm(64).to(DEV), lambda: L.Linear4.from_linear(nn.Linear(64, 64).to(DEV), 32)])
def test_tangents_and_second_derivatives_are_refused(make):
    layer = make()
    run = (lambda x: layer(x, x)[1]) if isinstance(layer, L.QBlockNorm) else layer
    x = _randn(4, 64, seed=1).to(DEV).requires_grad_()
    (g,) = torch.autograd.grad(run(x).square().sum(), x, create_graph=True)
    with pytest.raises(NotImplementedError, match="second derivative"):
        g.sum().backward()
    with torch.no_grad(), forward_ad.dual_level():
        dual = forward_ad.make_dual(x.detach(), torch.ones_like(x))
        with pytest.raises(NotImplementedError, match="forward-mode"):
            run(dual)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bias", [True, False])
def test_linear4_module(dtype, bias):
    """Outputs and gradients are those of a linear layer with the weights that the codes stand for, off by roundings: of the result, and of a weight to 11 bits
    at least in the gradient; binary32 sums over at most 200 numbers."""
    torch.manual_seed(3)
    linear = nn.Linear(200, 77, bias=bias).to(DEV, dtype)
    layer = L.Linear4.from_linear(linear, 64)
    layer.half()   # the format of the weights is not a module's type
    if bias:
        layer.bias.data = linear.bias.detach().clone()
    w = layer.weight().double()
    x = _randn(2, 9, 200, seed=4, dtype=dtype).to(DEV).requires_grad_()
    y = layer(x)
    want = x.detach().double() @ w.t() + (linear.bias.double() if bias else 0)
    unit = torch.finfo(dtype).eps / 2
    limit = unit * want.abs() + 200 * 2.0 ** -24 * (x.detach().double().abs() @ w.abs().t() + 1) * 40
    assert y.dtype == dtype and ((y.detach().double() - want).abs() <= limit).all()
    g = _randn(2, 9, 77, seed=5, dtype=dtype).to(DEV)
    y.backward(g)
    want = g.double() @ w
    limit = unit * want.abs() + (2.0 ** -11 + 200 * 2.0 ** -24) * (g.double().abs() @ w.abs())
    assert x.grad.shape == x.shape and ((x.grad.double() - want).abs() <= limit).all()
    if bias:
        want = g.double().sum((0, 1))
        assert ((layer.bias.grad.double() - want).abs() <= unit * want.abs() + 18 * 2.0 ** -24 * g.double().abs().sum((0, 1))).all()
    again = L.Linear4(torch.zeros_like(layer.codes), torch.zeros_like(layer.header).view(torch.bfloat16), 200, layer.bias.detach().clone() if bias else None)
    again.load_state_dict(layer.state_dict())
    with torch.no_grad():
        assert torch.equal(again(x), y)


class _Layer(nn.Module):
    """Norm, projections with 4-bit weights, head norm, attention, norm behind it, a gated block."""

    def __init__(self, width, heads, kv_heads, dim, dtype):
        super().__init__()
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        four = lambda a, b: L.Linear4.from_linear(nn.Linear(a, b, bias=False).to(DEV, dtype), 64)   # noqa: E731
        self.first, self.middle, self.last = (L.QBlockNorm(width, gate=g, scale=0.8, dtype=dtype).to(DEV) for g in (False, True, False))
        self.project, self.back = four(width, (heads + 2 * kv_heads) * dim), four(heads * dim, width)
        self.up, self.down = four(width, 2 * width), four(2 * width, width)
        self.norm = L.QHeadNorm(dim, dtype=dtype).to(DEV)

    def split(self, x):
        return self.project(x).view(len(x), -1, self.dim).split((self.heads, self.kv_heads, self.kv_heads), 1)

    def rest(self, x, out):
        x, y = self.middle(x, self.back(out.reshape(len(x), -1)))
        return self.last(x, self.down(torch.nn.functional.silu(self.up(y))))[1]

    def whole(self, x, positions, cos, sin):
        q, k, v = self.split(self.first(x)[1])
        q, k = self.norm(q, k, positions, cos, sin)
        k, v = (t.repeat_interleave(self.heads // self.kv_heads, 1) for t in (k, v))
        scores = torch.matmul(q.transpose(0, 1).float(), k.permute(1, 2, 0).float().contiguous()) * self.dim ** -0.5
        p = scores.masked_fill(torch.ones(scores.shape[-2:], dtype=torch.bool, device=x.device).triu(1), float("-inf")).softmax(-1)
        return self.rest(x, torch.matmul(p, v.transpose(0, 1).float().contiguous()).transpose(0, 1).to(x.dtype))

    def answer(self, x, positions, cos, sin, cache, slots, *where):
        q, k, v = self.split(self.first(x)[1])
        q = cache.append(q, k, v, self.norm.q_weight, self.norm.k_weight, positions, cos, sin, slots)
        return self.rest(x, cache.attend(q, *where))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_a_layer_answers_from_its_cache_as_it_computes_a_whole_sequence(dtype):
    """Keys and values of 8 bits are off by up to half a 255th of their groups' range (about 1 % of their size), attention averages that, and what follows
    scales it with the attention's output: below 3 % of the result, with 16-bit roundings along the way."""
    torch.manual_seed(1)
    layer = _Layer(256, 8, 2, 64, dtype)
    lengths, total = (70, 33), 103
    angle = torch.rand((128, 32), generator=torch.Generator().manual_seed(2)).to(DEV) * 6.3
    tables = torch.cos(angle), torch.sin(angle)
    sequences = [_randn(n, 256, seed=n, dtype=dtype).to(DEV) for n in lengths]
    cache = PagedCache(16, 16, 2, 64, device=DEV)
    table = torch.randperm(16, generator=torch.Generator().manual_seed(3))[:10].view(2, 5).int().to(DEV)
    done, outputs = [0, 0], [[], []]
    with torch.no_grad():
        for chunk in (50, 1, 1, 17, 1, 200):   # a chunk of the prompts, single tokens, the rest
            new = [min(chunk, n - d) for n, d in zip(lengths, done)]
            sequence = torch.tensor([s for s, n in enumerate(new) for _ in range(n)], device=DEV)
            position = torch.tensor([d + i for d, n in zip(done, new) for i in range(n)], device=DEV)
            rows = torch.cat([s[d:d + n] for s, d, n in zip(sequences, done, new)])
            done = [d + n for d, n in zip(done, new)]
            start = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device=DEV)
            if not sum(new):
                continue
            y = layer.answer(rows, position.int(), *tables, cache, cache.slots(table, sequence, position), table, torch.tensor(done, dtype=torch.int32, device=DEV), start,
                             max(new), max(done))
            for s, part in enumerate(y.split(new)):
                outputs[s].append(part)
        assert sum(done) == total
        for s, x in enumerate(sequences):
            want = layer.whole(x, torch.arange(len(x), dtype=torch.int32, device=DEV), *tables)
            got = torch.cat(outputs[s])
            assert float((got.float() - want.float()).norm() / want.float().norm()) < 0.03


def test_a_layer_trains_its_norms_over_frozen_weights():
    """Gradients reach the input and every parameter; with contexts of 8 bits they are those of exact contexts (bits kept as they are) to 10 % of their size."""
    L.set_optimization_level("L2", bits=8)
    torch.manual_seed(1)
    layer = _Layer(256, 4, 2, 64, torch.float32)
    angle = torch.rand((128, 32), generator=torch.Generator().manual_seed(2)).to(DEV) * 6.3
    args = torch.arange(90, dtype=torch.int32, device=DEV), torch.cos(angle), torch.sin(angle)
    x = _randn(90, 256, seed=7).to(DEV).requires_grad_()
    target = _randn(90, 256, seed=8).to(DEV)

    def gradients():
        names, tensors = zip(("input", x), *layer.named_parameters())
        unused = {"first.post_weight"}   # the first norm has no block behind it
        wanted = [t for n, t in zip(names, tensors) if n not in unused]
        return dict(zip([n for n in names if n not in unused], torch.autograd.grad((layer.whole(x, *args) - target).square().mean(), wanted)))

    got = gradients()
    before, L._DTYPES = L._DTYPES, ()
    try:
        want = gradients()
    finally:
        L._DTYPES = before
    assert len(got) > 6
    for name, value in want.items():
        assert torch.isfinite(got[name]).all() and float((got[name] - value).norm() / value.norm()) < 0.1, name
    assert B.version() >= 400
