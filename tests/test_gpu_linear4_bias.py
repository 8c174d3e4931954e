"""The gradient of the bias behind a product with 4-bit weights, and a layer's training step captured into a graph."""
import pytest
import torch
import torch.nn as nn

import _layer as Y
from paper_2104_14129_amd import binding as B
from paper_2104_14129_amd import layers as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("rows, outputs", [(1, 1), (3, 7), (16, 512), (17, 513), (63, 1000), (5000, 70), (4097, 2000), (200, 5001), (70000, 9), (33, 300000)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("wide", [True, False])
def test_sums(rows, outputs, dtype, wide):
    """Three roundings of four numbers' sum, one of a part, one of the result in binary32, one of it to its type; a part is at most the sum of the magnitudes."""
    grad = torch.randn((rows, outputs), generator=torch.Generator().manual_seed(rows)).to(dtype).to(DEV)
    to = F32 if wide else dtype
    got = B.linear4_backward_bias(grad, to)
    want, size = grad.double().sum(0), grad.double().abs().sum(0)
    assert got.dtype == to and got.shape == (outputs,)
    assert bool(((got.double() - want).abs() <= torch.finfo(to).eps / 2 * want.abs() + 5 * Y.UNIT * size + 2.0 ** -25).all())
    odd = torch.full((rows, outputs + 5), 9.0, dtype=dtype, device=DEV)
    odd[:, 3:3 + outputs] = grad
    assert torch.equal(B.linear4_backward_bias(odd[:, 3:3 + outputs], to), got)
    assert torch.equal(B.linear4_backward_bias(grad.view(1, rows, outputs), to), got)


def test_no_rows_rows_that_share_memory_and_refusals():
    assert (B.linear4_backward_bias(torch.zeros((0, 40), device=DEV), F32) == 0).all()
    row = torch.arange(40.0, device=DEV)
    assert torch.equal(B.linear4_backward_bias(row.expand(300, 40), F32), 300 * row)
    bad = torch.zeros((50, 40), device=DEV)
    bad[7, 3], bad[9, 5] = float("nan"), float("inf")
    got = torch.isfinite(B.linear4_backward_bias(bad, F32))
    assert not got[3] and not got[5] and int(got.sum()) == 38
    for args, error in (((bad.double(), F32), TypeError), ((bad, F16), TypeError), ((bad.half(), BF16), TypeError), ((bad, "f32"), TypeError), ((bad.t(), F32), ValueError),
                        ((bad.cpu(), F32), ValueError)):
        with pytest.raises(error):
            B.linear4_backward_bias(*args)
    with pytest.raises(B.ActqError, match="outputs"):
        B.linear4_backward_bias(torch.zeros((3, 0), device=DEV), F32)


@pytest.mark.parametrize("rows, inputs, outputs", [(4096, 256, 2000), (33, 512, 300), (20000, 128, 70)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_a_training_step_captured_and_replayed(rows, inputs, outputs, dtype):
    """A norm without a context that is drawn anew, a product and a bias: replays give what eager steps do, with eager work and synchronizations between."""
    torch.manual_seed(3)
    norm = L.QBlockNorm(inputs, gate=True, dtype=dtype).to(DEV)
    layer = L.Linear4.from_linear(nn.Linear(inputs, outputs).to(DEV, dtype), 64)
    x, h, grad = (torch.zeros((rows, n), dtype=dtype, device=DEV) for n in (inputs, inputs, outputs))
    x.requires_grad_()
    h.requires_grad_()
    wanted = (x, h, *norm.parameters(), layer.bias)
    kept, L._DTYPES = L._DTYPES, ()   # contexts as they are
    try:
        def step():
            return torch.autograd.grad(layer(norm(x, h)[1]), wanted, grad)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.Generator().manual_seed(8)
        for i in range(4):
            with torch.no_grad():
                for t in (x, h, grad):
                    t.copy_(torch.randn(t.shape, generator=g).to(dtype))
            graph.replay()
            torch.cuda.synchronize()
            want = step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), (i, [torch.equal(a, b) for a, b in zip(out, want)])
    finally:
        L._DTYPES = kept
