"""Every kernel of the products with 4-bit weights, in every type and group: values, rows that lie inside wider matrices at any element, and what lies beside the results."""
import pytest
import torch

import _layer as Y
import test_gpu_linear4 as L
from paper_2104_14129_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [pytest.param(t, id=str(t)[6:]) for t in (F32, F16, BF16)]


def _inside(rows, columns, dtype, seed, before):
    """A matrix inside a wider one whose rows start at any element."""
    wide = L._rows(rows, columns + 13, dtype, seed).to(DEV)
    return wide[:, before:before + columns]


def _within(off, limit):
    assert bool((off <= limit).all()), float((off / limit).max())


# rows, inputs, outputs: few rows; few rows of many outputs; few or tiles of 32 rows; these in several parts; tiles of 128 rows in one part, the last of them cut, and in several; tiles of 32 rows in
# one part (binary32: of 128)
@pytest.mark.parametrize("rows, inputs, outputs", [(5, 1000, 300), (13, 600, 8201), (40, 600, 5003), (33, 4200, 1030), (1029, 1152, 4099), (1030, 1100, 4099), (1030, 8320, 600), (1025, 8300, 777), (100, 500, 20000)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", TYPES)
def test_products(rows, inputs, outputs, group, dtype):
    codes, header = Y.random_weights(outputs, inputs, group, rows)
    x = _inside(rows, inputs, dtype, 5, 3)
    aligned = x.contiguous()
    weights = codes.to(DEV), header.to(DEV)
    bias = torch.randn(outputs, generator=torch.Generator().manual_seed(3)).to(DEV)
    got = B.linear4(aligned, *weights, bias)
    w, step = (t.to(DEV) for t in Y.weights(codes, header, inputs))
    zero = header[..., :1].double().abs().expand(-1, -1, group).flatten(1)[:, :inputs].to(DEV)
    want = aligned.double() @ w.t().contiguous() + bias.double()
    _within((got.double() - want).abs(), L._forward_bound(aligned, step, zero, group, want, dtype))
    assert torch.equal(B.linear4(x, *weights, bias), got)
    out = torch.full((rows + 1, outputs + 29), 7.0, dtype=dtype, device=DEV)
    B.linear4(x, *weights, bias, out=out[:rows, 11:11 + outputs])
    assert torch.equal(out[:rows, 11:11 + outputs], got)
    assert (out[:, :11] == 7).all() and (out[:, 11 + outputs:] == 7).all() and (out[rows] == 7).all()
    backwards = torch.flip(aligned, (0,))
    assert torch.equal(B.linear4(backwards, *weights, bias).flip(0), got)
    assert torch.equal(B.linear4(aligned[:1].expand(rows, inputs), *weights, bias), got[:1].expand(rows, outputs))


# rows, inputs, outputs: few rows in one part of the outputs and several; from weights in memory in one part and several
@pytest.mark.parametrize("rows, inputs, outputs", [(70, 3000, 200), (9, 500, 3001), (1031, 5003, 1999), (2049, 1000, 4400)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients(rows, inputs, outputs, group, dtype):
    """Off by what the formats of the parts leave, a quarter at most of what the test of the gradients beside the products allows for weights of 11 bits, and by binary32 sums."""
    codes, header = Y.random_weights(outputs, inputs, group, rows)
    grad = _inside(rows, outputs, dtype, 5, 5)
    aligned = grad.contiguous()
    weights = codes.to(DEV), header.to(DEV)
    got = B.linear4_backward(aligned, *weights, inputs)
    w = Y.weights(codes, header, inputs)[0].to(DEV)
    middle = (header[..., :1].double().abs() + 8 * header[..., 1:].double().abs()).expand(-1, -1, group).flatten(1)[:, :inputs].to(DEV)
    want = aligned.double() @ w
    e = ((aligned.double() ** 2) @ (w ** 2 + middle ** 2)) ** 0.5
    unit = torch.finfo(dtype).eps / 2
    limit = unit * want.abs() + (8 * {F32: 2.0 ** -21, F16: 2.0 ** -15, BF16: 2.0 ** -15}[dtype] + 32 * Y.UNIT * (3 * outputs) ** 0.5) * e + 2.0 ** -25
    _within((got.double() - want).abs(), limit)
    assert torch.equal(B.linear4_backward(grad, *weights, inputs), got)
    assert torch.equal(B.linear4_backward(aligned.flip(0), *weights, inputs).flip(0), got)
    assert torch.equal(B.linear4_backward(aligned[:1].expand(rows, outputs), *weights, inputs), got[:1].expand(rows, inputs))
