"""How exact the sums of products with 4-bit weights are before they are rounded to 16 bits."""
import pytest
import torch

import _heads as H
import _layer as Y
from paper_2104_14129_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16


def _weights(codes, header, inputs):
    """[outputs, inputs] in 64 bits on the GPU, and the largest of 16 + code in their place."""
    group = codes.shape[1] * 8 // header.shape[1]
    at = torch.tensor(Y.SHIFTS, device=DEV)
    code = (codes.long()[..., None] >> at & 15).view(*header.shape[:2], group).double()
    zero, step = header.double()[..., :1], header.double()[..., 1:]
    return [t.flatten(1)[:, :inputs].contiguous() for t in (code * step + zero, (16 + code) * step.abs())]


# rows, inputs, outputs, group: few rows, few rows of many outputs, tiles of 32 rows in one part and several, tiles of 128 rows likewise
@pytest.mark.parametrize("rows, inputs, outputs, group", [
    (16, 4096, 1024, 128), (16, 8192, 8192, 64), (64, 8192, 2048, 32), (500, 1024, 5120, 128), (1024, 8192, 2048, 128), (1024, 8192, 2048, 64), (1024, 8192, 2048, 32), (4096, 8192, 4096, 128)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_sums_are_as_good_as_binary32_ones(rows, inputs, outputs, group, dtype):
    """A sum that is off by d before its last rounding is rounded the other way with a probability of |d| in the distance of two numbers, at most 2 u |y|, and is off by
    that distance then: the mean square of what differs from the exact sum, rounded, is at most 2 u |d| |y|.  d: of a group there is a rounding where its sum
    of products comes in, one where its plain sum does, and eight or fewer of smaller sums inside; each is half a unit of a partial sum at most, and of
    either sign.  A partial sum is at most as large as the root of the sum of squares of x step (16 + code)."""
    codes, header = (t.to(DEV) for t in Y.random_weights(outputs, inputs, group, 1))
    x = torch.randn((rows, inputs), generator=torch.Generator().manual_seed(2)).to(dtype).to(DEV)
    w, shifted = _weights(codes, header, inputs)
    y = x.double() @ w.t().contiguous()
    partial = ((x.double() ** 2) @ (shifted ** 2).t().contiguous()) ** 0.5
    got = B.linear4(x, codes, header).double()
    d = Y.UNIT * (3 * inputs / group / 3) ** 0.5 * partial
    limit = float((2 * H.ROUNDOFF[dtype] * d * y.abs()).sum()) ** 0.5
    off = float((got - y.to(dtype).double()).norm())
    assert off <= limit, (off / limit, off / float(y.norm()))


# rows, inputs, outputs, group: more than 2^33 products, from weights in memory, whole tiles and cut ones, one part of the outputs and several
@pytest.mark.parametrize("rows, inputs, outputs, group", [(2048, 4096, 8192, 128), (1100, 4224, 2100, 32), (1500, 3001, 2100, 64), (9000, 2048, 1000, 128)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_gradients_from_weights_in_memory_are_as_good_as_binary32_ones(rows, inputs, outputs, group, dtype):
    """As above.  d: weights are exact but for the middles of their groups (22 bits, below the rest), sixteen products come in at a time, with two roundings at most; a
    partial sum is at most as large as the root of the sum of squares of grad_y times what a weight is made of, step (code - 8) and zero + 8 step."""
    codes, header = (t.to(DEV) for t in Y.random_weights(outputs, inputs, group, 1))
    grad = torch.randn((rows, outputs), generator=torch.Generator().manual_seed(2)).to(dtype).to(DEV)
    w, _ = _weights(codes, header, inputs)
    middle = (header[..., :1].double() + 8 * header[..., 1:].double()).expand(-1, -1, group).flatten(1)[:, :inputs]
    y = grad.double() @ w
    partial = ((grad.double() ** 2) @ ((w - middle) ** 2 + middle ** 2)) ** 0.5
    got = B.linear4_backward(grad, codes, header, inputs).double()
    d = Y.UNIT * (outputs / 8 / 3) ** 0.5 * partial
    limit = float((2 * H.ROUNDOFF[dtype] * d * y.abs()).sum()) ** 0.5
    off = float((got - y.to(dtype).double()).norm())
    assert off <= limit, (off / limit, off / float(y.norm()))
