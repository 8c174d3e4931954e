"""A layer's operators at sizes whose elements, eight or a row of them a thread or workgroup, need 2^32 threads and more."""
import pytest
import torch

import _layer as Y
from paper_2104_14129_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def _memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("tokens, width", [((1 << 22) + 3, 8193), ((1 << 24) + 2, 2050)])
def test_block_norm(tokens, width):
    """Every row is the same one but for the last two."""
    x = torch.randn((1, width), generator=torch.Generator().manual_seed(1)).to(BF16).to(DEV)
    w = torch.randn(width, generator=torch.Generator().manual_seed(2)).to(BF16).to(DEV)
    _, want = B.block_norm(x, None, None, w)
    y = torch.empty((tokens, width), dtype=BF16, device=DEV)
    B.block_norm(x.expand(tokens, width), None, None, w, y=y)
    for rows in y.split(1 << 20):
        assert bool((rows.view(torch.int16) == want.view(torch.int16)).all())
    y[-2:] = 1.0
    y[-1, 0] = 3.0
    last = B.block_norm(y[-2:].clone(), None, None, w)[1]
    B.block_norm(y, None, None, w, y=y)
    assert torch.equal(y[-2:], last)


def test_weights():
    """2^35 weights and more; every output is the same one."""
    outputs, inputs = (1 << 15) + 1, 1 << 20
    w = torch.randn((1, inputs), generator=torch.Generator().manual_seed(1)).to(BF16).to(DEV)
    one = B.quantize_weights(w, 128)
    codes, header = B.quantize_weights(w.expand(outputs, inputs), 128)
    assert all(bool((rows == one[0]).all()) for rows in codes.split(4096)) and bool((header == one[1]).all())
    value = B.dequantize_weights(*one, inputs, BF16)
    for rows in B.dequantize_weights(codes, header, inputs, BF16).split(2048):
        assert bool((rows == value).all())


def test_rows_of_a_product():
    rows, inputs, outputs = (1 << 15) + 1, 1 << 20, 20
    codes, header = (t.to(DEV) for t in Y.random_weights(outputs, inputs, 128, 4))
    x = torch.randn((1, inputs), generator=torch.Generator().manual_seed(1)).to(BF16).to(DEV)
    y = B.linear4(x.expand(rows, inputs), codes, header)
    assert torch.equal(y, y[:1].expand(rows, outputs))
    w, _ = Y.weights(codes.cpu(), header.cpu(), inputs)
    want = x.cpu().double() @ w.t()
    assert float((y[:1].cpu().double() - want).norm() / want.norm()) <= 2.0 ** -8
