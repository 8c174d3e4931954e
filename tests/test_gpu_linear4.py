"""Products with 4-bit weights, the gradient of their rows and the quantizer, against their definitions in 64 bits."""
import pytest
import torch

import _heads as H
import _layer as Y
from paper_2104_14129_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16

# rows, inputs, outputs, group, dtype
CASES = [
    (1, 1, 1, 32, F32), (1, 31, 2, 32, F16), (1, 33, 17, 32, BF16), (2, 64, 64, 64, BF16), (1, 128, 100, 128, F16), (3, 100, 15, 64, F32), (16, 129, 33, 128, BF16),
    (17, 1000, 77, 32, F16), (5, 999, 130, 64, BF16), (31, 511, 48, 128, F32), (33, 640, 65, 64, F16), (64, 2048, 127, 128, BF16), (65, 1025, 129, 32, F32),
    (100, 300, 500, 64, F16), (127, 96, 257, 32, BF16), (128, 4096, 128, 128, F16), (129, 257, 300, 128, BF16), (200, 512, 256, 64, F32), (257, 1100, 513, 32, F16),
    (300, 2500, 100, 128, F32), (513, 384, 640, 128, BF16), (700, 64, 1000, 64, F16), (1, 8192, 40, 128, BF16), (1, 4097, 35, 64, F32), (260, 777, 259, 64, BF16),
    (1030, 160, 96, 32, BF16), (4, 5000, 3, 32, F16), (48, 3000, 200, 128, F32),
    # many outputs for few rows; tiles of 32 rows, one part and several; tiles of 128 rows, likewise
    (1, 300, 8200, 64, BF16), (16, 1111, 8193, 128, F16), (7, 129, 9000, 128, F32), (40, 4100, 4000, 64, F16), (33, 8192, 1024, 128, BF16), (70, 3000, 5003, 32, BF16),
    (64, 1025, 3001, 32, F32), (500, 120, 5000, 64, F16), (130, 4100, 4203, 128, BF16), (100, 2500, 4500, 32, F32), (5000, 100, 4001, 32, BF16), (1100, 4224, 300, 64, F16),
    (300, 8200, 1000, 64, F32), (9000, 100, 4001, 32, BF16), (130, 4100, 8203, 128, BF16), (9, 4200, 500, 64, F16),
    # gradients from weights in memory
    (1100, 4224, 2100, 128, BF16), (1031, 4100, 2099, 64, F16), (701, 3001, 2100, 32, F32),
]


def _rows(rows, columns, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, columns), generator=g) * torch.exp(torch.randn((rows, 1), generator=g))).to(dtype)


def _forward_bound(x, step, zero, group, want, dtype):
    """A product of x and a code is exact (codes that are converted numbers, or 128 + code under a bfloat16 x, which then takes 135 instead of 7.5 units of
    the step); what is left out are the roundings of binary32 sums.  A sum of a group passes at most `group` of them, each off by half a unit of a
    partial sum, that of numbers of either sign: at most four times the root of the sum of squares.  The errors of roundings have either sign too: eight times the root of their number."""
    e = ((x.double() * x.double()) @ (((143 if dtype == BF16 else 15) * step + zero) ** 2).t()) ** 0.5
    groups = -(-x.shape[1] // group)
    return H.ROUNDOFF[dtype] * want.abs() + 32 * Y.UNIT * (3 * group + 2 * groups) ** 0.5 * e + 2.0 ** -25


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("bias", [None, "own", "wide"])
def test_product(case, bias):
    rows, inputs, outputs, group, dtype = case
    codes, header = Y.random_weights(outputs, inputs, group, rows + inputs)
    x = _rows(rows, inputs, dtype, outputs)
    b = None if bias is None else torch.randn(outputs, generator=torch.Generator().manual_seed(3)).to(dtype if bias == "own" else F32)
    got = B.linear4(x.to(DEV), codes.to(DEV), header.to(DEV), None if b is None else b.to(DEV))
    w, step = Y.weights(codes, header, inputs)
    zero = header[..., :1].double().abs().expand(-1, -1, group).flatten(1)[:, :inputs]
    want = x.double() @ w.t()
    if b is not None:
        want = want + b.double()
    assert got.dtype == dtype and got.shape == (rows, outputs)
    off, limit = (got.cpu().double() - want).abs(), _forward_bound(x, step, zero, group, want, dtype)
    assert (off <= limit).all(), float((off / limit).max())


@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradient(case):
    """What a product is off by, of either sign.  bfloat16: a weight may go as 11 bits of it, off by 2^-11, an element of grad_y as it is.  binary16: a weight as 16 bits
    or more, 2^-16, and what is left of products of parts, 2^-16.  binary32: 22 bits of both, 2^-23 each, without the product of the lower halves, 2^-22.
    Eight times that for the root of the sum of squares.  Sums over the outputs as above."""
    rows, inputs, outputs, group, dtype = case
    codes, header = Y.random_weights(outputs, inputs, group, rows + inputs + 1)
    grad = _rows(rows, outputs, dtype, inputs)
    got = B.linear4_backward(grad.to(DEV), codes.to(DEV), header.to(DEV), inputs)
    w, _ = Y.weights(codes, header, inputs)
    want = grad.double() @ w
    e = ((grad.double() ** 2) @ (w ** 2)) ** 0.5
    assert got.dtype == dtype and got.shape == (rows, inputs)
    limit = H.ROUNDOFF[dtype] * want.abs() + (8 * {F32: 2.0 ** -21, F16: 2.0 ** -15, BF16: 2.0 ** -11}[dtype] + 32 * Y.UNIT * (3 * outputs) ** 0.5) * e + 2.0 ** -25
    off = (got.cpu().double() - want).abs()
    assert (off <= limit).all(), float((off / limit).max())
    assert torch.equal(got, B.linear4_backward(grad.to(DEV), codes.to(DEV), header.to(DEV), inputs)), "the order of the sums is fixed"


@pytest.mark.parametrize("rows, inputs, outputs", [(20, 640, 400), (1100, 4224, 2100)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_past_outputs_without_weights_and_of_very_different_ones(rows, inputs, outputs, dtype):
    """Outputs whose weights are all zero take no part, however large grad_y is there; others'
    weights differ by 2^12 and grad_y makes up for it.  Errors as above."""
    codes, header = Y.random_weights(outputs, inputs, 128, 3)
    header[::3] = 0
    grad = _rows(rows, outputs, dtype, 4)
    grad[:, ::3] *= 2.0 ** 20
    header[1::3] *= 2.0 ** 12
    grad[:, 1::3] *= 2.0 ** -12
    got = B.linear4_backward(grad.to(DEV), codes.to(DEV), header.to(DEV), inputs)
    w, _ = Y.weights(codes, header, inputs)
    want, e = grad.double() @ w, ((grad.double() ** 2) @ (w ** 2)) ** 0.5
    limit = H.ROUNDOFF[dtype] * want.abs() + (8 * {F32: 2.0 ** -21, BF16: 2.0 ** -11}[dtype] + 32 * Y.UNIT * (3 * outputs) ** 0.5) * e
    off = (got.cpu().double() - want).abs()
    assert (off <= limit).all(), float((off / limit).max())
    assert float((got.cpu().double() - want).norm() / want.norm()) <= (2.0 ** -21 if dtype == F32 else 1.1 * H.ROUNDOFF[dtype] / 3 ** 0.5)


@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_errors_as_a_whole(rows, dtype):
    """Over many elements the error is that of one rounding (a third of whose square is its mean square at most), and of binary32 sums a few per cent of that at
    most; binary32 itself: a fraction of 2^-21 of the result."""
    inputs, outputs = 2048, 512
    codes, header = Y.random_weights(outputs, inputs, 128, 5)
    x, w = _rows(rows, inputs, dtype, 6), Y.weights(codes, header, inputs)[0]
    grad = _rows(rows, outputs, dtype, 7)
    for got, want in ((B.linear4(x.to(DEV), codes.to(DEV), header.to(DEV)), x.double() @ w.t()), (B.linear4_backward(grad.to(DEV), codes.to(DEV), header.to(DEV), inputs), grad.double() @ w)):
        off = float((got.cpu().double() - want).norm() / want.norm())
        assert off <= (2.0 ** -21 if dtype == F32 else 1.1 * H.ROUNDOFF[dtype] / 3 ** 0.5), off


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("outputs, inputs", [(1, 1), (3, 31), (65, 128), (17, 129), (200, 1000), (5, 4096)])
def test_quantizer(outputs, inputs, group, dtype):
    """Bit for bit; what is read back is within half a step, what rounding zero and step to bfloat16 costs, and the last rounding."""
    w = _rows(outputs, inputs, dtype, inputs)
    w[0, :] = 0.25   # a group of equal weights
    if inputs > 40:
        w[outputs // 2, :32] *= 1e-3
    codes, header = B.quantize_weights(w.to(DEV), group)
    want, zero, step = Y.quantise_weights(w, group)
    assert torch.equal(codes.cpu(), Y.pack(want)) and torch.equal(header.cpu(), torch.stack((zero, step), -1).bfloat16())
    back = B.dequantize_weights(codes, header, inputs, dtype).cpu()
    held, steps = Y.weights(codes.cpu(), header.cpu(), inputs)
    assert back.dtype == dtype
    assert (back.double() - held).abs().le((H.ROUNDOFF[dtype] + 2 * Y.UNIT) * (held.abs() + 16 * steps) + 2.0 ** -25).all()
    zeros = zero.double().abs()[..., None].expand(-1, -1, group).flatten(1)[:, :inputs]
    assert (held - w.double()).abs().le(0.5 * steps + 2.0 ** -8 * (zeros + 15 * steps) + 1e-30).all()


def test_groups_that_are_not_finite_read_as_nan():
    w = torch.randn((4, 256), generator=torch.Generator().manual_seed(1))
    w[1, 130], w[2, 5], w[3, 0], w[3, 1] = float("nan"), float("inf"), 3e38, -3e38
    codes, header = B.quantize_weights(w.to(DEV), 128)
    back = B.dequantize_weights(codes, header, 256, F32).cpu()
    nan = torch.isnan(back)
    assert nan[1, 128:].all() and nan[2, :128].all() and nan[3, :128].all() and nan.sum() == 3 * 128
    x = torch.ones((2, 256), device=DEV)
    y = B.linear4(x, codes, header).cpu()
    assert torch.isfinite(y[:, 0]).all() and torch.isnan(y[:, 1:]).all()
    g = B.linear4_backward(torch.ones((2, 4), device=DEV), codes, header, 256).cpu()
    assert torch.isnan(g).all()
    g = B.linear4_backward(torch.ones((2, 1), device=DEV), codes[:1], header[:1], 256).cpu()
    assert torch.isfinite(g).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, inputs, outputs", [(5, 2560, 8200), (40, 2560, 5000), (700, 2560, 5000)])
def test_groups_of_many_that_are_not_finite(rows, inputs, outputs, dtype):
    """In every kernel such a group is seen by its output, and in the gradient by its inputs, alone."""
    codes, header = (t.to(DEV) for t in Y.random_weights(outputs, inputs, 64, 2))
    header[17, 3, 0], header[outputs - 1, 39, 1] = float("nan"), float("inf")
    y = B.linear4(_rows(rows, inputs, dtype, 3).to(DEV), codes, header)
    bad = ~torch.isfinite(y)
    assert bad[:, 17].all() and bad[:, outputs - 1].all() and int(bad.sum()) == 2 * rows
    g = B.linear4_backward(_rows(rows, outputs, dtype, 4).to(DEV), codes, header, inputs)
    bad = ~torch.isfinite(g)
    assert bad[:, 192:256].all() and int(bad[:, :2496].sum()) == 64 * rows   # of the last group a code of zero times infinity is what its column has


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows, inputs, outputs", [(3, 300, 100), (300, 300, 100), (40, 4100, 4000), (1100, 4100, 2100)])
def test_rows_that_are_not_finite_are_their_own_business(rows, inputs, outputs, dtype):
    codes, header = (t.to(DEV) for t in Y.random_weights(outputs, inputs, 64, 2))
    for call, columns in ((lambda x: B.linear4(x, codes, header), inputs), (lambda x: B.linear4_backward(x, codes, header, inputs), outputs)):
        x = _rows(rows, columns, dtype, 3).to(DEV)
        fine = call(x)
        bad = x.clone()
        bad[1, 7], bad[rows - 1, 0] = float("nan"), float("inf")
        got = call(bad)
        keep = [i for i in range(rows) if i not in (1, rows - 1)]
        assert torch.equal(got[keep], fine[keep])
        assert torch.isnan(got[1]).all() and not torch.isfinite(got[rows - 1]).any()


@pytest.mark.parametrize("rows, inputs, outputs", [(1, 200, 70), (40, 200, 70), (5, 1024, 8201), (40, 4096, 4003), (200, 5001, 3001), (300, 512, 2050)])
def test_strides_shapes_and_neighbours(rows, inputs, outputs):
    codes, header = (t.to(DEV) for t in Y.random_weights(outputs, inputs, 32, 4))
    wide = _rows(rows, inputs + 107, BF16, 5).to(DEV)
    x = wide[:, 3:3 + inputs]
    want = B.linear4(x.contiguous(), codes, header)
    assert torch.equal(B.linear4(x, codes, header), want)
    out = torch.full((rows, outputs + 29), 7.0, dtype=BF16, device=DEV)
    assert torch.equal(B.linear4(x, codes, header, out=out[:, 11:11 + outputs]), want)
    assert (out[:, :11] == 7).all() and (out[:, 11 + outputs:] == 7).all()
    assert torch.equal(B.linear4(x.contiguous().view(rows, 1, 1, inputs), codes, header), want.view(rows, 1, 1, outputs))
    assert torch.equal(B.linear4(x[:1].expand(rows, inputs), codes, header), want[:1].expand(rows, outputs))   # rows that share memory may be read
    assert torch.equal(B.linear4(x.flip(0), codes, header).flip(0), want)
    grad = _rows(rows, outputs + 20, F16, 6).to(DEV)[:, 5:5 + outputs]
    assert torch.equal(B.linear4_backward(grad, codes, header, inputs), B.linear4_backward(grad.contiguous(), codes, header, inputs))
    assert torch.equal(B.linear4_backward(grad.contiguous().view(rows, 1, outputs), codes, header, inputs).view(rows, inputs), B.linear4_backward(grad, codes, header, inputs))


def test_one_vector_and_no_rows():
    codes, header = (t.to(DEV) for t in Y.random_weights(70, 200, 32, 4))
    x = _rows(1, 200, F16, 5).to(DEV)
    assert torch.equal(B.linear4(x[0], codes, header), B.linear4(x, codes, header)[0])
    assert B.linear4(x[:0], codes, header).shape == (0, 70) and B.linear4_backward(torch.zeros((2, 0, 70), device=DEV), codes, header, 200).shape == (2, 0, 200)


def test_weights_beyond_two_to_the_32():
    """Offsets of the last outputs pass 32 bits: 2^33 weights, of which the last rows are looked at."""
    outputs, inputs = (1 << 19) + 3, 16384
    header = torch.zeros((outputs, inputs // 128, 2), dtype=BF16, device=DEV)
    codes = torch.zeros((outputs, inputs // 8), dtype=torch.int32, device=DEV)
    some, head = Y.random_weights(5, inputs, 128, 6)
    codes[-5:], header[-5:] = some.to(DEV), head.to(DEV)
    x = _rows(2, inputs, F32, 7)
    y = B.linear4(x.to(DEV), codes, header)
    w, step = Y.weights(some, head, inputs)
    want = x.double() @ w.t()
    zero = head[..., :1].double().abs().expand(-1, -1, 128).flatten(1)
    assert ((y[:, -5:].cpu().double() - want).abs() <= _forward_bound(x, step, zero, 128, want, F32)).all() and (y[:, :-5] == 0).all()
    grad = torch.zeros((1, outputs), device=DEV)
    grad[:, -5:] = 1.0
    g = B.linear4_backward(grad, codes, header, inputs).cpu().double()
    assert ((g - w.sum(0)).abs() <= 2.0 ** -20 * w.abs().sum(0)).all()


def test_refused_by_the_binding():
    codes, header = (t.to(DEV) for t in Y.random_weights(70, 200, 32, 4))
    x = torch.zeros((3, 200), device=DEV)
    for args, error in (((x[:, :192], codes, header), ValueError), ((torch.zeros((3, 225), device=DEV), codes, header), ValueError), ((x.double(), codes, header), TypeError),
                        ((x, codes.long(), header), TypeError), ((x, codes, header.float()), TypeError), ((x, codes[:, :-1], header), ValueError), ((x, codes, header[:-1]), ValueError),
                        ((x, codes, header, torch.zeros(69, device=DEV)), ValueError), ((x, codes, header, torch.zeros(70, device=DEV, dtype=F16)), TypeError),
                        ((x, codes, header, None, torch.zeros((3, 71), device=DEV)), ValueError), ((x, codes, header, None, torch.zeros((3, 70), device=DEV, dtype=F16)), TypeError),
                        ((x, codes.t().contiguous().t(), header), ValueError), ((x.t().contiguous().t(), codes, header), ValueError)):
        with pytest.raises(error):
            B.linear4(*args)
    with pytest.raises(ValueError, match="overlap"):
        B.linear4(x, codes, header, None, torch.zeros((1, 70), device=DEV).expand(3, 70))
    square = torch.zeros((40, 200), device=DEV)
    with pytest.raises(RuntimeError):   # a result over what others still read
        B.linear4(square, *(t.to(DEV) for t in Y.random_weights(200, 200, 32, 5)), None, square)
    with pytest.raises(ValueError, match="per output"):
        B.linear4_backward(x, codes, header, 200)
    with pytest.raises(B.ActqError, match="group"):
        B.linear4(torch.zeros((3, 200), device=DEV), torch.zeros((5, 32), dtype=torch.int32, device=DEV), torch.zeros((5, 1, 2), dtype=BF16, device=DEV))


def test_captured_and_replayed_with_several_graphs():
    """Graphs of the same weights, each with its own workspace, replayed in turn with other inputs and eager calls between."""
    codes, header = (t.to(DEV) for t in Y.random_weights(2000, 3000, 64, 4))
    g = torch.Generator().manual_seed(8)
    graphs = []
    side = torch.cuda.Stream()
    for rows in (1, 60, 1500):
        x, grad = torch.zeros((rows, 3000), dtype=BF16, device=DEV), torch.zeros((rows, 2000), dtype=BF16, device=DEV)
        call = lambda x=x, grad=grad: (B.linear4(x, codes, header), B.linear4_backward(grad, codes, header, 3000))   # noqa: E731
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = call()
        torch.cuda.current_stream().wait_stream(side)
        graphs.append((graph, x, grad, out, call))
    for i in range(3):
        for _, x, grad, _, _ in graphs:
            x.copy_(torch.randn(x.shape, generator=g).to(BF16))
            grad.copy_(torch.randn(grad.shape, generator=g).to(BF16))
        for graph, *_ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, _, _, out, call in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, call())), i
