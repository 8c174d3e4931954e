"""Products with 4-bit weights at the ends of the range of their types: what is finite stays finite, in every kernel."""
import pytest
import torch

import _layer as Y
from paper_2104_14129_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16

# rows, inputs, outputs, group: few rows, few rows of many outputs, tiles of 32 rows (several parts and one), tiles of 128 rows
KERNELS = [(3, 300, 100, 32), (5, 300, 8200, 128), (40, 4100, 4000, 64), (64, 300, 5000, 128), (700, 2560, 5000, 64), (700, 2500, 5000, 128), (130, 4100, 8203, 32)]


def _rows(rows, columns, dtype, seed):
    return torch.randn((rows, columns), generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def _shape(case):
    return pytest.param(*case, id="-".join(map(str, case)))


@pytest.mark.parametrize("rows, inputs, outputs, group", map(_shape, KERNELS))
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("power", [124, -60])
def test_a_power_of_two_in_x_is_one_in_the_result(rows, inputs, outputs, group, dtype, power):
    """Every rounding commutes with it as long as nothing leaves the range.  x is below 2^3 times that power, weights below 2^-9, a result of 4100 of them (a sum of
    either sign, 64 of its parts) below 2^120: finite in both types, while x times a code would not be."""
    codes, header = (t.to(DEV) for t in Y.random_weights(outputs, inputs, group, 1))
    header *= 2.0 ** -10
    x = _rows(rows, inputs, dtype, 2)
    y = B.linear4(x, codes, header)
    scaled = B.linear4(x * 2.0 ** power, codes, header)
    assert torch.isfinite(scaled).all() and (y != 0).any()
    assert torch.equal(scaled, y * 2.0 ** power)


@pytest.mark.parametrize("rows, inputs, outputs, group", map(_shape, KERNELS))
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_zeros_times_the_largest_weights(rows, inputs, outputs, group, dtype):
    codes, header = (t.to(DEV) for t in Y.random_weights(outputs, inputs, group, 3))
    header[..., 1] = header[..., 1].abs() * 2.0 ** 120
    header[..., 0] = -header[..., 1]
    assert torch.isfinite(header).all()
    y = B.linear4(torch.zeros((rows, inputs), dtype=dtype, device=DEV), codes, header)
    assert (y == 0).all()


# rows, inputs, outputs: few rows, and from weights in memory
@pytest.mark.parametrize("rows, inputs, outputs", [(20, 640, 400), (1100, 4224, 2100)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("of_grad, of_weights", [(-90, 0), (100, 0), (60, -100), (-60, 117)])
def test_powers_of_two_in_a_gradient(rows, inputs, outputs, dtype, of_grad, of_weights):
    """Every rounding commutes with them as long as nothing leaves the range: weights are between 2^-8 and 2 (but for what is rounded off in any case), elements of
    grad_y below 2^3, so that 24 bits of both and of their products fit it with these powers."""
    codes, header = (t.to(DEV) for t in Y.random_weights(outputs, inputs, 64, 1))
    grad = _rows(rows, outputs, dtype, 2)
    want = B.linear4_backward(grad, codes, header, inputs)
    got = B.linear4_backward(grad * 2.0 ** of_grad, codes, header * 2.0 ** of_weights, inputs)
    assert torch.isfinite(got).all() and (want != 0).any()
    assert torch.equal(got, want * 2.0 ** (of_grad + of_weights))


@pytest.mark.parametrize("rows, inputs, outputs, group", map(_shape, KERNELS))
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_an_infinity_in_a_row_leaves_nothing_finite_there(rows, inputs, outputs, group, dtype):
    """Nor does it where every weight is above zero, and nothing takes from it."""
    codes, header = (t.to(DEV) for t in Y.random_weights(outputs, inputs, group, 1))
    header[..., 1] = header[..., 1].abs()
    header[: outputs // 2, :, 0] = 300 * header[: outputs // 2, :, 1]
    x = _rows(rows, inputs, dtype, 2)
    x[0, 5], x[rows - 1, inputs - 1] = float("inf"), -float("inf")
    finite = torch.isfinite(B.linear4(x, codes, header))
    assert not finite[0].any() and not finite[rows - 1].any() and finite[1:rows - 1].all()
