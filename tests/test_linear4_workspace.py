"""How much memory the products with 4-bit weights ask for (nothing here needs a GPU)."""
import ctypes

import pytest

from paper_2104_14129_amd import binding as B


def _bytes(f, dt, rows, inputs, outputs, group=128):
    size = ctypes.c_uint64()
    assert f(B.Weights4Desc(0x1000, 0x1000, inputs, outputs, group), dt, rows, ctypes.addressof(size)) == B.ACTQ_OK
    return size.value


@pytest.mark.parametrize("dt, most_rows", [(0, 64), (1, 128), (2, 128)])
@pytest.mark.parametrize("inputs, outputs", [(4096, 4096), (8192, 16384), (8192, 131072), (16384, 524291), (1 << 20, 1 << 20), (64, 1 << 20), (1 << 20, 64), (1001, 333)])
def test_gradients_of_few_rows_ask_for_their_parts_alone(dt, most_rows, inputs, outputs):
    """At most 512 tiles of 128 columns in binary32, whatever the weights are."""
    f = B.lib().actq_linear4_backward_workspace
    for rows in (1, 2, 9, 33, 64, 65, 128):
        if rows <= most_rows:
            assert _bytes(f, dt, rows, inputs, outputs) <= rows * 512 * 128 * 4


@pytest.mark.parametrize("dt, size", [(0, 4), (1, 2), (2, 2)])
def test_gradients_of_many_rows_ask_for_two_bytes_a_weight(dt, size):
    """And for grad_y, padded, the middles of the groups with their sums, and parts of the result."""
    f = B.lib().actq_linear4_backward_workspace
    for rows, inputs, outputs, group in ((300, 8192, 16384, 128), (4096, 4096, 8192, 32), (2047, 5000, 5001, 64)):
        padded, groups, padded_rows = (outputs + 63) // 64 * 64, (inputs + group - 1) // group, (rows + 255) // 256 * 256
        parts = max(1, 256 // (padded_rows // 256 * ((inputs + 127) // 128)))
        most = inputs * padded * 2 + rows * padded * size + groups * padded * 4 + padded_rows * groups * 4 * 257 + (parts * rows * inputs * 4 if parts > 1 else 0) + 4 * (outputs + padded_rows) + 64
        assert inputs * outputs * 2 <= _bytes(f, dt, rows, inputs, outputs, group) <= most
