"""The gradient of the bias: what the library refuses before anything is launched (nothing here needs a GPU)."""
import ctypes

from paper_2104_14129_amd import binding as B
from test_heads_refusals import FAKE, _refused
from test_layer_refusals import BAD_ROWS, _rows


def test_refusals():
    L = B.lib()
    # grad_y, dt, rows, outputs, grad_bias, bias_dt, workspace, bytes, stream
    ok = [_rows(), 2, 5000, 300, FAKE, 0, FAKE, 1 << 30, None]
    _refused(L.actq_linear4_backward_bias, ok, [(0, r) for r in BAD_ROWS] + [(1, 3), (1, -1), (2, -1), (2, 1 << 20), (3, 0), (3, (1 << 20) + 1), (4, None), (4, FAKE + 2), (5, 1), (5, 3),
                                                (6, None), (6, FAKE + 8), (7, 100)])
    size = ctypes.c_uint64()
    query = L.actq_linear4_backward_bias_workspace
    assert query(5000, 300, ctypes.addressof(size)) == 0 and size.value == 313 * 300 * 4
    assert query(16, 300, ctypes.addressof(size)) == 0 and size.value == 0
    assert query(0, 300, ctypes.addressof(size)) == 0 and size.value == 0
    assert query((1 << 20) - 1, 1 << 20, ctypes.addressof(size)) == 0 and size.value == 0
    for wrong in ((-1, 300, ctypes.addressof(size)), (1 << 20, 300, ctypes.addressof(size)), (5, 0, ctypes.addressof(size)), (5, (1 << 20) + 1, ctypes.addressof(size)), (5, 300, None)):
        assert query(*wrong) == B.ACTQ_EINVAL
