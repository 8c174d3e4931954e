"""A layer around the attention: what the library and the binding refuse, before anything is launched (nothing here needs a GPU)."""
import ctypes

import pytest
import torch

from paper_2104_14129_amd import binding as B
from paper_2104_14129_amd import layers as L
from test_heads_refusals import FAKE, INF, NAN, _cache, _heads, _refused, _rotation

E = B.ACTQ_EINVAL


def _rows(data=FAKE, stride=4096):
    return B.RowsDesc(data, stride)


def _block(gates=None, **other):
    b = dict(tokens=8, width=4096, dt=2, weight_dt=2, weight=FAKE, post_weight=FAKE, gate=FAKE, gates=None, scale=1.0, eps=1e-6)
    b.update(other)
    d = B.BlockDesc(*[b[name] for name, _ in B.BlockDesc._fields_ if name != "gates"][:7])
    d.scale, d.eps = b["scale"], b["eps"]
    if gates is not None:
        d.gates = ctypes.pointer(gates)
    return d


def _weights(**other):
    w = dict(codes=FAKE, header=FAKE, inputs=1000, outputs=77, group=128)
    w.update(other)
    return B.Weights4Desc(*[w[name] for name, _ in B.Weights4Desc._fields_])


BAD_BLOCKS = [None, _block(dt=3), _block(weight_dt=1), _block(tokens=-1), _block(tokens=1 << 26), _block(width=0), _block(width=16385), _block(weight=None),
              _block(weight=FAKE + 1), _block(post_weight=FAKE + 1), _block(gate=FAKE + 1), _block(gates=_rows()), _block(gate=None, gates=_rows(None)),
              _block(gate=None, gates=_rows(FAKE + 1)), _block(scale=INF), _block(scale=NAN), _block(eps=0.0), _block(eps=-1.0), _block(eps=NAN), _block(eps=INF)]
BAD_ROWS = [None, _rows(None), _rows(FAKE + 1), _rows(stride=1 << 36), _rows(stride=-(1 << 36))]


def test_block_norm_refusals():
    L_ = B.lib()
    # block, x, h, r, y, stream
    ok = [_block(), _rows(), _rows(), _rows(), _rows(), None]
    _refused(L_.actq_block_norm, ok, [(0, b) for b in BAD_BLOCKS] + [(i, r) for i in (1, 2, 3, 4) for r in BAD_ROWS])
    alone = [_block(post_weight=None, gate=None), _rows(), None, None, _rows(), None]
    _refused(L_.actq_block_norm, alone, [(0, _block(gate=None)), (0, _block(post_weight=None)), (3, _rows()), (0, _block(post_weight=None, gate=None, gates=_rows()))])
    empty = [_block(tokens=0), _rows(None), _rows(None), _rows(None), _rows(None), None]
    assert L_.actq_block_norm(*empty) == B.ACTQ_OK   # no token is no work
    # block, grad_r, grad_y, r, h, grad_x, grad_h, grad_gates, grad_weight, grad_post_weight, grad_gate, workspace, bytes, stream
    ok = [_block(), _rows(), _rows(), _rows(), _rows(), _rows(), _rows(), None, FAKE, FAKE, FAKE, FAKE, 1 << 30, None]
    _refused(L_.actq_block_norm_backward, ok, [(0, b) for b in BAD_BLOCKS] + [(1, r) for r in BAD_ROWS[1:]] + [(i, r) for i in (2, 3, 4, 5, 6) for r in BAD_ROWS] + [
        (7, _rows()), (8, None), (8, FAKE + 1), (9, None), (9, FAKE + 1), (10, None), (10, FAKE + 1), (11, None), (11, FAKE + 8), (12, 100), (4, None)])
    gates = list(ok)
    gates[0], gates[7], gates[10] = _block(gate=None, gates=_rows()), _rows(), None
    _refused(L_.actq_block_norm_backward, gates, [(7, None), (7, _rows(FAKE + 1)), (10, FAKE)])
    size = ctypes.c_uint64()
    assert L_.actq_block_norm_workspace(_block(), ctypes.addressof(size)) == 0 and size.value == 8 * 3 * 4096 * 4
    assert L_.actq_block_norm_workspace(_block(tokens=0), ctypes.addressof(size)) == 0 and size.value == 0
    assert L_.actq_block_norm_workspace(_block(width=0), ctypes.addressof(size)) == E and L_.actq_block_norm_workspace(_block(), None) == E


def test_linear4_refusals():
    L_ = B.lib()
    bad = [None, _weights(codes=None), _weights(codes=FAKE + 2), _weights(codes=FAKE + 8), _weights(header=None), _weights(header=FAKE + 2), _weights(inputs=0), _weights(inputs=(1 << 20) + 1),
           _weights(outputs=0), _weights(outputs=(1 << 20) + 1), _weights(group=16), _weights(group=256), _weights(group=96)]
    # weights, x, dt, rows, bias, bias_dt, y, workspace, bytes, stream
    ok = [_weights(), _rows(), 1, 5, FAKE, 0, _rows(), FAKE, 1 << 40, None]
    _refused(L_.actq_linear4, ok, [(0, w) for w in bad] + [(i, r) for i in (1, 6) for r in BAD_ROWS] + [(2, 3), (3, -1), (3, 1 << 20), (4, FAKE + 2), (5, 2)])
    # weights, grad_y, dt, rows, grad_x, workspace, bytes, stream
    back = [_weights(), _rows(), 1, 5, _rows(), FAKE, 1 << 40, None]
    _refused(L_.actq_linear4_backward, back, [(0, w) for w in bad] + [(i, r) for i in (1, 4) for r in BAD_ROWS] + [(2, 4), (3, -1), (3, 1 << 20)])
    assert L_.actq_linear4(_weights(), _rows(None), 1, 0, None, 1, _rows(None), None, 0, None) == B.ACTQ_OK
    assert L_.actq_linear4_backward(_weights(), _rows(None), 1, 0, _rows(None), None, 0, None) == B.ACTQ_OK
    size = ctypes.c_uint64()
    for f, call, args in ((L_.actq_linear4_workspace, L_.actq_linear4, lambda w, n: [w, _rows(), 1, 5000, FAKE, 0, _rows(), FAKE, n, None]),
                          (L_.actq_linear4_backward_workspace, L_.actq_linear4_backward, lambda w, n: [w, _rows(), 1, 5000, _rows(), FAKE, n, None])):
        for rows in (0, 1, 200, 5000):
            for dt in (0, 1, 2):
                for w in (_weights(), _weights(inputs=1, outputs=1), _weights(inputs=1 << 20, outputs=1 << 20)):
                    assert f(w, dt, rows, ctypes.addressof(size)) == 0 and (size.value == 0 or rows > 0)
        assert f(_weights(), 1, 5000, ctypes.addressof(size)) == 0
        if size.value:   # one byte less, none, or misaligned
            assert call(*args(_weights(), size.value - 1)) == E
            for bad_workspace in (None, FAKE + 8):
                a = args(_weights(), size.value)
                a[-3] = bad_workspace
                assert call(*a) == E
        for wrong in ((_weights(group=3), 1, 5, ctypes.addressof(size)), (_weights(), 7, 5, ctypes.addressof(size)), (_weights(), 1, -1, ctypes.addressof(size)), (_weights(), 1, 5, None)):
            assert f(*wrong) == E
    for f, args in ((L_.actq_weights4_quantize, [_rows(), 0, _weights(), None]), (L_.actq_weights4_dequantize, [_weights(), _rows(), 0, None])):
        at = args.index(next(a for a in args if isinstance(a, B.Weights4Desc)))
        _refused(f, args, [(at, w) for w in bad] + [(1 if at == 2 else 2, 3)] + [(0 if at == 2 else 1, r) for r in BAD_ROWS])


def test_append_refusals():
    L_ = B.lib()
    # cache, q, k, v, dt, tokens, q_weight, k_weight, weight_dt, rotation, norm, eps, slots, q_out, stream
    ok = [_cache(), _heads(8), _heads(2), _heads(2), 2, 5, FAKE, FAKE, 0, _rotation(), 1, 1e-6, FAKE, _heads(8), None]
    _refused(L_.actq_cache_append, ok, [(0, None), (0, _cache(dim=80)), (0, _cache(pages=0)), (0, _cache(key_codes=None)), (1, None), (1, _heads(0)), (1, _heads(data=None)),
                                        (2, None), (2, _heads(3)), (3, None), (3, _heads(2, data=FAKE + 1)), (4, 3), (5, -1), (5, 1 << 24), (6, FAKE + 2), (7, FAKE + 2), (8, 1), (9, None),
                                        (9, _rotation(rotated=8)), (9, _rotation(rows=0)), (9, _rotation(cos=None)), (10, 2), (10, 0), (11, 0.0), (11, NAN), (11, -1.0), (12, None),
                                        (12, FAKE + 4), (13, None), (13, _heads(7))])
    none = list(ok)
    none[5] = 0
    for i, heads in ((1, 8), (2, 2), (3, 2), (13, 8)):
        none[i] = _heads(heads, data=None)
    assert L_.actq_cache_append(*none) == B.ACTQ_OK
    none[10], none[6], none[7], none[11] = 0, None, None, NAN   # without norm eps takes no part
    assert L_.actq_cache_append(*none) == B.ACTQ_OK
    none[1] = none[13] = None
    assert L_.actq_cache_append(*none) == B.ACTQ_OK
    none[6] = FAKE
    assert L_.actq_cache_append(*none) == E


def test_host_tensors_are_refused():
    x, w, t = torch.zeros((2, 64)), torch.ones(64), torch.zeros((4, 32))
    q, codes, header = torch.zeros((2, 2, 64)), torch.zeros((1, 2, 16, 64), dtype=torch.uint8), torch.zeros((1, 2, 16, 2))
    i, slots = torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    c4, h4 = torch.zeros((3, 8), dtype=torch.int32), torch.zeros((3, 1, 2), dtype=torch.bfloat16)
    for call in (lambda: B.block_norm(x, x, None, w), lambda: B.block_norm_backward(x, x, x, x, None, w), lambda: B.quantize_weights(x, 64),
                 lambda: B.dequantize_weights(c4, h4, 64, torch.float32), lambda: B.linear4(x, c4, h4), lambda: B.linear4_backward(torch.zeros((2, 3)), c4, h4, 64),
                 lambda: B.cache_append(q, q, q, None, None, i, t, t, slots, codes, header, codes, header)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_groups_that_are_none_are_refused():
    for group in (16, 100, 256):
        with pytest.raises(ValueError, match="group"):
            B.quantize_weights(torch.zeros((2, 64)), group)
    with pytest.raises(ValueError, match="outputs, inputs"):
        B.quantize_weights(torch.zeros(64), 64)
