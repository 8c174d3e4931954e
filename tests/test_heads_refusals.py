"""Attention heads: what the library and the binding refuse, before anything is launched (nothing here needs a GPU)."""
import ctypes

import pytest
import torch

from paper_2104_14129_amd import binding as B
from paper_2104_14129_amd.cache import PagedCache

FAKE = 0x1000   # never dereferenced by validation
E = B.ACTQ_EINVAL


def _heads(heads=4, data=FAKE, token=512, head=128):
    return B.Heads(data, token, head, heads)


def _rotation(**other):
    r = dict(positions=FAKE, cos=FAKE, sin=FAKE, rows=10, rotated=128, interleaved=0)
    r.update(other)
    return B.RotationDesc(*[r[name] for name, _ in B.RotationDesc._fields_])


def _cache(**other):
    c = dict(key_codes=FAKE, key_header=FAKE, value_codes=FAKE, value_header=FAKE, pages=4, page_size=16, heads=2, dim=128, key_bits=8, value_bits=4)
    c.update(other)
    return B.CacheDesc(*[c[name] for name, _ in B.CacheDesc._fields_])


def _refused(f, ok, changes):
    for at, bad in changes:
        args = list(ok)
        args[at] = bad
        assert f(*args) == E, (at, bad)
        assert B.last_error()


NAN, INF = float("nan"), float("inf")


def test_head_norm_refusals():
    L = B.lib()
    # q, k, dt, tokens, dim, q_weight, k_weight, weight_dt, rotation, eps, q_out, k_out, stream
    ok = [_heads(), _heads(2), 1, 8, 128, FAKE, FAKE, 1, _rotation(), 1e-6, _heads(), _heads(2), None]
    changes = [(0, None), (2, 3), (2, -1), (3, -1), (3, 1 << 24), (4, 96), (4, 0), (7, 2), (5, FAKE + 1), (9, 0.0), (9, -1.0), (9, NAN), (9, INF), (8, None),
               (0, _heads(data=None)), (0, _heads(data=FAKE + 1)), (0, _heads(0)), (0, _heads(65536)), (0, _heads(token=1 << 40)), (10, None), (10, _heads(5)),
               (11, _heads(3)), (11, None), (8, _rotation(rotated=8)), (8, _rotation(rotated=136)), (8, _rotation(rotated=144)), (8, _rotation(rows=0)),
               (8, _rotation(cos=None)), (8, _rotation(positions=FAKE + 2)), (8, _rotation(interleaved=2))]
    _refused(L.actq_head_norm_rotate, ok, changes)
    none = list(ok)
    none[3], none[0], none[1], none[10], none[11] = 0, _heads(data=None), _heads(2, data=None), _heads(data=None), _heads(2, data=None)
    none[8] = _rotation(positions=None, cos=None, sin=None)
    assert L.actq_head_norm_rotate(*none) == B.ACTQ_OK   # no token is no work
    # grad_q, grad_k, q, k, dt, tokens, dim, q_weight, k_weight, weight_dt, rotation, eps, grad_q_in, grad_k_in, grad_q_weight, grad_k_weight, workspace, bytes, stream
    back = [_heads(), _heads(2), _heads(), _heads(2), 0, 8, 128, FAKE, FAKE, 0, _rotation(), 1e-6, _heads(), _heads(2), FAKE, FAKE, FAKE, 1 << 20, None]
    _refused(L.actq_head_norm_rotate_backward, back, [(0, None), (1, None), (2, None), (4, 5), (12, None), (13, _heads(1)), (14, FAKE + 2), (16, None), (16, FAKE + 8),
                                                      (17, 100), (3, None), (9, 1), (11, NAN)])
    size = ctypes.c_uint64()
    assert L.actq_head_norm_workspace(8, 128, ctypes.addressof(size)) == 0 and size.value == 2 * 2 * 128 * 4
    for args in ((8, 100, ctypes.addressof(size)), (-1, 128, ctypes.addressof(size)), (8, 128, None)):
        assert L.actq_head_norm_workspace(*args) == E


def test_cache_refusals():
    L = B.lib()
    caches = [None, _cache(pages=0), _cache(pages=1 << 31), _cache(page_size=8), _cache(page_size=24), _cache(page_size=2048), _cache(heads=0), _cache(dim=80),
              _cache(key_bits=2), _cache(value_bits=16), _cache(key_codes=None), _cache(key_codes=FAKE + 8), _cache(value_header=FAKE + 4)]
    # cache, k, v, dt, tokens, slots, stream
    ok = [_cache(), _heads(2), _heads(2), 2, 5, FAKE, None]
    _refused(L.actq_cache_write, ok, [(0, c) for c in caches] + [(1, None), (1, _heads(3)), (2, _heads(2, data=FAKE + 1)), (3, 7), (4, -1), (4, 1 << 26), (5, None), (5, FAKE + 4)])
    ok = [_cache(), FAKE, 5, _heads(2), _heads(2), 0, None]
    _refused(L.actq_cache_read, ok, [(0, c) for c in caches] + [(1, None), (2, -1), (3, _heads(1)), (4, None), (5, 3)])
    # cache, q, dt, tokens, sequences, table, table_width, lengths, query_start, max_query, max_length, scale, softcap, window, out, workspace, bytes, stream
    ok = [_cache(), _heads(8), 1, 3, 3, FAKE, 64, FAKE, FAKE, 1, 1000, 0.1, 0.0, 0, _heads(8), FAKE, 1 << 30, None]
    _refused(L.actq_cache_attention, ok, [(0, c) for c in caches] + [
        (1, None), (1, _heads(3)), (14, None), (14, _heads(4)), (2, 4), (3, -1), (4, -1), (4, 1 << 20), (5, None), (5, FAKE + 2), (6, 0), (6, 1 << 27), (7, None), (8, None),
        (9, -1), (9, 1 << 31), (10, -1), (11, INF), (11, NAN), (12, -1.0), (12, INF), (12, NAN), (13, -1), (15, None), (15, FAKE + 4), (16, 8)])
    none = list(ok)
    none[3], none[1], none[14] = 0, _heads(8, data=None), _heads(8, data=None)
    assert L.actq_cache_attention(*none) == B.ACTQ_OK
    size = ctypes.c_uint64(7)
    assert L.actq_cache_attention_workspace(_cache(), 8, 3, 3, 1, 100, 0, ctypes.addressof(size)) == 0 and size.value == 0   # one part
    assert L.actq_cache_attention_workspace(_cache(), 8, 3, 3, 1, 5000, 0, ctypes.addressof(size)) == 0 and size.value % (3 * 8 * 130 * 4) == 0 and size.value > 0
    assert L.actq_cache_attention_workspace(_cache(), 8, 3, 3, 1, 5000, 0, None) == E


def test_the_other_calls_do_not_take_bfloat16():
    L = B.lib()
    assert L.actq_relu_forward(FAKE, B.ACTQ_BF16, 10, FAKE, FAKE, None) == E
    assert L.actq_group_stats(FAKE, B.ACTQ_BF16, 1, 256, 256, FAKE, FAKE, None) == E


def test_host_tensors_are_refused():
    x, t, codes, header = torch.zeros((2, 2, 64)), torch.zeros((4, 32)), torch.zeros((1, 2, 16, 64), dtype=torch.uint8), torch.zeros((1, 2, 16, 2))
    i, slots = torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    cache = (codes, header, codes, header)
    for call in (lambda: B.head_norm_rotate(x, x, None, None, i, t, t), lambda: B.head_norm_rotate_backward(x, x, x, x, None, None, i, t, t),
                 lambda: B.cache_write(x, x, slots, *cache), lambda: B.cache_read(slots, *cache, 64, torch.float32),
                 lambda: B.cache_attention(x, *cache, i.view(2, 1), i, torch.zeros(3, dtype=torch.int32), 1, 1)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_a_cache_of_other_widths_is_refused():
    with pytest.raises(ValueError, match="4 or 8"):
        PagedCache(1, 16, 1, 64, key_bits=2, device="cpu")
