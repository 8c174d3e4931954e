"""Norm and rotation of attention heads, the quantised cache and the attention over it, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import _heads as H
from paper_2104_14129_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _randn(*shape, seed, dtype=F32, scale=1.0):
    return (scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(dtype)


# ----------------------------------------------------------------------------- norm and rotation

def _norm_case(tokens, q_heads, k_heads, dim, dtype, rotated, wide, seed):
    x = _randn(tokens, (q_heads + k_heads + 1) * dim, seed=seed, dtype=dtype, scale=2.0)   # strided as a projection leaves it
    g = torch.Generator().manual_seed(seed + 1)
    rows = 97
    angle = torch.rand((rows, rotated // 2), generator=g) * 6.3
    positions = torch.randint(-1, rows + 1, (tokens,), generator=g, dtype=torch.int32)   # paddings among them
    weights = [(1 + 0.3 * torch.randn(dim, generator=g)).to(F32 if wide else dtype) for _ in range(2)]
    return x, positions, torch.cos(angle), torch.sin(angle), weights


def _views(x, q_heads, k_heads, dim):
    return x[:, :q_heads * dim].view(len(x), q_heads, dim), x[:, q_heads * dim:(q_heads + k_heads) * dim].view(len(x), k_heads, dim)


NORMS = [
    (1, 1, 1, 64, F32, 64, True, False), (1, 1, 0, 256, F16, 256, False, False), (7, 32, 8, 128, BF16, 128, False, False),
    (33, 5, 3, 64, F16, 32, True, True), (130, 3, 1, 256, BF16, 64, True, True), (5, 9, 2, 128, F32, 16, True, False),
    (64, 12, 4, 64, F32, 32, True, True), (4100, 2, 1, 128, F16, 128, False, False), (3, 17, 17, 256, F32, 128, True, False),
    (2051, 4, 2, 64, BF16, 64, True, False),
]


@pytest.mark.parametrize("tokens, q_heads, k_heads, dim, dtype, rotated, wide, interleaved", NORMS)
def test_norm_and_rotation(tokens, q_heads, k_heads, dim, dtype, rotated, wide, interleaved):
    """One rounding of the result, and binary32 arithmetic before it: the sum of `dim` squares, a root and a division, five
    products and sums; a rotated element is the sum of two, whose errors go by the larger one of the pair."""
    x, positions, cos, sin, (qw, kw) = _norm_case(tokens, q_heads, k_heads, dim, dtype, rotated, wide, 11 * tokens + dim)
    q, k = _views(x, q_heads, k_heads, dim)
    dq, dk = _views(x.to(DEV), q_heads, k_heads, dim)
    table = positions.to(DEV), cos.to(DEV), sin.to(DEV)
    got = B.head_norm_rotate(dq, dk if k_heads else None, qw.to(DEV), kw.to(DEV) if k_heads else None, *table, 1e-5, interleaved)
    for y, x1, w in ((got[0], q, qw), (got[1], k, kw)):
        if x1.shape[1] == 0:
            assert y is None
            continue
        want = H.norm_rotate(x1, w, positions, cos, sin, 1e-5, interleaved)
        assert y.dtype == dtype and y.shape == x1.shape and y.is_contiguous()
        n = H.norm_rotate(x1, w, torch.where(positions < 0, 0, positions), torch.ones_like(cos), torch.zeros_like(sin), 1e-5, interleaved)
        bound = H.ROUNDOFF[dtype] * want.abs() + (dim + 16) * 2.0 ** -24 * n.abs().amax(-1, keepdim=True) + 1e-7   # 2^-25: subnormal binary16
        off = (y.cpu().double() - want).abs()
        assert (off <= bound).all(), float((off / bound).max())
        assert (y.cpu()[(positions < 0) | (positions >= cos.shape[0])] == 0).all()


def test_norm_in_place_without_weights_and_of_odd_strides():
    """Heads that start at any element, in place; no weight means ones."""
    dim, heads, tokens = 128, 3, 9
    flat = _randn(tokens * 1000 + 1, seed=5, dtype=F16).to(DEV)
    q = torch.as_strided(flat, (tokens, heads, dim), (1000, dim + 5, 1), 8)
    positions = torch.arange(tokens, dtype=torch.int32)
    angle = torch.rand((tokens, dim // 2), generator=torch.Generator().manual_seed(6))
    before = flat.clone()
    want = H.norm_rotate(q.cpu(), None, positions, torch.cos(angle), torch.sin(angle), 1e-6, False)
    y, none = B.head_norm_rotate(q, None, None, None, positions.to(DEV), torch.cos(angle).to(DEV), torch.sin(angle).to(DEV), q_out=q)
    assert none is None and y is not None and y.data_ptr() == q.data_ptr()
    assert (q.cpu().double() - want).abs().max() <= 2.0 ** -11 * want.abs().max() + 1e-6
    touched = torch.zeros_like(flat, dtype=torch.bool)
    torch.as_strided(touched, (tokens, heads, dim), (1000, dim + 5, 1), 8).fill_(True)
    assert torch.equal(flat[~touched], before[~touched])


def test_norm_of_zeros_and_no_tokens():
    zero = torch.zeros((2, 3, 64), device=DEV)
    table = torch.zeros(2, dtype=torch.int32, device=DEV), torch.ones((1, 32), device=DEV), torch.zeros((1, 32), device=DEV)
    assert (B.head_norm_rotate(zero, None, None, None, *table)[0] == 0).all()
    w = torch.ones(64, device=DEV)
    none = zero[:0]
    assert B.head_norm_rotate(none, none, w, w, table[0][:0], *table[1:])[1].shape == (0, 3, 64)
    gq, gk, qw, kw = B.head_norm_rotate_backward(none, none, none, none, w, w, table[0][:0], *table[1:])
    assert gq.shape == gk.shape == (0, 3, 64) and (qw == 0).all() and (kw == 0).all()


@pytest.mark.parametrize("tokens, q_heads, k_heads, dim, dtype, rotated, wide, interleaved", NORMS)
def test_norm_gradients(tokens, q_heads, k_heads, dim, dtype, rotated, wide, interleaved):
    """As above; a gradient of x is a difference of two terms of up to r |g w|, with r up to 2^6 here and means of `dim` products; a
    weight's gradient adds up one product per token and head, in binary32 along a wavefront's share (at most 160 heads here)."""
    x, positions, cos, sin, (qw, kw) = _norm_case(tokens, q_heads, k_heads, dim, dtype, rotated, wide, 13 * tokens + dim)
    grad = _randn(*x.shape, seed=tokens, dtype=dtype)
    q, k = _views(x, q_heads, k_heads, dim)
    gq, gk = _views(grad, q_heads, k_heads, dim)
    dq, dk = _views(x.to(DEV), q_heads, k_heads, dim)
    dgq, dgk = _views(grad.to(DEV), q_heads, k_heads, dim)
    some = k_heads > 0
    args = (dgq, dgk if some else None, dq, dk if some else None, qw.to(DEV), kw.to(DEV) if some else None, positions.to(DEV), cos.to(DEV), sin.to(DEV), 1e-5, interleaved)
    got = B.head_norm_rotate_backward(*args)
    again = B.head_norm_rotate_backward(*args)
    assert all(a is b or torch.equal(a, b) for a, b in zip(got, again)), "the order of the sums is fixed"
    for gx, gw, g1, x1, w in ((got[0], got[2], gq, q, qw), (got[1], got[3], gk, k, kw)):
        if x1.shape[1] == 0:
            assert gx is None and gw is None
            continue
        want_x, want_w, magnitude = H.norm_rotate_backward(g1, x1, w, positions, cos, sin, 1e-5, interleaved)
        assert gx.dtype == dtype and gw.dtype == w.dtype
        xd = x1.double()
        r = (xd.square().mean(-1, keepdim=True) + 1e-5) ** -0.5
        largest = r * (g1.double().abs().amax(-1, keepdim=True) * 2 * w.double().abs().amax()) * (1 + (xd * r).abs().amax(-1, keepdim=True))
        bound = H.ROUNDOFF[dtype] * want_x.abs() + (dim + 32) * 2.0 ** -24 * largest + 1e-7
        off = (gx.cpu().double() - want_x).abs()
        assert (off <= bound).all(), float((off / bound).max())
        bound = H.ROUNDOFF[w.dtype] * want_w.abs() + (dim + 256) * 2.0 ** -24 * magnitude + 1e-6
        off = (gw.cpu().double() - want_w).abs()
        assert (off <= bound).all(), float((off / bound).max())


def test_norm_gradients_agree_with_differences():
    """<grad, y(x + h d) - y(x - h d)> / 2h against the gradients, in binary32: the difference's error is h^2 of the third
    derivative and 2^-24 / h of the rounding, both below 1e-3 of the sum's size at h = 2^-8."""
    tokens, heads, dim, h = 6, 3, 64, 2.0 ** -8
    x, w = _randn(tokens, heads, dim, seed=1).to(DEV), (1 + _randn(dim, seed=2, scale=0.2)).to(DEV)
    grad, dx, dw = (_randn(tokens, heads, dim, seed=3).to(DEV), _randn(tokens, heads, dim, seed=4).to(DEV), _randn(dim, seed=5).to(DEV))
    angle = torch.rand((tokens, 32), generator=torch.Generator().manual_seed(7)).to(DEV)
    table = torch.arange(tokens, dtype=torch.int32, device=DEV), torch.cos(angle), torch.sin(angle)

    def inner(x1, w1):
        return float((grad.double() * B.head_norm_rotate(x1, None, w1, None, *table)[0].double()).sum())

    gx, _, gw, _ = B.head_norm_rotate_backward(grad, None, x, None, w, None, *table)
    for a, b, g, d in (((x + h * dx, w), (x - h * dx, w), gx, dx), ((x, w + h * dw), (x, w - h * dw), gw, dw)):
        numeric = (inner(*a) - inner(*b)) / (2 * h)
        exact = float((g.double() * d.double()).sum())
        size = float((g.double() * d.double()).abs().sum())
        assert abs(numeric - exact) <= 1e-3 * size, (numeric, exact, size)


# ----------------------------------------------------------------------------- the cache

@pytest.mark.parametrize("tokens, heads, dim, dtype, key_bits, value_bits, page", [
    (1, 1, 64, F32, 8, 8, 16), (5, 3, 128, F16, 4, 4, 16), (77, 8, 128, BF16, 8, 4, 64), (40, 2, 256, F32, 4, 8, 1024), (333, 5, 64, BF16, 4, 4, 32),
    (1000, 1, 256, F16, 8, 8, 128)])
def test_cache_write_and_read(tokens, heads, dim, dtype, key_bits, value_bits, page):
    """Codes and headers bit for bit; what is read back is one fused multiply-add and one rounding from the value they stand for."""
    pages = (tokens + page - 1) // page + 2
    cache = H.make_cache(pages, heads, page, dim, key_bits, value_bits, seed=tokens)
    want = [t.clone() for t in cache]
    both = _randn(tokens, heads, 2, dim, seed=dim + tokens, dtype=dtype, scale=3.0)   # keys and values interleaved by head
    both[0, 0] = 1.25                                       # no range
    if tokens > 4:
        both[1, 0, 0, :] = torch.tensor([1e-40]).to(dtype)  # subnormal
        both[2, 0] *= 1e-3
        both[3, 0, 1] = -0.0
    k, v = both[:, :, 0], both[:, :, 1]
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(3))[:tokens]
    skipped = torch.zeros(tokens, dtype=torch.bool)
    if tokens > 4:
        slots[4], slots[tokens - 1] = -1, pages * page
        skipped[4] = skipped[tokens - 1] = True
    device_both = both.to(DEV)
    B.cache_write(device_both[:, :, 0], device_both[:, :, 1], slots.to(DEV), *cache)
    H.fill(want, slots[~skipped].to(DEV), k[~skipped], v[~skipped], key_bits, value_bits)
    for got, w in zip(cache, want):
        assert torch.equal(got.view(torch.uint8) if got.dtype == torch.uint8 else got.view(torch.int32), w if w.dtype == torch.uint8 else w.view(torch.int32))
    rk, rv = B.cache_read(slots.to(DEV), *cache, dim, dtype)
    block, at = (slots[~skipped] // page).to(DEV), (slots[~skipped] % page).to(DEV)
    for got, codes, header, bits in ((rk, cache[0], cache[1], key_bits), (rv, cache[2], cache[3], value_bits)):
        held = torch.from_numpy(H.values(codes[block, :, at].cpu().numpy(), header[block, :, at].cpu().numpy(), bits))
        got = got.cpu()
        assert got.dtype == dtype and (got[skipped] == 0).all()
        assert ((got[~skipped].double() - held).abs() <= 1.01 * H.ROUNDOFF[dtype] * held.abs() + 2.0 ** -24 * 16 + 1e-7).all()


def test_cache_beyond_32_bits_of_offset():
    """Codes of more than 2^32 bytes: the last page is not the first one's."""
    pages, heads, page, dim = 2 ** 32 // (16 * 64 * 64) + 8, 16, 64, 64
    codes = torch.zeros((pages, heads, page, dim), dtype=torch.uint8, device=DEV)
    header = torch.zeros((pages, heads, page, 2), device=DEV)
    cache = (codes, header, codes.clone(), header.clone())
    tokens = 80
    k, v = (_randn(tokens, heads, dim, seed=s, dtype=F16).to(DEV) for s in (1, 2))
    j = torch.arange(tokens)
    table = torch.tensor([[pages - 2, pages - 1]], dtype=torch.int32)
    slots = (table[0].long()[j // page] * page + j % page).to(DEV)
    B.cache_write(k, v, slots, *cache)
    assert int(codes[:pages - 2].view(-1)[:: 4096].count_nonzero()) == 0 and int(codes[pages - 2:].count_nonzero()) > 0
    rk, _ = B.cache_read(slots, *cache, dim, F16)
    assert (rk - k).abs().max() < 0.05
    q = _randn(3, 16, dim, seed=3, dtype=F16)
    start, lengths = torch.tensor([0, 3], dtype=torch.int32), torch.tensor([tokens], dtype=torch.int32)
    out = B.cache_attention(q.to(DEV), *cache, table.to(DEV), lengths.to(DEV), start.to(DEV), 3, tokens)
    small = [c[pages - 2:] for c in cache]
    want, largest, widest = H.attention(q, *small, table - (pages - 2), lengths, start, dim)
    assert (np.abs(out.cpu().double().numpy() - want) <= H.attention_bound(F16, dim, want, largest, widest, tokens)).all()


# ----------------------------------------------------------------------------- attention

def _attention_case(lengths, news, q_heads, kv, dim, dtype, key_bits, value_bits, page, seed, extra_pages=3, scale_q=1.0):
    """Sequences whose pages lie anywhere; slots that hold no token are garbage with NaN headers."""
    per = max(1, (max(lengths) + page - 1) // page)
    pages = len(lengths) * per + extra_pages
    cache = H.make_cache(pages, kv, page, dim, key_bits, value_bits, seed)
    g = torch.Generator().manual_seed(seed + 1)
    table = torch.randperm(pages, generator=g)[:len(lengths) * per].view(len(lengths), per).int()
    shift = 1.5 * torch.randn((1, kv, dim), generator=g)
    for n, length in enumerate(lengths):
        if length > 0:
            j = torch.arange(length)
            slots = (table[n].long()[j // page] * page + j % page).to(DEV)
            k, v = (torch.randn((length, kv, dim), generator=g) for _ in range(2))
            H.fill(cache, slots, k + shift, v, key_bits, value_bits)
    start = torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32)
    q = (scale_q * torch.randn((int(start[-1]), q_heads, dim), generator=g)).to(dtype)
    return cache, table, torch.tensor(lengths, dtype=torch.int32), start, q


def _check(case, dim, dtype, max_query, max_length, **options):
    cache, table, lengths, start, q = case
    out = B.cache_attention(q.to(DEV), *cache, table.to(DEV), lengths.to(DEV), start.to(DEV), max_query, max_length, **options)
    want, largest, widest = H.attention(q, *cache, table, lengths, start, dim, **options)
    assert out.dtype == dtype and out.shape == q.shape
    bound = H.attention_bound(dtype, dim, want, largest, widest, max_length)
    off = np.abs(out.cpu().double().numpy() - want)
    assert np.isfinite(off).all() and (off <= bound).all(), float((off / bound).max())
    return out


ATTENTIONS = [
    # lengths, new tokens, q heads, kv heads, dim, type, key bits, value bits, page, options
    ([1], [1], 1, 1, 64, F32, 8, 8, 16, {}),
    ([1], [1], 8, 1, 128, F16, 4, 4, 16, {}),
    ([63, 64, 65], [1, 1, 1], 4, 2, 128, BF16, 8, 8, 16, {}),
    ([15, 1, 130, 0, 700], [1, 1, 1, 1, 1], 6, 2, 64, F16, 8, 4, 64, {}),
    ([2000], [1], 32, 8, 128, BF16, 8, 8, 128, {}),
    ([5000, 3], [1, 1], 5, 5, 64, F32, 4, 8, 32, {}),
    ([1111], [1], 16, 1, 256, F16, 8, 8, 16, {}),
    ([900, 33], [1, 1], 6, 2, 256, F32, 4, 4, 1024, {}),
    ([300, 700], [5, 3], 8, 2, 128, F16, 8, 8, 64, {}),
    ([300, 17, 250], [300, 17, 1], 4, 2, 64, BF16, 8, 8, 16, {}),
    ([257], [257], 8, 2, 128, F16, 4, 4, 32, {}),
    ([513, 70], [129, 70], 3, 1, 128, F32, 8, 4, 64, {}),
    ([260], [100], 4, 2, 256, BF16, 4, 8, 64, {}),
    ([200], [64], 4, 2, 256, F32, 8, 8, 16, {}),
    ([1500], [1], 4, 2, 128, F16, 8, 8, 64, dict(window=100)),
    ([1500, 40], [70, 40], 4, 2, 64, F16, 8, 8, 16, dict(window=33)),
    ([800], [90], 4, 1, 128, F32, 8, 8, 64, dict(window=1, softcap=20.0)),
    ([640, 31], [33, 31], 8, 4, 128, BF16, 4, 4, 16, dict(softcap=5.0)),
    ([400], [3], 2, 1, 64, F32, 8, 8, 32, dict(softcap=1.0, scale=2.0)),
    ([400], [200], 2, 2, 64, F16, 8, 8, 32, dict(scale=-0.3)),
    ([400], [20], 2, 2, 64, F16, 8, 8, 32, dict(scale=0.0)),
    ([1000, 1000], [600, 900], 16, 2, 64, F16, 8, 8, 128, {}),
]


@pytest.mark.parametrize("at", range(len(ATTENTIONS)))
def test_attention(at):
    lengths, news, q_heads, kv, dim, dtype, key_bits, value_bits, page, options = ATTENTIONS[at]
    case = _attention_case(lengths, news, q_heads, kv, dim, dtype, key_bits, value_bits, page, seed=100 + at)
    _check(case, dim, dtype, max(news), max(lengths), **options)


@pytest.mark.parametrize("key_bits, value_bits", [(8, 8), (8, 4), (4, 8), (4, 4)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("new", [1, 40])
def test_attention_of_every_kind(key_bits, value_bits, dim, dtype, new):
    case = _attention_case([333], [new], 4, 2, dim, dtype, key_bits, value_bits, 16, seed=dim + key_bits + new)
    _check(case, dim, dtype, new, 333)


@pytest.mark.parametrize("key_bits, value_bits", [(8, 8), (8, 4), (4, 8), (4, 4)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("new, options", [(50, {}), (190, dict(window=70)), (190, dict(softcap=4.0))])
def test_attention_of_every_kind_in_chunks(key_bits, value_bits, dim, dtype, new, options):
    """100 and 380 rows for a head of the cache."""
    case = _attention_case([420], [new], 2, 1, dim, dtype, key_bits, value_bits, 16, seed=dim + key_bits + new)
    _check(case, dim, dtype, new, 420, **options)


@pytest.mark.parametrize("max_query, max_length", [(1, 1), (7, 100), (1000, 30), (2, 1 << 20)])
def test_attention_bounds_that_are_wrong_only_shape_the_launch(max_query, max_length):
    case = _attention_case([700, 33], [61, 2], 4, 2, 128, F16, 8, 8, 16, seed=9)
    _check(case, 128, F16, max_query, max_length)


def test_attention_rows_that_see_nothing_and_sequences_without_rows():
    """More new tokens than tokens: the first rows lie before position zero.  An empty sequence gives zeros, one without new tokens nothing."""
    case = _attention_case([3, 0, 50, 9], [5, 2, 0, 9], 4, 2, 64, F16, 8, 8, 16, seed=10)
    out = _check(case, 64, F16, 9, 50)
    assert (out[:2] == 0).all() and (out[5:7] == 0).all() and (out[2:5] != 0).any()


def test_attention_of_extreme_values():
    """Scores of hundreds, steps of the values from 2^-40 to 2^12 in one sequence, constant groups: one tile's scale must not cost another's."""
    cache, table, lengths, start, q = _attention_case([500], [2], 2, 1, 64, F32, 8, 8, 16, seed=12, scale_q=30.0)
    cache[3][table[0].long()[10:20].to(DEV)] *= 2.0 ** -40
    cache[3][table[0].long()[25].to(DEV)] *= 2.0 ** 12
    cache[3][table[0].long()[3].to(DEV), ..., 1] = 0.0
    cache[1][table[0].long()[5].to(DEV), ..., 1] = 0.0
    _check((cache, table, lengths, start, q), 64, F32, 2, 500)
    _check((cache, table, lengths, start, (q * 1e-30).float()), 64, F32, 2, 500)
    _check((cache, table, lengths, start, (q * 1e-3).to(BF16)), 64, BF16, 2, 500)


def test_attention_does_not_look_past_a_window():
    """Keys that no row sees may hold infinities and NaN."""
    cache, table, lengths, start, q = _attention_case([640], [40], 4, 2, 128, F16, 8, 8, 64, seed=14)
    clean = _check((cache, table, lengths, start, q), 128, F16, 40, 640, window=50)
    first = 640 - 40 - 50 + 1
    for page in range(first // 64):
        for header in (cache[1], cache[3]):
            header[table[0, page].long()] = float("inf") if page % 2 else float("nan")
    inside = table[0, first // 64].long()
    for header in (cache[1], cache[3]):
        header[inside, :, : first % 64] = float("nan")
    args = (table.to(DEV), lengths.to(DEV), start.to(DEV), 40, 640)
    assert torch.equal(B.cache_attention(q.to(DEV), *cache, *args, window=50), clean)


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_attention_of_earlier_tokens_of_a_chunk_does_not_depend_on_later_ones(dtype, bad):
    """The same for 120 rows."""
    cache, table, lengths, start, q = _attention_case([300], [60], 2, 1, 128, dtype, 8, 8, 16, seed=20)
    args = (table.to(DEV), lengths.to(DEV), start.to(DEV), 60, 300)
    clean = B.cache_attention(q.to(DEV), *cache, *args)
    for at in (290, 296, 299):
        for header in (cache[1], cache[3]):
            header[table[0, at // 16].long(), :, at % 16] = bad
    out = B.cache_attention(q.to(DEV), *cache, *args)
    assert torch.equal(out[:50], clean[:50]) and not torch.isfinite(out[50:]).any()


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_attention_of_earlier_tokens_does_not_depend_on_later_ones(dtype, bad):
    """The last tokens' keys and values are infinite or NaN: rows before them give what they gave."""
    cache, table, lengths, start, q = _attention_case([300], [60], 4, 2, 64, dtype, 8, 8, 16, seed=18)
    args = (table.to(DEV), lengths.to(DEV), start.to(DEV), 60, 300)
    clean = B.cache_attention(q.to(DEV), *cache, *args)
    for at in (290, 296, 299):
        for header in (cache[1], cache[3]):
            header[table[0, at // 16].long(), :, at % 16] = bad
    out = B.cache_attention(q.to(DEV), *cache, *args)
    first = 60 - 10
    assert torch.equal(out[:first], clean[:first]) and not torch.isfinite(out[first:]).any()


def test_attention_of_strided_queries_into_a_strided_output_on_another_stream():
    cache, table, lengths, start, q = _attention_case([90, 700], [4, 30], 4, 2, 128, BF16, 8, 8, 32, seed=15)
    packed = torch.zeros((q.shape[0], 3, 4, 131), dtype=BF16, device=DEV)
    view = packed[:, 1, :, 1:129]
    view.copy_(q)
    into = torch.full((q.shape[0], 4, 200), 7.0, dtype=BF16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = B.cache_attention(view, *cache, table.to(DEV), lengths.to(DEV), start.to(DEV), 30, 700, out=into[..., 3:131])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert out.data_ptr() == into[..., 3:].data_ptr()
    assert (into[..., :3] == 7).all() and (into[..., 131:] == 7).all()
    want, largest, widest = H.attention(q, *cache, table, lengths, start, 128)
    assert (np.abs(out.cpu().double().numpy() - want) <= H.attention_bound(BF16, 128, want, largest, widest, 700)).all()


def test_attention_is_the_same_every_time_and_in_a_graph():
    cache, table, lengths, start, q = _attention_case([3000, 100], [1, 1], 8, 2, 128, F16, 4, 4, 64, seed=16)
    args = [q.to(DEV), *cache, table.to(DEV), lengths.to(DEV), start.to(DEV)]
    eager = B.cache_attention(*args, 1, 3000)
    out = torch.empty_like(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.cache_attention(*args, 1, 3000, out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cache_attention(*args, 1, 3000, out=out)
    for length in (3000, 17, 1024):
        args[6].copy_(torch.tensor([length, 100], dtype=torch.int32))
        want = B.cache_attention(*args, 1, 3000)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), length
    args[6].copy_(lengths)
    assert torch.equal(B.cache_attention(*args, 1, 3000), eager)


@pytest.mark.parametrize("new, length, sequences", [(1, 6000, 24), (40, 1500, 6)])
def test_attention_of_many_workgroups_is_the_same_every_time(new, length, sequences):
    """Workgroups that share a compute unit run at different paces: what they exchange inside must not depend on it."""
    lengths = [length - 137 * i for i in range(sequences)]
    case = _attention_case(lengths, [new] * sequences, 32, 8, 128, F16, 4, 4, 64, seed=19)
    cache, table, lengths, start, q = case
    args = [q.to(DEV), *cache, table.to(DEV), lengths.to(DEV), start.to(DEV), new, length]
    first = B.cache_attention(*args)
    for _ in range(8):
        assert torch.equal(B.cache_attention(*args), first)


def test_attention_without_tokens_or_sequences():
    cache, table, lengths, start, q = _attention_case([30], [3], 4, 2, 64, F16, 8, 8, 16, seed=17)
    args = (table.to(DEV), lengths.to(DEV), start.to(DEV), 3, 30)
    assert B.cache_attention(q[:0].to(DEV), *cache, *args).shape == (0, 4, 64)
    none = B.cache_attention(q[:0].to(DEV), *cache, table[:0].to(DEV), lengths[:0].to(DEV), start[:1].to(DEV), 0, 0)
    assert none.shape == (0, 4, 64)


# ----------------------------------------------------------------------------- refusals of the binding

def test_tensors_that_do_not_fit_are_refused():
    q, k = torch.zeros((3, 4, 64), device=DEV), torch.zeros((3, 2, 64), device=DEV)
    i, t = torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros((5, 32), device=DEV)
    w = torch.ones(64, device=DEV)
    ok = [q, k, w, w, i, t, t]
    B.head_norm_rotate(*ok)
    for at, bad, error in ((0, q[0], ValueError), (0, q.double(), TypeError), (0, q.transpose(1, 2), ValueError), (1, k[:2], ValueError), (1, k.half(), TypeError),
                           (2, w[:32], ValueError), (2, w.half(), TypeError), (4, i.long(), TypeError), (4, i[:2], ValueError), (5, t[:, :16], ValueError),
                           (5, t.double(), TypeError), (6, t.cpu(), ValueError), (0, q.cpu(), ValueError)):
        args = list(ok)
        args[at] = bad
        with pytest.raises(error):
            B.head_norm_rotate(*args)
    with pytest.raises(ValueError, match="expanded"):
        B.head_norm_rotate(*ok, q_out=torch.zeros((3, 1, 64), device=DEV).expand(3, 4, 64))
    with pytest.raises(B.ActqError, match="eps"):
        B.head_norm_rotate(*ok, eps=0.0)
    with pytest.raises(ValueError, match="grad_k"):
        B.head_norm_rotate_backward(q, None, *ok)
    cache = H.make_cache(4, 2, 16, 64, 8, 4, 0, poison=False)
    slots = torch.arange(3, device=DEV)
    B.cache_write(k, k, slots, *cache)
    for args, error in (((k, k[:2], slots, *cache), ValueError), ((k, k.half(), slots, *cache), TypeError), ((k, k, slots.int(), *cache), TypeError), ((q, q, slots, *cache), B.ActqError),
                        ((k, k, slots, cache[0][:2], *cache[1:]), ValueError), ((k, k, slots, cache[0][..., :8], *cache[1:]), ValueError),
                        ((k, k, slots, cache[0], cache[1].half(), *cache[2:]), TypeError)):
        with pytest.raises(error):
            B.cache_write(*args)
    with pytest.raises(TypeError):
        B.cache_read(slots, *cache, 64, torch.int32)
    with pytest.raises(ValueError):
        B.cache_read(slots, *cache, 64, torch.float32, k=torch.zeros((2, 2, 64), device=DEV))
    table, lengths, start = i.view(3, 1), i, torch.zeros(4, dtype=torch.int32, device=DEV)
    ok = [q, *cache, table, lengths, start, 1, 16]
    B.cache_attention(*ok)
    for at, bad, error in ((0, q[..., :32], ValueError), (5, table.long(), TypeError), (5, table[:2], ValueError), (7, start[:3], ValueError), (6, lengths.cpu(), ValueError),
                           (8, -1, B.ActqError), (0, q[:, :3], B.ActqError)):
        args = list(ok)
        args[at] = bad
        with pytest.raises(error):
            B.cache_attention(*args)
    for options in (dict(window=-1), dict(softcap=-1.0), dict(scale=float("inf")), dict(out=torch.zeros((3, 4, 64), dtype=F16, device=DEV))):
        with pytest.raises((ValueError, TypeError, B.ActqError)):
            B.cache_attention(*ok, **options)
