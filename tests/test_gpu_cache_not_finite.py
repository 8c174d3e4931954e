"""Keys and values that are no finite numbers, written into a cache: their groups read as NaN, and nothing else changes."""
import pytest
import torch

import _heads as H
from paper_2104_14129_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("key_bits, value_bits", [(8, 8), (4, 8), (8, 4)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_groups_that_are_not_finite_read_as_nan(dtype, dim, key_bits, value_bits):
    tokens, heads, page, pages = 23, 3, 16, 3
    g = torch.Generator().manual_seed(dim)
    k, v = (torch.randn((tokens, heads, dim), generator=g).to(dtype) for _ in range(2))
    clean = k.clone(), v.clone()
    bad = torch.zeros((2, tokens, heads), dtype=torch.bool)
    marks = [(0, [(0, NAN)]), (1, [(dim - 1, NAN)]), (2, [(7, INF)]), (3, [(8, -INF)]), (4, [(3, INF), (dim - 5, -INF)]), (5, [(9, NAN), (9 + dim // 2, INF)]),
             (6, [(i, NAN) for i in range(dim)]), (7, [(i, INF) for i in range(dim)]), (8, [(i, -INF) for i in range(dim)]), (9, [(i, NAN) for i in range(8)])]
    if dtype != torch.float16:   # a range beyond binary32
        marks.append((10, [(1, 3e38), (20, -3e38)]))
    for at, places in marks:
        for which, x in ((0, k), (1, v)):
            token, head = at + which, (at + which) % heads
            for element, value in places:
                x[token, head, element] = value
            bad[which, token, head] = True
    cache, want = (H.make_cache(pages, heads, page, dim, key_bits, value_bits, 1, poison=False) for _ in range(2))
    slots = torch.randperm(pages * page, generator=g)[:tokens].to(DEV)
    B.cache_write(k.to(DEV), v.to(DEV), slots, *cache)
    H.fill(want, slots, *clean, key_bits, value_bits)
    for which, x in enumerate(B.cache_read(slots, *cache, dim, dtype)):
        x = x.cpu()
        assert torch.isnan(x[bad[which]]).all() and torch.isfinite(x[~bad[which]]).all()
        codes, header = ((t[slots // page, :, slots % page]).cpu() for t in cache[2 * which:2 * which + 2])
        assert torch.isnan(header[bad[which]]).all() and (codes[bad[which]] == 0).all()
        for got, right in zip((codes, header), want[2 * which:2 * which + 2]):
            assert torch.equal(got[~bad[which]], right[slots // page, :, slots % page].cpu()[~bad[which]])


@pytest.mark.parametrize("of", ["keys", "values"])
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("options", [{}, dict(softcap=5.0)])
@pytest.mark.parametrize("value", [INF, NAN])
def test_rows_that_see_one_are_nan(of, new, options, value):
    """A token written with one element that is no number: rows from it on are NaN in the heads that read its group, the others are what they were."""
    tokens, dim, page = 120, 64, 16
    k, v, q = (torch.randn((tokens, h, dim), generator=torch.Generator().manual_seed(s)).to(DEV) for s, h in ((1, 2), (2, 2), (3, 4)))
    slots = torch.arange(tokens, device=DEV)
    table = torch.arange(8, dtype=torch.int32, device=DEV).view(1, 8)
    lengths, start = (torch.tensor(t, dtype=torch.int32, device=DEV) for t in ([tokens], [0, new]))
    cache = H.make_cache(8, 2, page, dim, 8, 8, 2)
    B.cache_write(k, v, slots, *cache)
    args = (q[-new:], *cache, table, lengths, start, new, tokens)
    clean = B.cache_attention(*args, **options)
    at = tokens - 1 - new // 2
    (k if of == "keys" else v)[at, 1, 5] = value
    B.cache_write(k[at:at + 1], v[at:at + 1], slots[at:at + 1], *cache)
    out = B.cache_attention(*args, **options)
    first = at - (tokens - new)   # the row at the token's own position
    assert torch.equal(out[:first], clean[:first]) and torch.equal(out[:, :2], clean[:, :2])
    assert torch.isnan(out[first:, 2:]).all()
