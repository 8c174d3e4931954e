"""Every row of the attention by itself: against its own bound, and unmoved by what other rows of a tile hold."""
import numpy as np
import pytest
import torch

import _attention_rows as R
import _heads as H
from paper_2104_14129_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _case(lengths, news, q_heads, kv, dim, dtype, key_bits=8, value_bits=8, page=16, seed=0):
    """Sequences whose pages lie anywhere, garbage with NaN headers in the slots that hold no token."""
    per = (max(lengths) + page - 1) // page
    pages = len(lengths) * per + 2
    cache = H.make_cache(pages, kv, page, dim, key_bits, value_bits, seed)
    g = torch.Generator().manual_seed(seed + 1)
    table = torch.randperm(pages, generator=g)[:len(lengths) * per].view(len(lengths), per).int()
    for n, length in enumerate(lengths):
        j = torch.arange(length)
        k, v = (torch.randn((length, kv, dim), generator=g) for _ in range(2))
        H.fill(cache, (table[n].long()[j // page] * page + j % page).to(DEV), k + 1.5 * torch.randn((1, kv, dim), generator=g), v, key_bits, value_bits)
    start = torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32)
    return torch.randn((int(start[-1]), q_heads, dim), generator=g).to(dtype), cache, table, torch.tensor(lengths, dtype=torch.int32), start, dim


def _attend(case, max_query=0, **options):
    q, cache, table, lengths, start, _ = case
    return B.cache_attention(q.to(DEV), *cache, table.to(DEV), lengths.to(DEV), start.to(DEV), max(max_query, int(start.diff().max())), int(lengths.max()), **options)


def _within(out, case, **options):
    want, bound = R.attention(*case, **options)
    off = np.abs(out.cpu().double().numpy() - want)
    assert (off <= bound).all(), float((off / np.maximum(bound, 1e-300)).max())


SHAPES = [
    # new tokens of 300, q heads, kv heads, dim, key bits, value bits: 6 rows, 80, and 104 and 300 for the kernel of many rows; heads of 256 in both
    (3, 4, 2, 64, 8, 8), (40, 4, 2, 128, 4, 8), (52, 2, 1, 128, 8, 8), (150, 4, 2, 64, 8, 4), (5, 2, 1, 256, 8, 4), (170, 2, 1, 256, 4, 4),
]


@pytest.mark.parametrize("options", [{}, dict(softcap=5.0), dict(window=30)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("at", range(len(SHAPES)))
def test_rows_keep_to_their_own_bound(at, dtype, options):
    new, q_heads, kv, dim, key_bits, value_bits = SHAPES[at]
    case = _case([300], [new], q_heads, kv, dim, dtype, key_bits, value_bits, seed=at)
    _within(_attend(case, **options), case, **options)


@pytest.mark.parametrize("new", [1, 60])
def test_binary32_is_held_in_two_numbers_of_binary16_in_every_row(new):
    """Thousands of rows over few keys, where a single weight of which only one number counts shows."""
    case = _case([64] * 24, [new] * 24, 4, 2, 64, F32, seed=60 + new)
    _within(_attend(case), case)


@pytest.mark.parametrize("options", [{}, dict(softcap=5.0), dict(window=30)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("at", range(len(SHAPES)))
def test_a_row_of_q_that_is_not_finite_or_large_leaves_the_others_as_they_were(at, dtype, options):
    """One element of one token's head: the row itself is NaN where it is no finite number, every other row is what it was, bit for bit."""
    new, q_heads, kv, dim, key_bits, value_bits = SHAPES[at]
    case = _case([300], [new], q_heads, kv, dim, dtype, key_bits, value_bits, seed=at)
    clean = _attend(case, **options)
    q = case[0]
    for token, head, element, value in ((new - 1, 0, 5, float("inf")), (new // 2, q_heads - 1, dim - 1, float("-inf")), (0, 1, 0, float("nan")), (new - 1, q_heads - 1, 3, 2.0 ** (15 if dtype == F16 else 40))):
        changed = q.clone()
        changed[token, head, element] = value
        out = _attend((changed, *case[1:]), **options)
        if np.isfinite(value):
            assert torch.isfinite(out[token, head]).all()
        else:
            assert torch.isnan(out[token, head]).all()
        out[token, head] = clean[token, head]
        assert torch.equal(out, clean), (token, head, value)


@pytest.mark.parametrize("new", [2, 60])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_very_different_sizes(new, dtype):
    """Rows of 2^-30 to 2^3 and zeros side by side: each keeps to its own bound."""
    q, *rest = case = _case([200], [new], 4, 2, 64, dtype, seed=40)
    sizes = torch.tensor([2.0 ** -30, 1.0, 0.0, 8.0, 2.0 ** -12]).repeat(q.shape[0] * 4)[:q.shape[0] * 4].view(q.shape[0], 4, 1)
    case = ((q.float() * sizes).to(dtype), *rest)
    for options in ({}, dict(softcap=3.0)):
        _within(_attend(case, **options), case, **options)


def test_rows_before_the_first_position_are_zeros_whatever_they_hold():
    q, *rest = _case([3], [5], 2, 1, 64, F16, seed=41)
    q[0] = float("inf")
    q[1] = float("nan")
    assert (_attend((q, *rest))[:2] == 0).all()


@pytest.mark.parametrize("ratio", [12, 20, 40])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("at", range(len(SHAPES)))
def test_values_that_only_later_rows_see_leave_the_earlier_ones_as_they_were(at, dtype, ratio):
    """The last two tokens' values are 2^ratio times larger: rows before them are what they were, bit for bit, and every row keeps to its own bound."""
    new, q_heads, kv, dim, key_bits, value_bits = SHAPES[at]
    q, cache, table, *rest = case = _case([300], [new], q_heads, kv, dim, dtype, key_bits, value_bits, seed=at)
    clean = _attend(case)
    for j in (298, 299):
        cache[3][table[0, j // 16].long(), :, j % 16] *= 2.0 ** ratio
    out = _attend(case)
    assert torch.equal(out[:-2], clean[:-2])
    if dtype != F16:   # the last rows' outputs are beyond binary16
        _within(out, case)


@pytest.mark.parametrize("ratio", [20, 30])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("new, dim", [(1, 64), (1, 128), (1, 256), (130, 128), (130, 64), (330, 256)])
def test_a_large_value_of_no_weight_takes_no_bits_from_the_others(new, dim, dtype, ratio):
    """One key's scores lie some 60 below the others (its weight is about e^-60) while its values are 2^ratio times theirs."""
    q, cache, table, *rest = case = _case([400], [new], 1, 1, dim, dtype, seed=70)
    q[:, 0] = q[:, 0].abs()
    block, j = table[0, 7 // 16].long(), 7
    cache[1][block, 0, j] = torch.tensor([-60.0 * dim ** 0.5 / (0.8 * dim), 0.0])
    cache[3][block, 0, j] *= 2.0 ** ratio
    _within(_attend(case), case)


@pytest.mark.parametrize("new, dim", [(1, 64), (1, 128), (130, 64), (330, 256)])
@pytest.mark.parametrize("factor", [-100, -60, 60, 100])
def test_values_of_any_size(new, dim, factor):
    """Half of a sequence's values, or all of them, are 2^factor times the others: binary32's range of steps on both sides."""
    for some in (slice(0, 7), slice(0, None)):
        q, cache, table, *rest = case = _case([400], [new], 2, 1, dim, F32, seed=71)
        cache[3][table[0, some].long()] *= 2.0 ** factor
        _within(_attend(case), case)


@pytest.mark.parametrize("softcap", [1e-39, 1e-30, 0.01, 1.0, 30.0, 1e3, 1e4, 1e6, 1e12, 3e38])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("new, dim", [(1, 64), (2, 128), (130, 64), (330, 256)])
def test_caps_of_any_size(new, dim, dtype, softcap):
    """Scores of up to some tens under caps that hold nearly all of them, some, or none: the cap's own error is that of the score."""
    q, *rest = _case([340], [new], 2, 1, dim, dtype, seed=80)
    case = (q * 4, *rest)
    _within(_attend(case, softcap=softcap), case, softcap=softcap)


@pytest.mark.parametrize("lengths, q_heads, dim, dtype, options", [
    ([16384], 1, 256, F16, {}),                     # 128 parts, all with keys
    ([16384, 300], 2, 256, F32, {}),                # the second sequence has keys in three of them
    ([16384], 4, 128, BF16, {}),                    # 64
    ([16384, 129, 5000], 1, 128, F32, {}),
    ([9000, 1], 3, 128, F16, dict(window=6000)),    # parts before the window see nothing
    ([16384, 77], 2, 64, F32, dict(softcap=5.0)),
    ([4200], 1, 256, BF16, {}),                     # 33
])
def test_one_token_over_many_parts_that_are_joined(lengths, q_heads, dim, dtype, options):
    case = _case(lengths, [1] * len(lengths), q_heads, 1, dim, dtype, page=64, seed=90 + dim)
    _within(_attend(case, **options), case, **options)


@pytest.mark.parametrize("key_bits, value_bits", [(8, 8), (8, 4), (4, 8), (4, 4)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("new, options", [(50, {}), (190, dict(window=70)), (190, dict(softcap=4.0)), (9, {})])
def test_heads_of_64_by_the_kernel_for_many_rows(new, options, dtype, key_bits, value_bits):
    """It takes heads of 64 where workgroups are many; a most number of new tokens that is not reached makes them so.  Both kernels keep to the bound, and
    what one row holds stays out of the others in this one too."""
    q, cache, table, *rest = case = _case([420, 33], [new, 7], 4, 2, 64, dtype, key_bits, value_bits, seed=100)
    out = _attend(case, max_query=4000, **options)
    _within(out, case, **options)
    _within(_attend(case, **options), case, **options)
    changed = q.clone()
    changed[new - 1, 0, 3] = float("inf")
    cache[3][table[0, 419 // 16].long(), :, 419 % 16] *= 2.0 ** 20
    again = _attend((changed, cache, table, *rest), max_query=4000, **options)
    assert torch.isnan(again[new - 1, 0]).all() and torch.equal(again[:new - 1], out[:new - 1]) and torch.equal(again[new:], out[new:])


@pytest.mark.parametrize("key_bits, value_bits", [(8, 8), (4, 4)])
@pytest.mark.parametrize("options", [{}, dict(window=20, softcap=4.0)])
def test_binary32_in_heads_of_256_by_the_kernel_for_many_rows(options, key_bits, value_bits):
    """It takes them where sequences and heads of the cache are more than 64."""
    case = _case([40 - n for n in range(33)], [36 - n for n in range(33)], 4, 2, 256, F32, key_bits, value_bits, seed=101)
    _within(_attend(case, **options), case, **options)


@pytest.mark.parametrize("lengths, news, max_query", [([1], [1], 0), ([2, 1, 3], [1, 1, 1], 0), ([15], [15], 0), ([100, 41], [1, 1], 0), ([1000], [3], 0), ([120], [120], 4000), ([60], [60], 0)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_16_bit_result_over_few_keys_is_off_by_its_own_rounding(dtype, dim, lengths, news, max_query):
    """The error is that of rounding the definition's result once, and 5 % for everything before that: a weight held in one binary16 number would add a half
    to a binary16 result's, and 1 to 3 % (a 64th of the squares, at most 2.5 times that over one key) to a bfloat16 one's."""
    case = _case(lengths, news, 8, 4, dim, dtype, seed=110)
    want = torch.from_numpy(R.attention(*case)[0])
    off = (_attend(case, max_query=max_query).cpu().double() - want).norm()
    assert float(off / (want.to(dtype).double() - want).norm()) < 1.05


@pytest.mark.parametrize("new, dim", [(1, 64), (130, 128), (330, 256)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [-95, 60])
def test_queries_of_any_size_under_a_scale_that_makes_up_for_it(new, dim, dtype, size):
    """Powers of two on both sides: the scores, and so the outputs, are those of ordinary queries."""
    q, *rest = case = _case([340], [new], 2, 1, dim, dtype, seed=120)
    want = _attend(case)
    out = _attend(((q.float() * 2.0 ** size).to(dtype), *rest), scale=dim ** -0.5 * 2.0 ** -size)
    assert torch.equal(out, want)


@pytest.mark.parametrize("key_bits, value_bits", [(8, 4), (4, 4), (8, 8)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("seed", range(8))
def test_columns_that_the_heaviest_key_leaves_alone(seed, dtype, key_bits, value_bits):
    """Steps from 2^-12 to 2^12 of their size: in a column where the heaviest key's code is the middle one, the others' small values count.  A matrix
    instruction's sum of bytes as they lie is off by 2^-19 of the largest product at worst, of nibbles by 2^-16, and a block of 64 keys takes two."""
    q, cache, table, *rest = case = _case([16, 15, 64, 33], [1, 15, 2, 5], 4, 2, 64, dtype, key_bits, value_bits, seed=seed)
    g = torch.Generator().manual_seed(seed)
    cache[3].mul_(torch.exp2(torch.randint(-12, 12, cache[3].shape[:3], generator=g)).to(DEV)[..., None])
    want, bound = R.attention(*case)
    for token, head, ((kc, kz, ks, _), (_, _, vs, _)) in R._rows(q.double().numpy(), cache, table, *rest[:2], 64, 0):
        s = (kz + ks * kc) @ q[token, head].double().numpy() / 8
        p = np.exp(s - s.max())
        bound[token, head] += 2.0 ** (-15 if value_bits == 4 else -18) * (p / p.sum() * vs[:, 0]).max() * (2 ** value_bits - 1)
    off = np.abs(_attend(case).cpu().double().numpy() - want)
    fits = np.abs(want) < (6e4 if dtype == F16 else 1e38)
    assert (off <= bound)[fits].all(), float((off / bound)[fits].max())
