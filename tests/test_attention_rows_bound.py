"""The bound that the attention kernels are held to, on the CPU: the kernels' arithmetic keeps to it, and what it is there to catch does not."""
import numpy as np
import pytest
import torch

import _attention_rows as R
import _heads as H

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _case(lengths, news, q_heads, kv, dim, dtype, key_bits, value_bits, seed, page=16):
    per = (max(lengths) + page - 1) // page
    cache = H.make_cache(len(lengths) * per, kv, page, dim, key_bits, value_bits, seed, device="cpu")
    g = torch.Generator().manual_seed(seed + 1)
    table = torch.randperm(len(lengths) * per, generator=g).view(len(lengths), per).int()
    for n, length in enumerate(lengths):
        j = torch.arange(length)
        k, v = (torch.randn((length, kv, dim), generator=g) for _ in range(2))
        H.fill(cache, table[n].long()[j // page] * page + j % page, k + 1.5 * torch.randn((1, kv, dim), generator=g), v, key_bits, value_bits)
    start = torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32)
    return torch.randn((int(start[-1]), q_heads, dim), generator=g).to(dtype), cache, table, torch.tensor(lengths), start, dim


SHAPES = [([1], [1], 2, 1, 64, 8, 8), ([40, 3], [40, 3], 4, 2, 64, 8, 8), ([300], [5], 2, 1, 128, 8, 8), ([257], [30], 2, 1, 128, 4, 4), ([90], [20], 2, 2, 256, 8, 4), ([1500], [1], 4, 1, 64, 4, 8)]


def _off(got, want, bound):
    return float((np.abs(got.double().numpy() - want) / np.maximum(bound, 1e-300)).max())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("options", [{}, dict(softcap=5.0), dict(window=20)])
@pytest.mark.parametrize("at", range(len(SHAPES)))
def test_the_bound_admits_the_arithmetic_and_not_zeros(at, options, dtype):
    lengths, news, q_heads, kv, dim, key_bits, value_bits = SHAPES[at]
    case = _case(lengths, news, q_heads, kv, dim, dtype, key_bits, value_bits, seed=at)
    want, bound = R.attention(*case, **options)
    assert _off(R.modelled(*case, **options), want, bound) <= 1
    zeros = np.abs(want) > bound
    assert zeros.mean() > 0.9 and zeros.any(-1).all(), "zeros pass for a row"


@pytest.mark.parametrize("at", range(1, len(SHAPES)))   # over one key the scores do not matter, and its weight is scaled to a power of two
def test_the_bound_of_binary32_does_not_admit_single_binary16_numbers(at):
    lengths, news, q_heads, kv, dim, key_bits, value_bits = SHAPES[at]
    case = _case(lengths, news, q_heads, kv, dim, F32, key_bits, value_bits, seed=at)
    want, bound = R.attention(*case)
    assert _off(R.modelled(*case, weight_parts=1), want, bound) > 1
    assert _off(R.modelled(*case, q_parts=1), want, bound) > 1


def test_the_bound_belongs_to_the_row():
    """Values 2^20 times larger that only the last row sees leave the other rows' bounds as they are."""
    q, cache, table, lengths, start, dim = _case([60], [10], 2, 1, 64, F32, 8, 8, seed=3)
    _, clean = R.attention(q, cache, table, lengths, start, dim)
    cache[3][table[0, 59 // 16].long(), :, 59 % 16] *= 2.0 ** 20
    _, bound = R.attention(q, cache, table, lengths, start, dim)
    assert np.array_equal(bound[:-1], clean[:-1]) and (bound[-1] > clean[-1]).all()
