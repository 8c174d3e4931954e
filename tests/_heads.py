"""The operators for attention heads from their definitions, in 64 bits and without the library: norm with rotation and its
gradient, the cache's quantizer, attention over pages."""
from __future__ import annotations

import numpy as np
import torch

ROUNDOFF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # of one rounding to nearest


def rotate(x, positions, cos, sin, interleaved, back=False):
    """Pairs of the first elements turned by their angles; tokens whose position is no row give zeros."""
    rows, half = cos.shape
    inside = (positions >= 0) & (positions < rows)
    at = torch.where(inside, positions, 0).long()
    c, s = cos.double()[at][:, None], sin.double()[at][:, None] * (-1 if back else 1)
    y = x.clone()
    i = torch.arange(half) * 2 if interleaved else torch.arange(half)
    j = i + 1 if interleaved else i + half
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return torch.where(inside[:, None, None], y, 0.0)


def norm_rotate(x, weight, positions, cos, sin, eps, interleaved):
    x = x.double()
    r = (x.square().mean(-1, keepdim=True) + eps) ** -0.5
    n = x * r * (1.0 if weight is None else weight.double())
    return rotate(n, positions, cos, sin, interleaved)


def norm_rotate_backward(grad, x, weight, positions, cos, sin, eps, interleaved):
    """(grad_x, grad_weight, sum of the magnitudes that grad_weight adds up)."""
    x, w = x.double(), 1.0 if weight is None else weight.double()
    g = rotate(grad.double(), positions, cos, sin, interleaved, back=True)
    r = (x.square().mean(-1, keepdim=True) + eps) ** -0.5
    grad_x = r * (g * w - x * r * r * (g * w * x).mean(-1, keepdim=True))
    return grad_x, (g * x * r).sum((0, 1)), (g * x * r).abs().sum((0, 1))


def quantise(x, bits):
    """(codes uint8, header float32 [..., 2]) of the groups along the last axis, in binary32 as the format says, by numpy."""
    x = np.asarray(x, dtype=np.float32)
    top = np.float32(2 ** bits - 1)
    zero = x.min(-1, keepdims=True) + np.float32(0)
    extent = x.max(-1, keepdims=True) - zero
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        inverse, step = top / extent, extent / top
    flat = (extent == 0) | np.isinf(inverse)
    inverse, step = np.where(flat, np.float32(0), inverse), np.where(flat, np.float32(0), step)
    u = np.minimum((x - zero) * inverse, top)
    return np.rint(u).astype(np.uint8), np.concatenate((zero, step), -1).astype(np.float32)


def pack(codes, bits):
    return codes if bits == 8 else codes[..., 0::2] | codes[..., 1::2] << 4


def unpack(stream, bits):
    stream = np.asarray(stream)
    return stream if bits == 8 else np.stack((stream & 15, stream >> 4), -1).reshape(*stream.shape[:-1], -1)


def values(stream, header, bits):
    header = np.asarray(header, dtype=np.float64)
    return unpack(stream, bits) * header[..., 1:] + header[..., :1]


def attention(q, key_codes, key_header, value_codes, value_header, table, lengths, query_start, dim, scale=None, softcap=0.0, window=0):
    """(out float64 [tokens, heads, dim], largest magnitude of a score, largest extent of the values of a group) on the host."""
    q = q.double().cpu().numpy()
    page, kv = key_codes.shape[2], key_codes.shape[1]
    bits = [8 if c.shape[3] == dim else 4 for c in (key_codes, value_codes)]
    keys = values(key_codes.cpu().numpy(), key_header.cpu().numpy(), bits[0])
    vals = values(value_codes.cpu().numpy(), value_header.cpu().numpy(), bits[1])
    extent = value_header[..., 1].double().cpu().numpy() * (2 ** bits[1] - 1)
    table, group = table.cpu().numpy(), q.shape[1] // kv
    scale = dim ** -0.5 if scale is None else scale
    out, largest, widest = np.zeros(q.shape), 0.0, 0.0
    start = query_start.tolist()
    for n, length in enumerate(lengths.tolist()):
        count = start[n + 1] - start[n]
        if count == 0 or length <= 0:
            continue
        j = np.arange(length)
        rows = table[n][j // page], j % page
        position = length - count + np.arange(count)[:, None]
        seen = j <= position
        if window:
            seen &= j > position - window
        for h in range(q.shape[1]):
            k, v = keys[rows[0], h // group, rows[1]], vals[rows[0], h // group, rows[1]]
            at = seen.any(0)
            s = q[start[n]:start[n + 1], h] @ k[at].T * scale
            if softcap:
                s = softcap * np.tanh(s / softcap)
            some = seen.any(1)
            if not some.any():
                continue
            largest = max(largest, float(np.abs(s[seen[:, at]]).max()))
            widest = max(widest, float(extent[rows[0], h // group, rows[1]][at].max()))
            s = np.where(seen[:, at], s, -np.inf)[some]
            p = np.exp(s - s.max(1, keepdims=True))
            out[start[n]:start[n + 1], h][some] = p @ v[at] / p.sum(1, keepdims=True)
    return out, largest, widest


def attention_bound(dtype, dim, out, largest, widest, keys_in_sight):
    """How far a correct kernel may be from the definition.  The result's own rounding; the weights p * step, rounded to binary16 (to
    two numbers of it, 22 bits, for binary32), times centred codes of at most half a group's extent; and scores off by e, which change a
    weight by its share e and so the result by at most 2 e times the spread of the values.  e: the sum of `dim` products in
    binary32 (each step rounded; the products themselves are exact for 16-bit types), the exponential and tanh, 2^-20 of the
    largest score and at least 2^-20."""
    fine = dtype == torch.float32
    weight = 2.0 ** -21 if fine else 2.0 ** -11
    scores = (dim + 16) * 2.0 ** -24 * max(largest, 1.0) * 4
    sums = 2.0 ** -24 * max(keys_in_sight, 1) ** 0.5 * 8
    return ROUNDOFF[dtype] * np.abs(out) + widest * (0.5 * weight + 2 * scores + sums) + sums * np.abs(out) + 1e-7


def make_cache(pages, heads, page, dim, key_bits, value_bits, seed, device="cuda:0", poison=True):
    """A cache whose every slot holds garbage: random codes, headers NaN (or finite ones)."""
    g = torch.Generator().manual_seed(seed)
    made = []
    for bits in (key_bits, value_bits):
        made.append(torch.randint(0, 256, (pages, heads, page, dim * bits // 8), generator=g, dtype=torch.uint8).to(device))
        header = torch.full((pages, heads, page, 2), float("nan")) if poison else torch.randn((pages, heads, page, 2), generator=g)
        made.append(header.to(device))
    return made


def fill(cache, slots, k, v, key_bits, value_bits):
    """Writes k and v [tokens, heads, dim] into the slots from the definition."""
    page = cache[0].shape[2]
    block, at = slots // page, slots % page
    for x, bits, codes, header in ((k, key_bits, cache[0], cache[1]), (v, value_bits, cache[2], cache[3])):
        c, h = quantise(x.float().cpu().numpy(), bits)
        codes[block, :, at] = torch.from_numpy(pack(c, bits)).to(codes.device)
        header[block, :, at] = torch.from_numpy(h).to(codes.device)
