"""Attention over a quantised cache from its definition in 64 bits, with a bound on a kernel's error for every row by itself."""
from __future__ import annotations

import numpy as np
import torch

import _heads as H

# of the two operands that the kernels hold in binary16: of one number of it, of two
ONE, TWO = 2.0 ** -11, 2.0 ** -22


def _rows(q, cache, table, lengths, start, dim, window):
    """(token, head, position, keys in sight of it, their parts) of every row that sees something; parts: (codes, zero, step) of keys and of values."""
    key_codes, key_header, value_codes, value_header = (t.cpu().numpy() for t in cache)
    page, kv = key_codes.shape[2], key_codes.shape[1]
    group = q.shape[1] // kv
    unpacked = [H.unpack(c, 8 if c.shape[3] == dim else 4) for c in (key_codes, value_codes)]
    centers = [128.0 if c.shape[3] == dim else 8.0 for c in (key_codes, value_codes)]
    table, start = table.cpu().numpy(), start.tolist()
    for n, length in enumerate(lengths.tolist()):
        count = start[n + 1] - start[n]
        for i in range(count):
            position = length - count + i
            if position < 0:
                continue
            j = np.arange(max(0, position - window + 1) if window else 0, position + 1)
            at = table[n][j // page], j % page
            for h in range(q.shape[1]):
                parts = [(u[at[0], h // group, at[1]].astype(np.float64), *(header[at[0], h // group, at[1]].astype(np.float64).T[..., None]), c)
                         for u, header, c in zip(unpacked, (key_header, value_header), centers)]
                yield start[n] + i, h, parts


def attention(q, cache, table, lengths, start, dim, scale=None, softcap=0.0, window=0):
    """(out, bound) float64 [tokens, heads, dim]; rows that see nothing are zeros.

    The bound of an element takes the roundings as independent and allows six times their root mean square, each at its largest:
      weights p * step   rounded to one binary16 number (16-bit types) or two (binary32), times the centred code
      scores             off by e, which moves a weight by its share e and so the result by e times the value's distance from it; e: products of `dim`
                         terms summed in binary32, the roundings of what they are multiplied with and of the two terms of a score, the exponential and
                         the cap; for binary32 the rest of q behind two binary16 numbers
      sums               of the weights and of the outputs, block by block, in binary32
    and beside it the result's own rounding and the smallest binary16 weight, 2^-31 of the largest."""
    fine, unit = q.dtype == torch.float32, 2.0 ** -24
    roundoff = H.ROUNDOFF[q.dtype]
    q = q.double().cpu().numpy()
    scale = dim ** -0.5 if scale is None else scale
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    for token, head, ((kc, kz, ks, k_center), (vc, vz, vs, v_center)) in _rows(q, cache, table, lengths, start, dim, window):
        x = q[token, head]
        k, v = kz + ks * kc, vz + vs * vc
        s = k @ x * scale
        raw = s
        if softcap:
            s = softcap * np.tanh(s / softcap)
        p = np.exp(s - s.max())
        p /= p.sum()
        y = p @ v
        out[token, head] = y
        centred = (kc - k_center) * ks
        terms = (kz[:, 0] + k_center * ks[:, 0]) * x.sum(), kz[:, 0] * x.sum(), centred @ x, ks[:, 0] * (kc @ x)
        e = unit * (2 * dim ** 0.5 * np.sqrt(((np.abs(kz) + ks * kc) ** 2) @ x ** 2) + 16 * sum(np.abs(t) for t in terms) + 16 * np.abs(raw / scale if scale else raw)) * abs(scale)
        e += 16 * unit * (np.abs(s) + np.abs(s).max()) + 2.0 ** -22 + (TWO * abs(scale) * np.sqrt(centred ** 2 @ x ** 2) if fine else 0.0)
        weight = (TWO if fine else ONE) * np.abs(vc - v_center) * vs
        random = np.sqrt((p[:, None] ** 2 * (weight ** 2 + (e[:, None] * (v - y)) ** 2)).sum(0))
        sums = (8 + len(p) ** 0.5) * unit * (p @ (np.abs(vz + v_center * vs) + np.abs(vc - v_center) * vs))
        smallest = 2.0 ** -31 * len(p) ** 0.5 * (p * vs[:, 0]).max() * 2 * v_center
        bound[token, head] = roundoff * np.abs(y) + 6 * random + sums + 6 * smallest + (2.0 ** -25 if roundoff == 2.0 ** -11 else 0.0)
    return out, bound


def _halves(x, parts):
    """x (binary32) as a sum of so many binary16 numbers."""
    high = x.astype(np.float16).astype(np.float32)
    return high if parts == 1 else high + (x - high).astype(np.float16).astype(np.float32)


def modelled(q, cache, table, lengths, start, dim, scale=None, softcap=0.0, window=0, q_parts=None, weight_parts=None):
    """The same in the kernels' arithmetic, by numpy in binary32: operands in binary16, products exact, sums in binary32."""
    dtype = q.dtype
    q_parts, weight_parts = (p or (2 if dtype == torch.float32 else 1) for p in (q_parts, weight_parts))
    q32 = q.float().cpu().numpy()
    f = np.float32
    scale = dim ** -0.5 if scale is None else scale
    out = np.zeros(q.shape, dtype=np.float32)
    for token, head, parts in _rows(q32, cache, table, lengths, start, dim, window):
        (kc, kz, ks, k_center), (vc, vz, vs, v_center) = ([a.astype(f) if isinstance(a, np.ndarray) else f(a) for a in part] for part in parts)
        x = q32[token, head]
        exponent = np.floor(np.log2(np.abs(x).max())) if np.abs(x).max() else 0
        x = _halves(x * f(2.0 ** (13 - exponent)), q_parts)
        s = ((kc - k_center) @ x * ks[:, 0] + (kz + k_center * ks)[:, 0] * x.sum(dtype=f)) * f(2.0 ** (exponent - 13)) * f(scale)
        if softcap:
            s = f(softcap) * np.tanh(s / f(softcap))
        y = s * f(np.log2(np.e)) + np.log2(np.maximum(vs[:, 0], f(2.0 ** -80)))
        p = np.exp2(s * f(np.log2(np.e)) - (y.max() - f(7)))
        weight = _halves(p * vs[:, 0], weight_parts)
        out[token, head] = ((weight @ (vc - v_center)) + p @ (vz + v_center * vs)) / p.sum(dtype=f)
    return torch.from_numpy(out).to(dtype)
