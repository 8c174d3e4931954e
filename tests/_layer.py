"""The operators of a layer around the attention from their definitions, in 64 bits and without the library."""
from __future__ import annotations

import torch

UNIT = 2.0 ** -24                      # of a rounding in binary32
SHIFTS = (0, 16, 4, 20, 8, 24, 12, 28)  # of a word's eight codes


def _rms(v, eps):
    return (v.square().mean(-1, keepdim=True) + eps) ** -0.5


def block_norm(x, h, gate, weight, post, scale, eps):
    """(r, y, magnitude of what r adds up)."""
    x = x.double()
    if h is None:
        return x, x * _rms(x, eps) * weight.double(), x.abs()
    n = h.double()
    if post is not None:
        n = n * _rms(n, eps) * post.double()
    if gate is not None:
        n = n * gate.double()
    r = x + scale * n
    return r, r * _rms(r, eps) * weight.double(), x.abs() + (scale * n).abs()


def block_norm_bounds(x, h, gate, weight, post, scale, eps, r, y, magnitude):
    """How far binary32 arithmetic may be off before the last rounding.  A row's sum of squares is at most 32 sums in a lane, 6 over a wavefront and 16 over
    the wavefronts, all of one sign: 54 roundings, halved by the root, with the division, the root, the mean and eps less than 32; then up to five products
    and sums.  y depends on r's error by itself and through the root, where it counts by the row's mean."""
    off_r = 40 * UNIT * magnitude
    q = _rms(r, eps)
    off_y = (off_r + r.abs() * q * (off_r.square().mean(-1, keepdim=True) ** 0.5)) * q * weight.double().abs() + 40 * UNIT * y.abs()
    return off_r, off_y


def block_norm_backward(grad_r, grad_y, r, h, gate, weight, post, scale, eps):
    """{name: (gradient, magnitude of the terms that it adds up)}."""
    r, u, w = r.double(), grad_y.double(), weight.double()
    q = _rms(r, eps)
    uw = u * w
    x = q * (uw - r * q * q * (uw * r).mean(-1, keepdim=True))
    a = q * (uw.abs() + r.abs() * q * q * (uw * r).abs().mean(-1, keepdim=True))
    if grad_r is not None:
        x, a = x + grad_r.double(), a + grad_r.double().abs()
    out = {"x": (x, a), "weight": ((u * r * q).sum(0), (u * r * q).abs().sum(0))}
    if h is None:
        return out
    h, s, b = h.double(), scale * x, abs(scale) * a
    t = _rms(h, eps) if post is not None else torch.ones_like(h[:, :1])
    n = h * t * (post.double() if post is not None else 1.0)
    if gate is not None:
        out["gate"] = (s * n, b * n.abs()) if gate.dim() == 2 else ((s * n).sum(0), (b * n.abs()).sum(0))
        s, b = s * gate.double(), b * gate.double().abs()
    if post is None:
        out["h"] = (s, b)
        return out
    out["post"] = ((s * h * t).sum(0), (b * (h * t).abs()).sum(0))
    s, b = s * post.double(), b * post.double().abs()
    out["h"] = (t * (s - h * t * t * (s * h).mean(-1, keepdim=True)), t * (b + h.abs() * t * t * (b * h.abs()).mean(-1, keepdim=True)))
    return out


def quantise_weights(w, group):
    """(codes [outputs, groups, group], zero, step [outputs, groups]) by binary32 operations one at a time; `w` without infinities and NaN."""
    w = w.float()
    outputs, inputs = w.shape
    groups = (inputs + group - 1) // group
    codes = torch.zeros((outputs, groups, group))
    zeros, steps = torch.zeros((outputs, groups)), torch.zeros((outputs, groups))
    for g in range(groups):
        part = w[:, g * group:min(inputs, (g + 1) * group)]
        low, high = part.amin(1), part.amax(1)
        zero = (low + 0.0).bfloat16().float()
        step = ((high - low) / 15.0).bfloat16().float()
        inverse = torch.ones_like(step) / step
        flat = (step == 0) | torch.isinf(inverse)
        zeros[:, g], steps[:, g] = zero, torch.where(flat, 0.0, step)
        code = torch.round(torch.clamp((part - zero[:, None]) * torch.where(flat, 0.0, inverse)[:, None], 0, 15))
        codes[:, g, :part.shape[1]] = code
    return codes, zeros, steps


def pack(codes):
    """Words int32 [outputs, groups * group / 8] of codes [outputs, groups, group]."""
    c = codes.flatten(1).long().view(codes.shape[0], -1, 8)
    words = torch.zeros(c.shape[:2], dtype=torch.int64)
    for i, shift in enumerate(SHIFTS):
        words |= c[..., i] << shift
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()


def unpack(words, group):
    w = words.long() & 0xffffffff
    return torch.stack([(w >> shift) & 15 for shift in SHIFTS], -1).view(w.shape[0], -1, group)


def weights(words, header, inputs):
    """[outputs, inputs] in 64 bits, and the steps of each element."""
    group = words.shape[1] * 8 // header.shape[1]
    h = header.double()
    w = unpack(words, group) * h[..., 1:] + h[..., :1]
    return w.flatten(1)[:, :inputs], h[..., 1:].expand(-1, -1, group).flatten(1)[:, :inputs].abs()


def random_weights(outputs, inputs, group, seed):
    """(codes, header) of every code, and zero points and steps of either sign."""
    g = torch.Generator().manual_seed(seed)
    groups = (inputs + group - 1) // group
    words = torch.randint(-2 ** 31, 2 ** 31, (outputs, groups * group // 8), generator=g).int()
    step = (0.02 + 0.1 * torch.rand((outputs, groups), generator=g)) * torch.where(torch.rand((outputs, groups), generator=g) < 0.1, -1.0, 1.0)
    zero = -7.5 * step + 0.1 * torch.randn((outputs, groups), generator=g)
    return words, torch.stack((zero, step), -1).bfloat16()
