"""Workloads of a layer's operators around the attention: norms of the residual stream, products with 4-bit weights, appending to the cache.

`listed()` names them, `draw(rng)` gives another of the same ranges, `prepare(case, seed)` makes what the program has in
hand before the call, `run(state)` is one pass (the plain form in elementary torch operations, or the library's kernels
where `own` is true), `work(case)` the bytes and operations a pass cannot do without, and `exact(case, seed)` the outputs
in 64 bits.

Kinds of work:
  block        the norms behind and before a block with its gate, its scale and the residual sum
  block_grad   its backward pass: gradients of the residual stream, the block's output, the gate and both weights
  linear       product of rows with weights of 4 bits and a zero point and step per group
  linear_grad  the gradient of those rows
  append       norm and rotation of new queries and keys, keys and values quantised into the cache; the outputs are the queries and
               the values that are held
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
POSITIONS = 32768   # entries of the rotation's tables


def _block(kind, tokens, width, dtype, post, gate, scale, **name):
    return dict(kind=kind, tokens=tokens, width=width, dtype=dtype, post=post, gate=gate, scale=scale, **name)


def _linear(kind, rows, inputs, outputs, group, dtype, bias=False, **name):
    return dict(kind=kind, rows=rows, inputs=inputs, outputs=outputs, group=group, dtype=dtype, bias=bias, **name)


def _append(tokens, q_heads, kv_heads, dim, dtype, key_bits, value_bits, page, pages, norm=True, rotated=None, interleaved=False, **name):
    return dict(kind="append", tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype, key_bits=key_bits, value_bits=value_bits, page=page,
                pages=pages, norm=norm, rotated=rotated or dim, interleaved=interleaved, **name)


def listed():
    return [
        # one decoding step of eight sequences, a learned gate per channel: latency
        _block("block", 8, 4096, "bf16", True, "channel", 1.0, name="block_step_bf16"),
        # a training batch of 4 x 2048 tokens with a residual scale and no gate, norm before the next block only
        _block("block", 8192, 4096, "f16", False, "none", 0.5, name="block_batch_f16"),
        # backward of a small model in binary32, odd in both sizes, gate of every token
        _block("block_grad", 1023, 2047, "f32", True, "token", 1.0, name="block_grad_odd_f32"),
        # backward of a large batch, gate per channel
        _block("block_grad", 16384, 4096, "bf16", True, "channel", 0.7, name="block_grad_batch_bf16"),
        # one token through a square projection: latency
        _linear("linear", 1, 4096, 4096, 128, "bf16", name="linear_token_bf16"),
        # a serving step of some sequences through a wide projection, small groups
        _linear("linear", 23, 8192, 16384, 64, "f16", name="linear_step_f16"),
        # a short chunk in binary32, odd sizes, with a bias
        _linear("linear", 301, 1000, 1501, 32, "f32", bias=True, name="linear_odd_f32"),
        # a chunk of a long prompt
        _linear("linear", 4096, 8192, 8192, 128, "bf16", name="linear_chunk_bf16"),
        # training in front of frozen weights
        _linear("linear_grad", 2047, 4096, 8192, 128, "bf16", name="linear_grad_bf16"),
        # one token of each of 32 sequences into a cache of 8 bits
        _append(32, 32, 8, 128, "bf16", 8, 8, 16, 4096, name="append_step_bf16"),
        # a prompt of odd length into a narrow cache
        _append(8191, 32, 8, 128, "f16", 4, 4, 64, 512, name="append_prompt_f16"),
        # evaluation in binary32 of a model that only rotates, half of every head, pairs side by side
        _append(333, 12, 4, 64, "f32", 8, 4, 16, 128, norm=False, rotated=32, interleaved=True, name="append_rotated_f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["block", "block_grad", "linear", "linear", "linear", "linear_grad", "append", "append"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if kind in ("block", "block_grad"):
        width = _log(rng, 64, 8192)
        width = width if rng.random() < 0.3 else max(64, width // 64 * 64)
        most = 16384 * 4096 // width // (2 if dtype == "f32" else 1)
        return _block(kind, _log(rng, 1, min(16384, most)), width, dtype, rng.random() < 0.6, rng.choice(["none", "channel", "token"]), rng.choice([1.0, 0.5, 0.22]))
    if kind in ("linear", "linear_grad"):
        inputs, outputs = _log(rng, 64, 8192), _log(rng, 64, 16384)
        if rng.random() < 0.6:
            inputs, outputs = max(128, inputs // 128 * 128), max(64, outputs // 64 * 64)
        # no more operations than the largest listed case, of which the gradient and binary32 get a half
        most = (1 << 38) // (inputs * outputs) // (1 if kind == "linear" and dtype != "f32" else 2)
        rows = rng.choice([1, _log(rng, 2, 64), _log(rng, 1, 4096)])
        return _linear(kind, max(1, min(rows, most)), inputs, outputs, rng.choice([32, 64, 128]), dtype, kind == "linear" and rng.random() < 0.3)
    kv_heads, dim = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128, 256])
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 8])
    key_bits, value_bits = rng.choice([(8, 8), (4, 4), (8, 4)])
    page = rng.choice([16, 32, 64, 128])
    tokens = _log(rng, 1, min(16384, (1 << 26) // ((q_heads + 2 * kv_heads) * dim)))
    return _append(tokens, q_heads, kv_heads, dim, dtype, key_bits, value_bits, page, (tokens + page - 1) // page + rng.randrange(1, 100), rng.random() < 0.7,
                   rng.choice([dim, dim, dim // 2]), rng.random() < 0.3)


# ----------------------------------------------------------------------------- inputs

# places of a word's eight codes: pair i of them lies in bits 4 i and 16 + 4 i
_SHIFTS = (0, 16, 4, 20, 8, 24, 12, 28)


def _quantised_weights(w, group):
    """(codes int32 [outputs, inputs / 8], header bfloat16 [outputs, groups, 2] = (zero, step)) of weights whose inputs are padded with zeros to whole groups."""
    outputs, inputs = w.shape
    groups = (inputs + group - 1) // group
    w = torch.nn.functional.pad(w, (0, groups * group - inputs)).view(outputs, groups, group)
    zero = w.amin(-1, keepdim=True).bfloat16()
    step = ((w.amax(-1, keepdim=True) - w.amin(-1, keepdim=True)) / 15).bfloat16()
    codes = torch.round((w - zero.float()) / step.float()).nan_to_num_().clamp_(0, 15).int().view(outputs, groups * group // 8, 8)
    packed = torch.zeros_like(codes[..., 0])
    for i, shift in enumerate(_SHIFTS):
        packed |= codes[..., i] << shift
    return packed, torch.cat((zero, step), -1)


def _tables(rotated):
    angle = torch.arange(POSITIONS, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rotated, 2, device=DEV, dtype=torch.float64) / rotated)
    return torch.cos(angle).float(), torch.sin(angle).float()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    s = dict(case)

    def randn(*shape):
        return torch.randn(shape, device=DEV, generator=g)

    if kind in ("block", "block_grad"):
        tokens, width = case["tokens"], case["width"]
        # a residual stream has channels of very different sizes
        channel = torch.exp(0.7 * randn(width))
        s["x"], s["h"] = (randn(tokens, width) * channel).to(dtype), (randn(tokens, width) * (0.3 + torch.rand(width, device=DEV, generator=g))).to(dtype)
        s["weight"] = (1 + 0.1 * randn(width)).to(dtype)
        s["post_weight"] = (0.5 + 0.1 * randn(width)).to(dtype) if case["post"] else None
        s["gate"] = {"none": lambda: None, "channel": lambda: 0.3 * randn(width).to(dtype), "token": lambda: torch.sigmoid(randn(tokens, width)).to(dtype)}[case["gate"]]()
        if kind == "block_grad":   # the saved sum in place of x
            s["r"] = s.pop("x")
            s["grad_r"], s["grad_y"] = randn(tokens, width).to(dtype), (randn(tokens, width) * (0.5 + torch.rand(tokens, 1, device=DEV, generator=g))).to(dtype)
        return s
    if kind in ("linear", "linear_grad"):
        rows, inputs, outputs = case["rows"], case["inputs"], case["outputs"]
        w = randn(outputs, inputs) * inputs ** -0.5 * (0.5 + torch.rand((outputs, 1), device=DEV, generator=g))
        s["codes"], s["header"] = _quantised_weights(w, case["group"])
        s["rows_in"] = (randn(rows, outputs if kind == "linear_grad" else inputs) * (0.3 + torch.rand((rows, 1), device=DEV, generator=g))).to(dtype)
        s["b"] = randn(outputs).to(dtype) if case["bias"] else None
        return s
    tokens, qh, kv, dim, page = case["tokens"], case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    # queries, keys and values of a token lie side by side, as one projection leaves them
    channel = 0.5 + torch.rand((qh + 2 * kv) * dim, device=DEV, generator=g)
    x = (randn(tokens, (qh + 2 * kv) * dim) * channel).to(dtype)
    s["q"], s["k"], s["v"] = (x[:, a * dim:b * dim].view(tokens, b - a, dim) for a, b in ((0, qh), (qh, qh + kv), (qh + kv, qh + 2 * kv)))
    s["q_weight"], s["k_weight"] = ((1 + 0.1 * randn(dim)).to(dtype) if case["norm"] else None for _ in range(2))
    s["positions"] = torch.randint(0, POSITIONS, (tokens,), device=DEV, generator=g, dtype=torch.int32)
    s["cos"], s["sin"] = _tables(case["rotated"])
    order = torch.randperm(case["pages"], device=DEV, generator=g)
    if tokens <= case["pages"]:   # a token of each of so many sequences
        s["slots"] = order[:tokens] * page + torch.randint(0, page, (tokens,), device=DEV, generator=g)
    else:                         # one sequence, page after page
        at = torch.arange(tokens, device=DEV)
        s["slots"] = order[at // page] * page + at % page
    for name, bits in (("key", case["key_bits"]), ("value", case["value_bits"])):
        s[name + "_codes"] = torch.zeros((case["pages"], kv, page, dim * bits // 8), dtype=torch.uint8, device=DEV)
        s[name + "_header"] = torch.zeros((case["pages"], kv, page, 2), device=DEV)
    return s


# ----------------------------------------------------------------------------- plain forms

def _plain_block(s):
    n = s["h"].float()
    if s["post_weight"] is not None:
        n = n * torch.rsqrt((n * n).mean(-1, keepdim=True) + EPS) * s["post_weight"].float()
    if s["gate"] is not None:
        n = n * s["gate"].float()
    r = s["x"].float() + s["scale"] * n
    y = r * torch.rsqrt((r * r).mean(-1, keepdim=True) + EPS) * s["weight"].float()
    return {"r": r.to(s["x"].dtype), "y": y.to(s["x"].dtype)}


def _plain_norm_grad(grad, x, weight):
    """Gradients of an RMS norm's input and weight (binary32)."""
    q = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * q
    gw = grad * weight
    return q * (gw - n * (gw * n).mean(-1, keepdim=True)), (grad * n).sum(0)


def _plain_block_grad(s):
    dtype = s["r"].dtype
    out = {}
    grad, weight = _plain_norm_grad(s["grad_y"].float(), s["r"].float(), s["weight"].float())
    grad += s["grad_r"].float()
    out["x"], out["weight"] = grad.to(dtype), weight.to(dtype)
    grad = grad * s["scale"]
    h = s["h"].float()
    if s["gate"] is not None:
        n = h
        if s["post_weight"] is not None:
            n = n * torch.rsqrt((n * n).mean(-1, keepdim=True) + EPS) * s["post_weight"].float()
        n = grad * n
        out["gate"] = (n if s["gate"].dim() == 2 else n.sum(0)).to(dtype)
        grad = grad * s["gate"].float()
    if s["post_weight"] is not None:
        grad, weight = _plain_norm_grad(grad, h, s["post_weight"].float())
        out["post_weight"] = weight.to(dtype)
    out["h"] = grad.to(dtype)
    return out


def _plain_weights(s):
    codes = (s["codes"].unsqueeze(-1) >> torch.tensor(_SHIFTS, dtype=torch.int32, device=DEV)) & 15
    header = s["header"].float()
    w = codes.view(header.shape[0], header.shape[1], -1).float() * header[..., 1:] + header[..., :1]
    return w.flatten(1)[:, :s["inputs"]]


def _plain_linear(s):
    y = torch.matmul(s["rows_in"].float(), _plain_weights(s).t())
    return (y if s["b"] is None else y + s["b"].float()).to(s["rows_in"].dtype)


def _rotated(x, cos, sin, s):
    turned, part = s["rotated"], x[..., :s["rotated"]]
    a, b = (part[..., 0::2], part[..., 1::2]) if s["interleaved"] else (part[..., :turned // 2], part[..., turned // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat((torch.stack((a, b), -1).flatten(-2) if s["interleaved"] else torch.cat((a, b), -1), x[..., turned:]), -1)


def _plain_head(x, weight, s, dtype):
    """Norm and rotation in `dtype`: 64 bits for keys, whose codes change at a border."""
    n = x.to(dtype)
    if s["norm"]:
        n = n * torch.rsqrt((n * n).mean(-1, keepdim=True) + EPS) * weight.to(dtype)
    return _rotated(n, s["cos"][s["positions"]][:, None].to(dtype), s["sin"][s["positions"]][:, None].to(dtype), s)


def _plain_write(x, slots, codes, header, bits, dtype):
    """Codes and headers of the groups of `x` (binary32) into the pages; the values that they stand for."""
    page, top = codes.shape[2], torch.full_like(x[..., :1], (1 << bits) - 1)
    zero = x.amin(-1, keepdim=True) + 0.0
    extent = x.amax(-1, keepdim=True) - zero
    inverse = top / extent
    flat = (extent == 0) | torch.isinf(inverse)
    step = torch.where(flat, 0.0, extent / top)
    c = torch.round(torch.minimum((x - zero) * torch.where(flat, 0.0, inverse), top))
    b = c.to(torch.uint8)
    codes[slots // page, :, slots % page] = b if bits == 8 else b[..., 0::2] | (b[..., 1::2] << 4)
    header[slots // page, :, slots % page] = torch.cat((zero, step), -1)
    return (c * step + zero).to(dtype)


def run(state):
    s, kind = state, state["kind"]
    if own:
        return _own(s)
    if kind == "block":
        return _plain_block(s)
    if kind == "block_grad":
        return _plain_block_grad(s)
    if kind == "linear":
        return {"y": _plain_linear(s)}
    if kind == "linear_grad":
        return {"x": torch.matmul(s["rows_in"].float(), _plain_weights(s)).to(s["rows_in"].dtype)}
    dtype = s["q"].dtype
    return {"q": _plain_head(s["q"], s["q_weight"], s, torch.float32).to(dtype),
            "k": _plain_write(_plain_head(s["k"], s["k_weight"], s, torch.float64).float(), s["slots"], s["key_codes"], s["key_header"], s["key_bits"], dtype),
            "v": _plain_write(s["v"].float(), s["slots"], s["value_codes"], s["value_header"], s["value_bits"], dtype)}


def _own(s):
    from paper_2104_14129_amd import binding as B
    kind = s["kind"]
    if kind == "block":
        r, y = B.block_norm(s["x"], s["h"], s["gate"], s["weight"], s["post_weight"], s["scale"], EPS)
        return {"r": r, "y": y}
    if kind == "block_grad":
        x, h, gate, weight, post = B.block_norm_backward(s["grad_r"], s["grad_y"], s["r"], s["h"], s["gate"], s["weight"], s["post_weight"], s["scale"], EPS)
        return {k: v for k, v in (("x", x), ("weight", weight), ("gate", gate), ("post_weight", post), ("h", h)) if v is not None}
    if kind == "linear":
        return {"y": B.linear4(s["rows_in"], s["codes"], s["header"], s["b"])}
    if kind == "linear_grad":
        return {"x": B.linear4_backward(s["rows_in"], s["codes"], s["header"], s["inputs"])}
    cache = s["key_codes"], s["key_header"], s["value_codes"], s["value_header"]
    q = B.cache_append(s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["positions"], s["cos"], s["sin"], s["slots"], *cache,
                       eps=EPS if s["norm"] else None, interleaved=s["interleaved"])
    k, v = B.cache_read(s["slots"], *cache, s["dim"], s["q"].dtype)
    return {"q": q, "k": k, "v": v}


# ----------------------------------------------------------------------------- what a pass has to do

def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    if case["kind"] in ("block", "block_grad"):
        values, grad = case["tokens"] * case["width"], case["kind"] == "block_grad"
        passes = (6 if grad else 4) + {"none": 0, "channel": 0, "token": 2 if grad else 1}[case["gate"]]
        vectors = (1 + case["post"] + (case["gate"] == "channel")) * (2 if grad else 1)
        return {"bytes": (passes * values + vectors * case["width"]) * size, "flops": values * (25 if grad else 11)}
    if case["kind"] in ("linear", "linear_grad"):
        rows, inputs, outputs = case["rows"], case["inputs"], case["outputs"]
        groups = (inputs + case["group"] - 1) // case["group"]
        return {"bytes": rows * (inputs + outputs) * size + outputs * groups * (case["group"] // 2 + 4) + case["bias"] * outputs * size, "flops": 2 * rows * inputs * outputs}
    tokens, kv, dim = case["tokens"], case["kv_heads"], case["dim"]
    held = dim * (case["key_bits"] + case["value_bits"]) // 8 + 16   # bytes of a token and head in the cache
    tables = min(tokens, POSITIONS) * case["rotated"] * 4
    values = tokens * (2 * case["q_heads"] + 4 * kv) * dim   # queries read and written, keys and values read and returned as they are held
    return {"bytes": values * size + tokens * (kv * held + 12) + tables + case["norm"] * 2 * dim * size, "flops": tokens * dim * (8 * case["q_heads"] + 20 * kv)}


# ----------------------------------------------------------------------------- the definitions in 64 bits

def _rms(v):
    return (torch.linalg.vector_norm(v, dim=-1, keepdim=True) ** 2 / v.shape[-1] + EPS) ** 0.5


def _exact_block(s):
    x, h = s["x"].double(), s["h"].double()
    after = h if s["post_weight"] is None else s["post_weight"].double() * h / _rms(h)
    r = torch.addcmul(x, after, torch.ones((), device=DEV, dtype=torch.float64) if s["gate"] is None else s["gate"].double(), value=s["scale"])
    return {"r": r, "y": s["weight"].double() * r / _rms(r)}


def _exact_norm_grad(u, v):
    """The derivative of v / rms(v) applied to u."""
    rms = _rms(v)
    return u / rms - v * torch.linalg.vecdot(u, v, dim=-1).unsqueeze(-1) / (v.shape[-1] * rms ** 3)


def _exact_block_grad(s):
    r, h, gy, w = (s[k].double() for k in ("r", "h", "grad_y", "weight"))
    total = s["grad_r"].double() + _exact_norm_grad(gy * w, r)
    back = total * s["scale"]
    out = {"x": total, "weight": (gy * (r / _rms(r))).sum(0)}
    p = None if s["post_weight"] is None else s["post_weight"].double()
    unit = h if p is None else h / _rms(h)
    gated = back if s["gate"] is None else back * s["gate"].double()
    if s["gate"] is not None:
        per_token = back * (unit if p is None else unit * p)
        out["gate"] = per_token if s["gate"].dim() == 2 else per_token.sum(0)
    if p is not None:
        out["post_weight"] = (gated * unit).sum(0)
    out["h"] = gated if p is None else _exact_norm_grad(gated * p, h)
    return out


def _exact_weights(s):
    """[outputs, inputs] in 64 bits, a code's place in the words at a time."""
    outputs, groups = s["header"].shape[:2]
    words, group = s["codes"].long(), s["group"]
    w = torch.empty((outputs, groups * group), dtype=torch.float64, device=DEV)
    for place in range(8):
        w[:, place::8] = ((words >> (4 * (place // 2) + 16 * (place % 2))) & 15).double()
    for i in range(groups):
        zero, step = s["header"][:, i].double().unbind(-1)
        w[:, i * group:(i + 1) * group].mul_(step[:, None]).add_(zero[:, None])
    return w[:, :s["inputs"]]


def _exact_turned(x, weight, s):
    y = x.double()
    if s["norm"]:
        y = y / _rms(y) * weight.double()
    z = y.clone()
    c, d = s["cos"].double()[s["positions"].long()], s["sin"].double()[s["positions"].long()]
    half = s["rotated"] // 2
    for p in range(half):
        i, j = (2 * p, 2 * p + 1) if s["interleaved"] else (p, p + half)
        z[..., i] = y[..., i] * c[:, p, None] - y[..., j] * d[:, p, None]
        z[..., j] = y[..., i] * d[:, p, None] + y[..., j] * c[:, p, None]
    return z


def _exact_held(x, bits):
    """The codes are defined in binary32 on the values rounded to it; what they stand for in 64 bits."""
    x, top = x.float(), float((1 << bits) - 1)
    low, high = x.aminmax(dim=-1, keepdim=True)
    low = low + 0.0
    extent = high - low
    scale = torch.full_like(extent, top) / extent
    usable = (extent != 0) & torch.isfinite(scale)
    code = torch.where(usable, torch.round(torch.clamp_max((x - low) * scale, top)), 0.0)
    return low.double() + code.double() * torch.where(usable, extent / torch.full_like(extent, top), 0.0).double()


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "block":
        return _exact_block(s)
    if kind == "block_grad":
        return _exact_block_grad(s)
    if kind == "linear":
        y = s["rows_in"].double() @ _exact_weights(s).T.contiguous()
        return {"y": y if s["b"] is None else y + s["b"].double()}
    if kind == "linear_grad":
        return {"x": s["rows_in"].double() @ _exact_weights(s)}
    return {"q": _exact_turned(s["q"], s["q_weight"], s), "k": _exact_held(_exact_turned(s["k"], s["k_weight"], s), case["key_bits"]), "v": _exact_held(s["v"], case["value_bits"])}
