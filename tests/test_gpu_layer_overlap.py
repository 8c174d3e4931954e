"""Outputs of a layer's operators that share memory with what is read: refused before anything is launched, also where rows lie inside wider ones; taken where
they replace an input element by element or take turns with it."""
import pytest
import torch

import _heads as H
import _layer as Y
from paper_2104_14129_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _randn(*shape, seed=1, dtype=F32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def _refused(call, match):
    with pytest.raises(RuntimeError, match=match):
        call()


def test_block_norm():
    b, h, w = _randn(9, 200), _randn(4, 64, seed=2), torch.ones(64, device=DEV)
    gate = _randn(4, 64, seed=3)
    x = b[:4, :64]
    before = b.clone()
    for r in (b[1:5, :64], b[:4, 1:65], b[:4, 63:127], b[:4, 32:96], b[::2, :64][:4], b.view(-1)[150:150 + 4 * 64].view(4, 64)):
        _refused(lambda: B.block_norm(x, h, None, w, r=r), "r must not share memory with x")
        _refused(lambda: B.block_norm(x, h, None, w, y=r), "y must not share memory with x")
        _refused(lambda: B.block_norm(h, x, None, w, r=r), "r must not share memory with h")
        _refused(lambda: B.block_norm(h, gate, x, w, y=r), "y must not share memory with gate")
    _refused(lambda: B.block_norm(h, gate, None, w, r=x, y=x), "r must not share memory with y")
    _refused(lambda: B.block_norm(h, gate, None, w, r=x, y=b[:4, 63:127]), "r must not share memory with y")
    flat = torch.ones(4 * 64, device=DEV)
    vector = flat[70:134]
    for call in (lambda: B.block_norm(x, h, None, vector, r=flat.view(4, 64)), lambda: B.block_norm(x, h, vector, w, r=flat.view(4, 64)),
                 lambda: B.block_norm(x, h, None, w, vector, y=flat.view(4, 64))):
        _refused(call, "must not share memory with (weight|post_weight|gate)")
    assert torch.equal(b, before) and (flat == 1).all()
    # by turns with x, and in its place
    want = B.block_norm(x.clone(), h, gate, w, w)
    r, y = B.block_norm(x, h, gate, w, w, r=b[:4, 64:128], y=b[4:8, :64])
    assert torch.equal(r, want[0]) and torch.equal(y, want[1]) and torch.equal(x, before[:4, :64])
    _, y = B.block_norm(b[::2, :64][:4].copy_(before[:4, :64]), h, gate, w, w, r=b[1::2, :64])
    assert torch.equal(b[1::2, :64], want[0]) and torch.equal(y, want[1])
    x.copy_(before[:4, :64])
    g = gate.clone()
    r, y = B.block_norm(x, h, g, w, w, r=x, y=g)
    assert torch.equal(x, want[0]) and torch.equal(g, want[1])
    row = b[:1, :64].copy_(before[:1, :64])
    r, _ = B.block_norm(row, h[:1], gate[:1], w, w, r=b.view(-1)[:64].view(1, 64))   # one row: its stride is of no account
    assert torch.equal(row, want[0][:1])


@pytest.mark.parametrize("rows", [3, 40, 300])
def test_linear4(rows):
    codes, header = (t.to(DEV) for t in Y.random_weights(96, 128, 32, 4))
    b = _randn(rows + 2, 512, dtype=BF16)
    before = b.clone()
    x = b[:rows, :128]
    for out in (b[:rows, :96], b[:rows, 127:223], b[1:1 + rows, 100:196], b[2:, 32:128]):
        _refused(lambda: B.linear4(x, codes, header, None, out), "out must not share memory with x")
    bias = b[rows // 2, 300:396]
    _refused(lambda: B.linear4(x, codes, header, bias, b[:rows, 395:491]), "out must not share memory with bias")
    over = codes.view(BF16).view(-1)[:3 * 96].view(3, 96)
    _refused(lambda: B.linear4(x[:3], codes, header, None, over), "out must not share memory with codes")
    _refused(lambda: B.linear4(x[:3], codes, header, None, header.view(-1)[:288].view(3, 96)), "out must not share memory with header")
    assert torch.equal(b, before)
    want = B.linear4(x, codes, header)
    assert torch.equal(B.linear4(x, codes, header, None, b[:rows, 128:224]), want) and torch.equal(b[:rows, 128:224], want)


def test_append():
    tokens, heads, kv, dim = 6, 4, 2, 64
    b = _randn(tokens + 1, (heads + 2 * kv + 2) * dim)
    before = b.clone()
    view = lambda t, first, n: t[:tokens, first * dim:(first + n) * dim].view(tokens, n, dim)   # noqa: E731
    q, k, v = view(b, 0, heads), view(b, heads, kv), view(b, heads + kv, kv)
    angle = _randn(8, dim // 2, seed=5)
    cos, sin = torch.cos(angle), torch.sin(angle)
    positions, slots = torch.arange(tokens, dtype=torch.int32, device=DEV), torch.arange(tokens, device=DEV)
    cache = H.make_cache(2, kv, 16, dim, 8, 8, 1, poison=False)
    kept = [t.clone() for t in cache]
    call = lambda out, k=k, v=v, q=q, cos=cos: B.cache_append(q, k, v, None, None, positions, cos, sin, slots, *cache, q_out=out)   # noqa: E731
    for out, name in ((view(b, 1, heads), "q"), (view(b[1:], 0, heads), "q"), (view(b, kv + heads, heads), "v")):
        _refused(lambda: call(out), f"q_out must not share memory with {name}")
    other = q.clone()
    for out, name in ((view(b, heads, heads), "k"), (view(b, heads + 1, heads), "k"), (view(b[1:], heads + kv - 1, heads), "k"), (view(b, heads + kv, heads), "v")):
        _refused(lambda: call(out, q=other), f"q_out must not share memory with {name}")
    _refused(lambda: call(b.as_strided((tokens, heads, dim), (dim * heads, 32, 1)), q=other.clone(), k=k.clone(), v=v.clone()), "elements that share memory")
    tables = torch.zeros(tokens * heads * dim, device=DEV)
    _refused(lambda: call(tables.view(tokens, heads, dim), cos=tables[:8 * dim // 2].view(8, dim // 2)), "with cos")
    assert torch.equal(b, before) and all(torch.equal(s, t) for s, t in zip(cache, kept))
    want = call(None)
    # heads first in memory; by turns with keys and values; in place
    assert torch.equal(call(torch.empty((heads, tokens, dim), device=DEV).transpose(0, 1)), want)
    wide = torch.zeros((tokens, (heads + 2 * kv + heads) * dim), device=DEV)
    wide[:, :(heads + 2 * kv) * dim] = b[:tokens, :(heads + 2 * kv) * dim]
    parts = [view(wide, 0, heads), view(wide, heads, kv), view(wide, heads + kv, kv), view(wide, heads + 2 * kv, heads)]
    assert torch.equal(call(parts[3], q=parts[0], k=parts[1], v=parts[2]), want) and torch.equal(parts[0], q)
    assert call(q) is q and torch.equal(q, want)
