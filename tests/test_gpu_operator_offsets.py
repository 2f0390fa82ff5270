"""Operands whose elements lie more than 2^32 bytes apart, against copies that do
not."""
import pytest
import torch

from paper_2405_15593_amd.attention import attention
from paper_2405_15593_amd.clip import clip_grads, grad_norm
from paper_2405_15593_amd.norm import layer_norm

pytestmark = pytest.mark.gpu

FAR = (1 << 31) + 1000   # elements of bfloat16: 2^32 bytes and more


@pytest.fixture(scope="module")
def room():
    store = torch.empty(2 * FAR + (1 << 20), dtype=torch.bfloat16, device="cuda")
    yield store
    del store
    torch.cuda.empty_cache()


def spread(room, shape, strides, start, seed):
    t = room.as_strided(shape, strides, start)
    t.copy_(torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
    return t


@pytest.mark.parametrize("queries", [1, 70])
@pytest.mark.parametrize("far", ["sequences", "positions", "heads"])
def test_attention(room, far, queries):
    print(f"[offsets] attention {far} {queries}", flush=True)
    b, s, h, d = (2, 300, 2, 64) if far != "positions" else (1, 300, 2, 64)
    strides = {"sequences": (FAR, 256, 128, 1), "positions": (0, 1 << 23, 128, 1), "heads": (300 * 128, 128, FAR, 1)}[far]
    k = spread(room, (b, s, h, d), strides, 0, 1)
    v = spread(room, (b, s, h, d), strides, 64 if far != "heads" else 1 << 19, 2)
    q = torch.randn(b, queries, 4, d, device="cuda").bfloat16()
    dout = torch.randn_like(q)
    results = []
    for kk, vv in ((k, v), (k.contiguous(), v.contiguous())):
        leaves = [t.detach().requires_grad_() for t in (q, kk, vv)]
        out = attention(*leaves, causal=queries > 1)
        results.append((out, *torch.autograd.grad(out, leaves, dout)))
    assert all(torch.equal(a, w) for a, w in zip(*results))


@pytest.mark.parametrize("cols", [1000, 1001, 20001])
def test_layer_norm(room, cols):
    print(f"[offsets] layer norm {cols}", flush=True)
    x = spread(room, (3, cols), (FAR, 1), 0, cols)
    dy = spread(room, (3, cols), (FAR, 1), 1 << 19, cols + 1)
    w, b = torch.randn(2, cols, device="cuda")
    results = []
    for xx, dd in ((x, dy), (x.contiguous(), dy.contiguous())):
        leaves = [t.detach().requires_grad_() for t in (xx, w, b)]
        y = layer_norm(*leaves)
        results.append((y, *torch.autograd.grad(y, leaves, dd)))
    assert all(torch.equal(a, c) for a, c in zip(*results))


def test_clipping(room):
    """One tensor of 2^32 bytes and more; the norm to its half step, of values that
    are all one, and every element scaled."""
    print("[offsets] clipping", flush=True)
    g = room[:FAR]
    g.fill_(1.0)
    room[FAR:FAR + 8] = 3.0
    want = float(FAR) ** 0.5
    assert abs(float(grad_norm([g])) - want) <= want * 2.0 ** -24 * 1.001
    clip_grads([g], 0.5 * want, eps=0.0)
    assert float(g[0]) == 0.5 and float(g[-1]) == 0.5
    assert all(bool((part == 0.5).all()) for part in g.split(1 << 28))
    assert bool((room[FAR:FAR + 8] == 3.0).all())
