"""grad_norm, clip_grads and clip_grad_norm against binary64 on the CPU.

Tolerances.  The norm is summed in binary64 and rounded once to binary32: half
a step, 2^-24.  A scaled binary32 gradient is rounded once, 2^-24; a bfloat16 one
to binary32 and then to bfloat16, 2^-24 + 2^-8.  Binary64's own errors (sums of
at most 2^24 terms in blocks: below 2^-40) go into the factor 1 + 2^-10.
"""
import math

import pytest
import torch

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.clip import clip_grad_norm, clip_grads, grad_norm, workspace_bytes

pytestmark = pytest.mark.gpu

SLACK = 1.0 + 2.0 ** -10
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -24 + 2.0 ** -8}


def reference_norm(grads):
    return math.sqrt(sum(float(g.detach().cpu().double().square().sum()) for g in grads))


def check_norm(got, want):
    assert got.dtype == torch.float32 and got.shape == ()
    assert abs(float(got) - want) <= want * 2.0 ** -24 * SLACK, (float(got), want)


def check_scaled(after, before, factor):
    for a, b in zip(after, before):
        want = b.cpu().double() * factor
        # (a result below the type's normal range: half a step there)
        floor = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134}[a.dtype]
        off = (a.cpu().double() - want).abs()
        assert bool((off <= want.abs() * HALF[a.dtype] * SLACK + floor).all())


def bucket(shapes, dtype, seed=0, start=0, scale=1e-2):
    """Gradients one behind the other in one buffer, from element `start`."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = sum(math.prod(s) for s in shapes)
    flat = (torch.randn(start + n + 5, generator=g, device="cuda") * scale).to(dtype)
    views, at = [], start
    for s in shapes:
        views.append(flat[at:at + math.prod(s)].view(s))
        at += math.prod(s)
    return flat, views


LISTS = {
    "one": [(1,)], "scalar": [()], "empty_among": [(0,), (5,), (0, 3), (1,)], "pieces": [(7,), (8,), (9,), (15,)],
    "chunk": [(16384,), (16385,), (8192,), (8193,), (8191,)], "odd": [(517, 1231), (33,), (3, 3, 3), (70001,)],
    "many": [(i % 37 + 1,) for i in range(500)], "launch": [(11,)] * 160, "launch_and_one": [(11,)] * 161,
    "large": [(2100, 4099), (1,)],
}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("start", [0, 1, 3])
@pytest.mark.parametrize("name", LISTS)
def test_lists(name, start, dtype):
    print(f"[clip] {name} start {start} {dtype}", flush=True)
    flat, grads = bucket(LISTS[name], dtype, start=start)
    before, whole = [g.clone() for g in grads], flat.clone()
    want = reference_norm(before)
    check_norm(grad_norm(grads), want)
    assert torch.equal(flat, whole)
    # a limit above: nothing is written
    check_norm(clip_grads(grads, want * 1.01 + 1e-5), want)
    assert torch.equal(flat, whole)
    limit = 0.37 * want
    check_norm(clip_grads(grads, limit), want)
    check_scaled(grads, before, limit / (want + 1e-6))
    # what is beside the list stays as it was
    assert torch.equal(flat[:start], whole[:start]) and torch.equal(flat[-5:], whole[-5:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_beyond_the_caches(dtype):
    """More than 256 MiB, tensors of all ends among them; above the limit and below."""
    print(f"[clip] beyond the caches {dtype}", flush=True)
    wide = 9001 if dtype == torch.float32 else 18001
    flat, grads = bucket([(3,), (8009, wide), (8193,), (1,), (16385,), (40000, 7)], dtype, start=1)
    before, whole = [g.clone() for g in grads], flat.clone()
    want = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    check_norm(grad_norm(grads), want)
    check_norm(clip_grads(grads, 2.0 * want), want)
    assert torch.equal(flat, whole)
    check_norm(clip_grads(grads, 0.37 * want), want)
    factor = 0.37 * want / (want + 1e-6)
    for a, b in zip(grads, before):
        for x, y in zip(a.reshape(-1).split(1 << 24), b.reshape(-1).split(1 << 24)):
            exact = y.double() * factor
            floor = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134}[dtype]
            assert bool(((x.double() - exact).abs() <= exact.abs() * HALF[dtype] * SLACK + floor).all())
    assert torch.equal(flat[:1], whole[:1]) and torch.equal(flat[-5:], whole[-5:])
    again = whole.clone()
    views, at = [], 1
    for g in before:
        views.append(again[at:at + g.numel()].view(g.shape))
        at += g.numel()
    clip_grads(views, 0.37 * want)
    assert torch.equal(again, flat)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_more_than_the_caches_hold(dtype):
    """A list of 300 MB, in binary64 on the device."""
    print(f"[clip] 300 MB {dtype}", flush=True)
    n = 300_000_000 // dtype.itemsize
    flat, grads = bucket([(n // 3,), (7,), (n - n // 3 - 7,)], dtype, start=1)
    before = flat.clone()
    want = math.sqrt(sum(float(p.double().square().sum()) for p in before[1:-5].split(1 << 26)))
    limit = 0.3 * want
    check_norm(grad_norm(grads), want)
    check_norm(clip_grads(grads, limit), want)
    factor = limit / (want + 1e-6)
    for a, b in zip(flat[1:-5].split(1 << 26), before[1:-5].split(1 << 26)):
        exact = b.double() * factor
        assert bool(((a.double() - exact).abs() <= exact.abs() * HALF[dtype] * SLACK + 2.0 ** -134).all())
    assert torch.equal(flat[:1], before[:1]) and torch.equal(flat[-5:], before[-5:])


def test_mixed_types_and_orders():
    """Both dtypes in one list, transposed gradients, gradients in any order of
    addresses."""
    print("[clip] mixed", flush=True)
    a, (a1, a2) = bucket([(65, 300), (129,)], torch.bfloat16, seed=1, start=1)
    b, (b1, b2, b3) = bucket([(31, 17, 5), (4097,), (1,)], torch.float32, seed=2)
    c = bucket([(40, 60)], torch.float32, seed=3)[1][0].t()
    grads = [b3, a2, c, b1.permute(2, 0, 1), a1, b2]
    before = [g.clone() for g in grads]
    want = reference_norm(grads)
    check_norm(clip_grads(iter(grads), 0.1), want)
    check_scaled(grads, before, 0.1 / (want + 1e-6))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-36, 1e-22, 1e22, 1e36])
def test_far_from_one(scale, dtype):
    """Squares that binary32 cannot hold."""
    print(f"[clip] scale {scale} {dtype}", flush=True)
    _, grads = bucket([(1000, 7)], dtype, scale=scale)
    before, want = [g.clone() for g in grads], reference_norm(grads)
    check_norm(grad_norm(grads), want)
    limit = want / 64
    check_norm(clip_grads(grads, limit, eps=0.0), want)
    check_scaled(grads, before, limit / want)
    grads = [torch.full((5,), 3e38, device="cuda")]           # a norm beyond binary32
    assert math.isinf(float(clip_grads(grads, 1.0)))
    check_scaled(grads, [torch.full((5,), 3e38)], 1.0 / (float(torch.tensor(3e38, dtype=torch.float32)) * 5 ** 0.5))


def test_not_finite():
    print("[clip] not finite", flush=True)
    for dtype in (torch.float32, torch.bfloat16):
        _, grads = bucket([(5000,), (3,)], dtype)
        grads[0][4999] = math.inf
        assert float(grad_norm(grads)) == math.inf
        assert float(clip_grads(grads, 1.0)) == math.inf
        assert bool(grads[0][4999].isnan()) and not grads[0][:4999].any() and not grads[1].any()
        _, grads = bucket([(5000,), (3,)], dtype)
        grads[1][1] = math.nan
        assert math.isnan(float(clip_grads(grads, 1.0)))
        assert all(bool(g.isnan().all()) for g in grads)
        _, grads = bucket([(50,)], dtype)
        grads[0][7] = -math.inf
        same = grads[0].clone()
        clip_grads(grads, math.inf)
        assert torch.equal(grads[0], same)


def test_limits():
    print("[clip] limits", flush=True)
    _, grads = bucket([(300,)], torch.float32)
    clip_grads(grads, 0.0)
    assert not grads[0].any()
    check_norm(clip_grads(grads, 0.0, eps=0.0), 0.0)
    assert not grads[0].any()                                 # and no NaN of 0 / 0
    check_norm(grad_norm([torch.zeros(0, device="cuda")]), 0.0)
    check_norm(clip_grads([torch.zeros(0, device="cuda")], 1.0), 0.0)
    for bad in (-1.0, math.nan):
        with pytest.raises(ma.MicroAdamError):
            clip_grads(grads, bad)
    for bad in (-1.0, math.nan, math.inf):
        with pytest.raises(ma.MicroAdamError):
            clip_grads(grads, 1.0, eps=bad)


def test_refusals():
    print("[clip] refusals", flush=True)
    x = torch.randn(64, 64, device="cuda")
    for f in (grad_norm, lambda g, **k: clip_grads(g, 1.0, **k)):
        for bad, kind in (([], ValueError), ([x.cpu()], ValueError), ([x.half()], TypeError), ([x, x.double()], TypeError),
                          ([x, torch.ones(2)], ValueError), ([x[:, :3]], ValueError), ([x[0].expand(3, 64)], ValueError),
                          ([x.clone().requires_grad_()], NotImplementedError)):
            with pytest.raises(kind):
                f(bad)
        for ws in (torch.empty(workspace_bytes(), dtype=torch.uint8), torch.empty(1 << 20, device="cuda"),
                   torch.empty(2 * workspace_bytes(), dtype=torch.uint8, device="cuda")[::2]):
            with pytest.raises(ValueError):
                f([x], workspace=ws)
        with pytest.raises(ma.MicroAdamError):
            f([x], workspace=torch.empty(workspace_bytes() - 1, dtype=torch.uint8, device="cuda"))
    same = x.clone()
    for twice in ([x, x], [x, x[3]], [x[1:], x[:2]], [x, x.view(-1)[5:6]]):
        grad_norm(twice)
        with pytest.raises(ma.MicroAdamError, match="overlap"):
            clip_grads(twice, 1e-3)
    with pytest.raises(ma.MicroAdamError, match="workspace"):
        clip_grads([x], 1e-3, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    whole = torch.zeros(workspace_bytes() + 64, dtype=torch.uint8, device="cuda")
    with pytest.raises(ma.MicroAdamError, match="workspace"):
        clip_grads([whole[:64].view(torch.float32)], 1.0, workspace=whole)
    assert torch.equal(x, same)


def test_versions_and_parameters():
    print("[clip] versions", flush=True)
    w = [torch.nn.Parameter(torch.randn(30, 20, device="cuda")), torch.nn.Parameter(torch.randn(7, device="cuda")),
         torch.nn.Parameter(torch.randn(9, device="cuda"))]
    loss = (w[0].sum() * 3.0).square() + w[1].square().sum()
    loss.backward()
    grads, before = [w[0].grad, w[1].grad], [w[0].grad.clone(), w[1].grad.clone()]
    want, versions = reference_norm(grads), [g._version for g in grads]
    check_norm(clip_grad_norm(w, 0.5), want)
    assert w[2].grad is None and [g._version for g in grads] == [v + 1 for v in versions]
    check_scaled(grads, before, 0.5 / (want + 1e-6))
    check_norm(clip_grad_norm(w[1], 1e9), reference_norm([w[1].grad]))
    check_norm(clip_grad_norm([w[2]], 1.0), 0.0)
    check_norm(clip_grad_norm([], 1.0), 0.0)


def test_same_bits():
    print("[clip] same bits", flush=True)
    got = []
    for _ in range(3):
        flat, grads = bucket([(3000, 1001), (17,), (100001,)], torch.bfloat16, start=3)
        got.append((clip_grads(grads, 0.01), flat))
    assert all(torch.equal(n, got[0][0]) and torch.equal(f, got[0][1]) for n, f in got[1:])


def test_graphs_and_streams():
    """Two captured graphs that share a workspace on one stream, replayed with
    new gradients, and calls on two streams at once."""
    print("[clip] graphs", flush=True)
    ws = torch.empty(workspace_bytes(), dtype=torch.uint8, device="cuda")
    sets = [bucket([(513, 77), (1001,)], d, start=1) for d in (torch.float32, torch.bfloat16)]
    side = torch.cuda.Stream()
    graphs, norms = [], []
    for _, grads in sets:
        with torch.cuda.stream(side):
            clip_grads(grads, 1e9, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            norms.append(clip_grads(grads, 0.05, workspace=ws))
        graphs.append(graph)
    for seed in range(4):
        for (flat, grads), graph, norm in zip(sets, graphs, norms):
            flat.copy_(torch.randn(flat.shape, device="cuda") * 10.0 ** -seed)
            eager = [g.clone() for g in grads]
            want = clip_grads(eager, 0.05)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(norm, want) and all(torch.equal(a, b) for a, b in zip(grads, eager))
    a, b = bucket([(2048, 2048)], torch.float32, seed=5), bucket([(2048, 2047)], torch.float32, seed=6)
    wants = [reference_norm(x[1]) for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for x, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            got.append(clip_grads(x[1], 0.5))
    torch.cuda.synchronize()
    for n, want in zip(got, wants):
        check_norm(n, want)
