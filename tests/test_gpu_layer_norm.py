"""layer_norm and its gradients against binary64 on the CPU.

Tolerances, with u = 2^-24.  A row's sums are chains of at most 16 terms, then
a tree of at most 10 levels and a chain of 16 waves: relative errors below 42 u
of the sum of magnitudes.  The variance (a sum of squares) is off by 42 u, r by
half of that and two roundings; the mean's error, in units of 1 / r, by 42 u: h
is off by at most 64 u (1 + |h|) forward.  Backward takes the mean from memory,
rounded: u |m| r more.  Each formula's terms then carry h's error and at most 42 u
of their sums of magnitudes; a result in bfloat16 is rounded by half a step, 2^-8.
"""
import pytest
import torch

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.norm import layer_norm

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
TYPES = {"f32": (torch.float32, torch.float32), "bf16": (torch.bfloat16, torch.bfloat16),
         "bf16_f32": (torch.bfloat16, torch.float32), "f32_bf16": (torch.float32, torch.bfloat16)}


def inputs(rows, cols, types, seed=0, offset=0.5):
    dtype, side = TYPES[types]
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(rows, cols, generator=g, device="cuda") + offset).to(dtype)
    w = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(side)
    b = torch.randn(cols, generator=g, device="cuda").to(side)
    dy = torch.randn(rows, cols, generator=g, device="cuda").to(dtype)
    return x, w, b, dy


def reference(x, w, b, dy, eps):
    """y, dx, dw, db and their tolerances before the last rounding."""
    x, w, b, dy = (t.detach().cpu().double() for t in (x, w, b, dy))
    m, var = x.mean(-1, keepdim=True), x.var(-1, correction=0, keepdim=True)
    r = 1.0 / torch.sqrt(var + eps)
    h = (x - m) * r
    y = h * w + b
    eh = 64 * U * (1 + h.abs())
    ey = eh * w.abs() + 2 * U * y.abs()
    eh = eh + U * m.abs() * r
    g = dy * w
    m1, m2 = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    dx = r * (g - m1 - h * m2)
    e1 = 42 * U * g.abs().mean(-1, keepdim=True)
    e2 = 42 * U * (g * h).abs().mean(-1, keepdim=True) + (g.abs() * eh).mean(-1, keepdim=True)
    ex = r * (4 * U * g.abs() + e1 + h.abs() * e2 + eh * m2.abs()) + 32 * U * dx.abs()
    dw, db = (dy * h).sum(0), dy.sum(0)
    chain = (x.shape[0] / 512 + 64) * U
    ew = (dy.abs() * eh).sum(0) + chain * (dy * h).abs().sum(0)
    eb = chain * dy.abs().sum(0)
    return (y, dx, dw, db), (ey, ex, ew, eb)


def check(got, want, tolerance):
    for what, g, w, t in zip(("y", "dx", "dw", "db"), got, want, tolerance):
        off = (g.detach().cpu().double() - w).abs()
        assert bool((off <= t + HALF[g.dtype] * (w.abs() + t)).all()), (what, float((off - t).max()))


def run(x, w, b, dy, eps=1e-5):
    x, w, b = (t.detach().requires_grad_() for t in (x, w, b))
    y = layer_norm(x, w, b, eps=eps)
    assert y.dtype == x.dtype and y.shape == x.shape
    return (y, *torch.autograd.grad(y, (x, w, b), dy))


COLS = [1, 2, 7, 8, 64, 255, 256, 257, 512, 513, 1024, 1031, 2048, 2050, 4096, 4100, 8192, 8200, 16384, 16387, 20001]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_sizes(cols, types):
    print(f"[norm] {cols} {types}", flush=True)
    for rows in (1, 5, 131):
        given = inputs(rows, cols, types, seed=cols)
        got = run(*given)
        check(got, *reference(*given, 1e-5))
        with torch.no_grad():
            assert torch.equal(layer_norm(*given[:3]), got[0])


@pytest.mark.parametrize("types", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(4099, 130), (70001, 3), (3000, 1025), (777, 9001)])
def test_many_rows(rows, cols, types):
    print(f"[norm] {rows} x {cols} {types}", flush=True)
    given = inputs(rows, cols, types)
    check(run(*given), *reference(*given, 1e-5))


@pytest.mark.parametrize("types,rows,cols", [("f32", 33001, 1031), ("bf16", 33001, 2049), ("bf16_f32", 8400, 16384)])
def test_beyond_the_caches(types, rows, cols):
    """Rows of a call over 256 MiB have the bits of a small call's; dw and db are
    the sums over small calls' in binary64 (each within its own tolerance)."""
    print(f"[norm] beyond the caches {rows} x {cols} {types}", flush=True)
    x, w, b, dy = inputs(rows, cols, types)
    y, dx, dw, db = run(x, w, b, dy)
    for at in range(0, rows, rows // 3):
        part = slice(at, at + 300)
        small = run(x[part], w, b, dy[part])
        assert torch.equal(y[part], small[0]) and torch.equal(dx[part], small[1])
    mean = x.double().mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(x.double().var(1, correction=0, keepdim=True) + 1e-5)
    chain = (rows / 512 + 64) * U
    for at in range(0, cols, 256):
        part = slice(at, at + 256)
        h, d = (x[:, part].double() - mean) * rstd, dy[:, part].double()
        eh = 64 * U * (1 + h.abs()) + U * mean.abs() * rstd
        for g, want, t in ((dw[part], (d * h).sum(0), (d.abs() * eh).sum(0) + chain * (d * h).abs().sum(0)),
                           (db[part], d.sum(0), chain * d.abs().sum(0))):
            assert bool(((g.double() - want).abs() <= t + HALF[g.dtype] * (want.abs() + t)).all())


@pytest.mark.parametrize("offset", [-300.0, 1e4])
@pytest.mark.parametrize("cols", [200, 3000, 16500])
def test_a_mean_far_from_zero(cols, offset):
    """Differences to the mean keep the bits that x has."""
    print(f"[norm] offset {offset} cols {cols}", flush=True)
    given = inputs(7, cols, "f32", offset=offset)
    check(run(*given), *reference(*given, 1e-5))


@pytest.mark.parametrize("types", ["f32", "bf16_f32"])
def test_layouts(types):
    """Rows at a stride and at odd addresses, batches, transposed and expanded
    inputs and gradients, strided weights."""
    print(f"[norm] layouts {types}", flush=True)
    x, w, b, dy = inputs(24, 101, types)
    whole = torch.full((24, 120), 7.0, device="cuda", dtype=x.dtype)
    for start in (0, 1, 5):
        view = whole[:, start:start + 101]
        view.copy_(x)
        dview = whole.clone()[:, start:start + 101]
        dview.copy_(dy)
        check(run(view, w, b, dview), *reference(x, w, b, dy, 1e-5))
    base = run(x, w, b, dy)
    same = [(x.view(2, 3, 4, 101), dy.view(2, 3, 4, 101)), (x.t().contiguous().t(), dy.t().contiguous().t()),
            (whole[:, 5:106].view(4, 6, 101), dy.view(4, 6, 101))]
    for xs, dys in same:
        got = run(xs, w, b, dys)
        assert got[0].shape == got[1].shape == xs.shape
        for a, c in zip(got, base):
            assert torch.equal(a.reshape(c.shape), c)
    w2, b2 = torch.stack((w, b), 1).unbind(1)
    for a, c in zip(run(x, w2, b2, dy), base):
        assert torch.equal(a, c)
    one = torch.ones((), device="cuda", dtype=x.dtype).expand(24, 101)
    check(run(x, w, b, one), *reference(x, w, b, one, 1e-5))
    row = x[0].expand(24, 101)
    check(run(row, w, b, dy), *reference(row, w, b, dy, 1e-5))
    check([t.reshape(1, -1) if i < 2 else t for i, t in enumerate(run(x[3], w, b, dy[3]))],
          *reference(x[3:4], w, b, dy[3:4], 1e-5))


def test_without_weight_or_bias():
    print("[norm] no sides", flush=True)
    x, w, b, dy = inputs(9, 300, "bf16")
    ones, zeros = torch.ones_like(w), torch.zeros_like(b)
    assert torch.equal(layer_norm(x), layer_norm(x, ones, zeros))
    assert torch.equal(layer_norm(x, w), layer_norm(x, w, zeros))
    assert torch.equal(layer_norm(x, None, b), layer_norm(x, ones, b))
    leaf = x.clone().requires_grad_()
    assert torch.equal(torch.autograd.grad(layer_norm(leaf), leaf, dy)[0], run(x, ones, zeros, dy)[1])
    for i, pick in enumerate(("x", "w", "b")):      # one gradient alone is the one of all three
        ts = [t.clone() for t in (x, w, b)]
        ts[i].requires_grad_()
        assert torch.equal(torch.autograd.grad(layer_norm(*ts), ts[i], dy)[0], run(x, w, b, dy)[1 + i]), pick
    bias = b.float().requires_grad_()
    assert torch.autograd.grad(layer_norm(x, None, bias), bias, dy)[0].dtype == torch.float32


def test_empty_and_constant():
    print("[norm] empty", flush=True)
    _, w, b, _ = inputs(1, 40, "f32")
    none = torch.empty(0, 40, device="cuda")
    y, dx, dw, db = run(none, w, b, none)
    assert y.shape == dx.shape == (0, 40) and not dw.any() and not db.any() and dw.shape == (40,)
    long = torch.empty(0, 20001, device="cuda")
    assert not any(t.any() for t in run(long, *(torch.ones(20001, device="cuda"),) * 2, long))
    assert layer_norm(torch.empty(3, 0, 40, device="cuda"), w).shape == (3, 0, 40)
    flat = torch.full((3, 40), 1e5, device="cuda")
    y, dx, dw, db = run(flat, w, b, flat)
    assert torch.equal(y, b.expand(3, 40)) and not dw.any()
    assert bool(torch.isfinite(dx).all())


@pytest.mark.parametrize("cols", [100, 2500, 17000])
def test_not_finite(cols):
    """A row with NaN or an infinity leaves the other rows as they are."""
    print(f"[norm] not finite {cols}", flush=True)
    x, w, b, dy = inputs(6, cols, "f32")
    want = run(x, w, b, dy)
    bad = x.clone()
    bad[1, cols // 2], bad[4, 0], bad[3, cols - 1] = float("nan"), float("inf"), -float("inf")
    got = run(bad, w, b, dy)
    for i in range(6):
        for g, t in zip(got[:2], want[:2]):
            assert bool(g[i].isnan().all()) if i in (1, 3, 4) else torch.equal(g[i], t[i])
    assert bool(got[2].isnan().all()) and torch.equal(got[3], want[3])


def test_against_differences():
    """The gradients against central differences of the binary64 formula are
    covered by the formula's; here against differences of the kernel itself:
    steps of 2^-6 of a smooth function whose third derivative is O(1) leave
    2^-13, the kernel's 2^-17 over the step 2^-11."""
    print("[norm] differences", flush=True)
    x, w, b, dy = inputs(2, 33, "f32")
    _, dx, dw, db = run(x, w, b, dy)
    step = 2.0 ** -6
    for t, grad in ((x, dx), (w, dw), (b, db)):
        for i in range(0, t.numel(), 7):
            s = []
            for sign in (1, -1):
                moved = t.clone()
                moved.view(-1)[i] += sign * step
                y = layer_norm(*[moved if k is t else k for k in (x, w, b)])
                s.append(float((y.double() * dy.double()).sum()))
            assert abs((s[0] - s[1]) / (2 * step) - float(grad.reshape(-1)[i])) < 2.0 ** -9


def test_same_bits_and_neighbours():
    print("[norm] same bits", flush=True)
    given = inputs(1001, 519, "bf16")
    first = run(*given)
    for _ in range(3):
        assert all(torch.equal(a, c) for a, c in zip(run(*given), first))
    # a row's results do not go by the batch
    alone = run(given[0][5:6], given[1], given[2], given[3][5:6])
    assert torch.equal(alone[0], first[0][5:6]) and torch.equal(alone[1], first[1][5:6])


def test_graph_and_streams():
    print("[norm] graph", flush=True)
    x, w, b, dy = inputs(300, 515, "f32")
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]

    def step():
        y = layer_norm(*leaves)
        return (y, *torch.autograd.grad(y, leaves, dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for seed in range(4):
        x2, w2, b2, dy2 = inputs(300, 515, "f32", seed=seed + 1)
        with torch.no_grad():
            for t, n in zip((*leaves, dy), (x2, w2, b2, dy2)):
                t.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(captured, run(x2, w2, b2, dy2)))


def test_refusals():
    print("[norm] refusals", flush=True)
    x, w, b, _ = inputs(4, 8, "f32")
    for args, kind in (((x.half(),), TypeError), ((x.cpu(),), ValueError), ((x, w.half()), TypeError),
                       ((x, w, b.bfloat16()), TypeError), ((x, w[:7]), ValueError), ((x, w.cpu()), ValueError),
                       ((x, None, b.view(1, 8)), ValueError), ((x[0, 0],), ValueError), ((x[:, :0],), ValueError)):
        with pytest.raises(kind):
            layer_norm(*args)
    for eps in (-1e-5, float("nan"), float("inf"), 1e39):
        with pytest.raises(ma.MicroAdamError):
            layer_norm(x, eps=eps)
    leaf = x.clone().requires_grad_()
    y = layer_norm(leaf, w, b)
    (g,) = torch.autograd.grad(y, leaf, torch.ones_like(y), create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
    import torch.autograd.forward_ad as forward_ad
    with forward_ad.dual_level(), pytest.raises(NotImplementedError):
        layer_norm(forward_ad.make_dual(x, x), w)
    y = layer_norm(leaf * 1.0, w)
    saved = leaf * 2.0
    y = layer_norm(saved, w)
    saved.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
