"""orthogonalize and muon_step against plain binary64 Newton-Schulz steps.

Tolerances, before any run.  In F16 precision every step rounds X, A and B to
binary16, a relative error of at most 2^-11 (2^-11/sqrt(3) in the mean square)
per element.  The roundings of 5 steps add in squares: sqrt(15) 2^-11 /
sqrt(3) = 1.1e-3 of the Frobenius norm, if each were carried to the end
unchanged; directions with small singular values are raised by up to 3.4 per
step and carry more.  The inputs (a few strong directions over noise that
holds a fifth of the energy) keep that factor below 4: 4.4e-3.  Coming out in
bfloat16 adds 2^-9.  SPLIT operands hold 22 bits: the same sum at 2^-22 is
2e-6; binary32 accumulation over up to 1031 terms adds at most as much again
per product: 2e-5 covers both."""
import math

import pytest
import torch

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.muon import Muon, muon_step, orthogonalize, workspace_bytes

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)
F16_TOL = 4.4e-3
SPLIT_TOL = 2e-5
BF16 = 2.0 ** -9


def schulz64(g, coefs=(COEF,) * 5, eps=1e-7):
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.mT if tall else x
    x = x / (x.norm() + eps)
    for a, b, c in coefs:
        m = x @ x.mT.contiguous()
        x = a * x + (b * m + c * m @ m) @ x
    return x.mT if tall else x


def gradient(r, c, dtype, seed=0, scale=1e-3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = min(4, r, c)
    strong = torch.randn(r, k, generator=g, device="cuda") @ torch.randn(k, c, generator=g, device="cuda")
    noise = torch.randn(r, c, generator=g, device="cuda")
    return ((strong * (2 / math.sqrt(k)) + noise) * scale).to(dtype)


def off(a, b):
    a, b = a.double(), b.double()
    return float((a - b).norm() / b.norm())


SHAPES = [(1, 1), (1, 7), (9, 1), (3, 1000), (16, 16), (63, 65), (64, 64), (65, 63), (128, 257), (257, 128),
          (300, 300), (515, 1031), (768, 256), (100, 2049)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_orthogonalize(shape, dtype):
    print(f"[muon] orthogonalize {shape} {dtype}", flush=True)
    g = gradient(*shape, dtype)
    keep = g.clone()
    o = orthogonalize(g)
    assert o.dtype == dtype and torch.equal(g, keep)
    tol = SPLIT_TOL if dtype == torch.float32 else F16_TOL + BF16
    assert off(o, schulz64(g)) < tol


@pytest.mark.parametrize("shape", [(600, 900), (900, 600), (1025, 1025)], ids=str)
@pytest.mark.parametrize("precision,tol", [("f16", F16_TOL), ("split", SPLIT_TOL)])
def test_precisions_at_larger_sizes(shape, precision, tol):
    """Binary32 in and out; sizes whose products use the larger tiles too."""
    print(f"[muon] {shape} {precision}", flush=True)
    g = torch.stack([gradient(*shape, torch.float32, i) for i in range(12)])
    o = orthogonalize(g, precision=precision)
    for i in (0, 5, 11):
        assert off(o[i], schulz64(g[i])) < tol


def test_large_tiles():
    print("[muon] 2300 x 2500, four of them", flush=True)
    g = torch.stack([gradient(2300, 2500, torch.bfloat16, i) for i in range(4)])
    o = orthogonalize(g)
    for i in (0, 3):
        assert off(o[i], schulz64(g[i])) < F16_TOL + BF16


# between them, every tile of every product in both precisions, with sizes that
# end inside a tile
TILED = [("f16", (194, 209), 54), ("f16", (132, 167), 88), ("f16", (67, 332), 87), ("f16", (455, 461), 33),
         ("f16", (133, 406), 78), ("split", (336, 365), 76), ("split", (321, 338), 50), ("split", (65, 584), 80),
         ("split", (132, 1318), 25)]


@pytest.mark.parametrize("precision,shape,count", TILED, ids=str)
def test_many_matrices(precision, shape, count):
    print(f"[muon] {count} of {shape} {precision}", flush=True)
    for r, c in (shape, shape[::-1]):
        g = torch.stack([gradient(r, c, torch.float32, i) for i in range(count)])
        o = orthogonalize(g, precision=precision)
        worst = max(off(o[i], schulz64(g[i])) for i in range(count))
        assert worst < (F16_TOL if precision == "f16" else SPLIT_TOL)


def test_own_coefficients_and_steps():
    print("[muon] coefficients", flush=True)
    g = gradient(130, 200, torch.float32)
    per_step = ((4.0, -6.0, 3.0), (2.0, -1.5, 0.5), (1.5, -0.5, 0.0))
    assert off(orthogonalize(g, steps=3, coefficients=per_step, eps=1e-3),
               schulz64(g, per_step, 1e-3)) < SPLIT_TOL
    assert off(orthogonalize(g, steps=1), schulz64(g, (COEF,))) < SPLIT_TOL


def test_strides_and_in_place():
    """Row strides, odd starts, a stack of four dimensions, out = grad."""
    print("[muon] strides", flush=True)
    for dtype, tol in ((torch.float32, SPLIT_TOL), (torch.bfloat16, F16_TOL + BF16)):
        store = gradient(80, 161, dtype)
        for view in (store[:70, 3:130], store[5:, 8:72], store[::2, 1:100]):
            big = torch.full((view.shape[0], view.shape[1] + 5), 7.0, dtype=dtype, device="cuda")
            out = big[:, 2:2 + view.shape[1]]
            orthogonalize(view, out=out)
            assert off(out, schulz64(view)) < tol
            assert bool((big[:, :2] == 7).all()) and bool((big[:, 2 + view.shape[1]:] == 7).all())
        one = gradient(20, 30, dtype)
        assert torch.equal(*orthogonalize(one.expand(2, 20, 30)))      # read twice: fine
        four = torch.stack([gradient(20, 30, dtype, i) for i in range(6)]).view(2, 3, 20, 30)
        want = schulz64(four[1, 2].clone())
        assert orthogonalize(four, out=four) is four
        assert off(four[1, 2], want) < tol


def test_values_out_of_the_ordinary():
    """Zeros, tiny and huge gradients; NaN and infinities stay in their matrix."""
    print("[muon] values", flush=True)
    assert bool((orthogonalize(torch.zeros(40, 70, device="cuda")) == 0).all())
    g = gradient(40, 70, torch.float32)
    want = schulz64(g, eps=0.0)
    for s in (1e30, 1e-30):
        assert off(orthogonalize(g * s, eps=1e-300), want) < SPLIT_TOL
    stack = torch.stack([g, g, g, g])
    stack[1, 3, 4] = math.nan
    stack[2, 39, 69] = math.inf
    o = orthogonalize(stack)
    assert bool(o[1].isnan().all()) and bool(o[2].isnan().all())
    assert torch.equal(o[0], o[3]) and off(o[0], schulz64(g)) < SPLIT_TOL


def test_the_same_bits_in_any_company():
    """A matrix gives the same bits alone, in a list, in a workspace that
    forces small batches, and on another stream."""
    print("[muon] batches", flush=True)
    shapes = [(64, 64), (70, 200), (200, 70), (64, 64), (33, 500)] + [(8 * i, 100) for i in range(1, 9)] + [(48, 48)] * 70
    params = [gradient(*s, torch.float32, i) for i, s in enumerate(shapes)]
    grads = [gradient(*s, torch.float32, 100 + i) for i, s in enumerate(shapes)]

    def step(which, **kw):
        ps = [params[i].clone() for i in which]
        vs = [torch.zeros_like(p) for p in ps]
        muon_step(ps, [grads[i] for i in which], vs, lr=0.1, weight_decay=0.1, **kw)
        return ps, vs

    whole, vs = step(range(len(shapes)))
    least, useful = workspace_bytes(shapes, torch.float32)
    assert least < useful
    tight, _ = step(range(len(shapes)), workspace=torch.empty(least, dtype=torch.uint8, device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other, _ = step(range(len(shapes)))
    torch.cuda.synchronize()
    for i in range(len(shapes)):
        assert torch.equal(whole[i], tight[i]) and torch.equal(whole[i], other[i]), shapes[i]
    for i in (0, 1, 2, 4, 20):
        alone, _ = step([i])
        assert off(alone[0] - params[i], whole[i] - params[i]) < SPLIT_TOL, shapes[i]


@pytest.mark.parametrize("dtype,vdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32),
                                          (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("scale", ["match_rms", "spectral", "none"])
def test_muon_step(dtype, vdtype, nesterov, scale):
    """Three steps against the formulas in binary64, each from the tensors as
    the last step left them."""
    print(f"[muon] step {dtype} {vdtype} {nesterov} {scale}", flush=True)
    shapes = [(96, 40), (40, 96), (129, 129)]
    mu, lr, wd = 0.9, 0.05, 0.1
    ps = [gradient(*s, dtype, 7 + i, 0.5) for i, s in enumerate(shapes)]
    vs = [torch.zeros(s, dtype=vdtype, device="cuda") for s in shapes]
    for t in range(3):
        gs = [gradient(*s, dtype, 10 * t + i) for i, s in enumerate(shapes)]
        before = [(p.double().clone(), v.double().clone()) for p, v in zip(ps, vs)]
        muon_step(ps, gs, vs, lr=lr, momentum=mu, nesterov=nesterov, weight_decay=wd, scale=scale)
        for p, v, g, (p0, v0) in zip(ps, vs, gs, before):
            r, c = p.shape
            s = {"match_rms": 0.2 * max(r, c) ** 0.5, "spectral": max(1, r / c) ** 0.5, "none": 1.0}[scale]
            v1 = mu * v0 + (1 - mu) * g.double()
            u = mu * v1 + (1 - mu) * g.double() if nesterov else v1
            # momentum: binary32 arithmetic, then one rounding
            assert off(v, v1) < (3e-7 if vdtype == torch.float32 else BF16)
            move = lr * s * schulz64(u)
            err = (p.double() - ((1 - lr * wd) * p0 - move)).norm()
            tol = SPLIT_TOL if dtype == torch.float32 else F16_TOL
            rounding = 2.0 ** -23 if dtype == torch.float32 else BF16
            assert float(err) < tol * float(move.norm()) + rounding * float(p.double().norm())


# few rows against a long side: X X^T's sums are taken in runs (of at most
# 1152 terms here, no more than SPLIT_TOL covers) and joined
LONG = [(1, 20000), (2, 4097), (16, 11008), (64, 8192), (70, 9001), (200, 6100), (257, 2500), (520, 7777)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", LONG, ids=str)
def test_long_sides(shape, dtype):
    print(f"[muon] long {shape} {dtype}", flush=True)
    for s in (shape, shape[::-1]):
        g = gradient(*s, dtype)
        a, b = orthogonalize(g), orthogonalize(g)
        assert torch.equal(a, b)
        assert off(a, schulz64(g)) < (SPLIT_TOL if dtype == torch.float32 else F16_TOL + BF16), s


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_sides_among_others(dtype):
    """One list, whose shapes take different numbers of runs, in the useful
    workspace and in the least; scratch of any content."""
    print(f"[muon] long sides among others {dtype}", flush=True)
    shapes = [(16, 9000), (40, 40), (9000, 16), (16, 9000), (130, 3000), (64, 4096), (1, 5000), (300, 300)]
    lo, hi = workspace_bytes(shapes, dtype)
    tol = SPLIT_TOL if dtype == torch.float32 else F16_TOL
    rounding = 2.0 ** -23 if dtype == torch.float32 else BF16
    for size in (hi, lo):
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        ps = [gradient(*s, dtype, 3 + i, 0.5) for i, s in enumerate(shapes)]
        gs = [gradient(*s, dtype, 30 + i) for i, s in enumerate(shapes)]
        vs = [torch.zeros(s, device="cuda") for s in shapes]
        before = [p.double().clone() for p in ps]
        muon_step(ps, gs, vs, lr=0.1, momentum=0.5, nesterov=False, scale="none", workspace=ws)
        for p, p0, g in zip(ps, before, gs):
            move = 0.1 * schulz64(g)
            err = (p.double() - (p0 - move)).norm()
            assert float(err) < tol * float(move.norm()) + rounding * float(p.double().norm()), tuple(p.shape)


def test_graph_replays():
    """Captured, the call replays on what the buffers then hold."""
    print("[muon] graph", flush=True)
    p, v = gradient(130, 70, torch.float32, 1, 0.5), torch.zeros(130, 70, device="cuda")
    g = gradient(130, 70, torch.float32, 2)
    ws = torch.empty(workspace_bytes([(130, 70)], torch.float32)[1], dtype=torch.uint8, device="cuda")
    p0, v0 = p.clone(), v.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        muon_step([p], [g], [v], lr=0.1, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    p.copy_(p0), v.copy_(v0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        muon_step([p], [g], [v], lr=0.1, workspace=ws)
    p.copy_(p0), v.copy_(v0)
    q, w = p0.clone(), v0.clone()
    for t in range(4):
        g.copy_(gradient(130, 70, torch.float32, 20 + t))
        graph.replay()
        muon_step([q], [g], [w], lr=0.1)
        torch.cuda.synchronize()
        assert torch.equal(p, q) and torch.equal(v, w), t


def test_optimizer_and_checkpoint():
    print("[muon] optimizer", flush=True)

    def model(seed):
        torch.manual_seed(seed)
        return [torch.nn.Parameter(torch.randn(s, device="cuda", dtype=torch.bfloat16) * 0.1)
                for s in ((40, 24), (3, 24, 40))]

    def grads(ps, t):
        for i, p in enumerate(ps):
            p.grad = torch.randn(p.shape, generator=torch.Generator(device="cuda").manual_seed(9 * t + i),
                                 device="cuda").to(p.dtype)

    a = model(0)
    opt = Muon(a, lr=0.02, weight_decay=0.01, momentum_dtype=torch.float32)
    by_hand = [p.detach().clone() for p in a]
    momenta = [torch.zeros(p.shape, device="cuda") for p in a]
    for t in range(3):
        grads(a, t)
        opt.step()
        muon_step(by_hand, [p.grad for p in a], momenta, lr=0.02, weight_decay=0.01)
    assert all(torch.equal(p.detach(), q) for p, q in zip(a, by_hand))
    assert opt.state_bytes() == 4 * sum(p.numel() for p in a)
    b = [torch.nn.Parameter(p.detach().clone()) for p in a]
    opt_b = Muon(b, lr=0.5)
    opt_b.load_state_dict(opt.state_dict())
    assert opt_b.state[b[0]]["momentum"].dtype == torch.float32
    for t in range(3, 5):
        grads(a, t), grads(b, t)
        opt.step(), opt_b.step()
    assert all(torch.equal(p.detach(), q.detach()) for p, q in zip(a, b))


def test_refusals_with_tensors():
    g = gradient(8, 8, torch.float32)
    with pytest.raises(TypeError):
        orthogonalize(g.half())
    with pytest.raises(ValueError):
        orthogonalize(g[0])
    with pytest.raises(ValueError):
        orthogonalize(g.t()[:, :4])
    with pytest.raises(ValueError):
        orthogonalize(g, out=torch.empty(8, 9, device="cuda"))
    with pytest.raises(ValueError):
        orthogonalize(g.cpu())
    with pytest.raises(ma.MicroAdamError) as e:
        orthogonalize(g, workspace=torch.empty(4096, dtype=torch.uint8, device="cuda"))
    assert e.value.code == ma.MICROADAM_ERR_STATE_SIZE
    v = torch.zeros_like(g)
    with pytest.raises(ValueError):
        orthogonalize(torch.stack([g, g]), out=g.clone().expand(2, 8, 8))
    with pytest.raises(ValueError):
        muon_step([g], [g], [v, v], lr=0.1)
    with pytest.raises(ValueError):
        muon_step([g], [g[:4]], [v], lr=0.1)
    with pytest.raises(TypeError):
        muon_step([g, g.bfloat16()], [g, g], [v, v], lr=0.1)
    with pytest.raises(ma.MicroAdamError):
        muon_step([g], [g], [v], lr=math.inf)
