"""token_logprobs and token_logprobs_and_grad against plain binary64 formulas.

Tolerances, before any run.  The sums over up to 70,000 binary32 terms are
tree sums over threads with chains of at most 64 in each: relative error below
1e-5; exponents carry |d| 2^-23 with |d| < 100 where it matters: 1e-5.  So
logp, entropy and the alternatives are within 2e-5 (1 + |value|).  A binary32
gradient row is within 4e-5 of its largest element, a bfloat16 one rounds each
element by at most 2^-8 of itself on top."""
import math

import pytest
import torch

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.logprobs import token_logprobs, token_logprobs_and_grad

pytestmark = pytest.mark.gpu

NINF = -math.inf
TOL = 2e-5


def logits_of(rows, vocab, dtype, seed=0, pad=0, scale=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(rows, vocab + pad, generator=g, device="cuda") * scale).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    return x[:, :vocab], t


def exact(x, t, temperature=1.0, ignore=-100):
    z = x.double() / temperature
    top = z.amax(1, keepdim=True)
    d = z - torch.where(top == NINF, 0.0, top)
    e = d.exp()
    s = e.sum(1, keepdim=True)
    some = s > 0
    lp = torch.where(some, d - torch.where(some, s, 1.0).log(), NINF)
    p = torch.where(some, e / torch.where(some, s, 1.0), 0.0)
    h = -(p * torch.where(p > 0, lp, 0.0)).sum(1)
    live = t != ignore
    logp = lp.gather(1, torch.where(live, t, 0)[:, None])[:, 0]
    return lp, p, torch.where(live, logp, 0.0), torch.where(live, h, 0.0), live


def exact_grad(x, t, gp, gh, temperature=1.0, ignore=-100):
    lp, p, _, h, live = exact(x, t, temperature, ignore)
    onehot = torch.zeros_like(p)
    onehot.scatter_(1, torch.where(live, t, 0)[:, None], 1.0)
    g = gp.double()[:, None] * (onehot - p)
    if gh is not None:
        g = g - gh.double()[:, None] * torch.where(p > 0, p * (lp + h[:, None]), 0.0)
    use = live & (p.sum(1) > 0)
    return torch.where(use[:, None], g / temperature, 0.0)


def close(a, b, tol=TOL):
    a, b = a.double(), b.float().double()   # a value beyond binary32 rounds to an infinity
    same = (a == b) | (a.isnan() & b.isnan())
    return bool((same | ((a - b).abs() <= tol * (1 + b.abs()))).all())


def check_values(x, t, k=0, temperature=1.0):
    r = token_logprobs(x, t, top_k=k, temperature=temperature)
    lp, _, logp, h, live = exact(x, t, temperature)
    assert close(r.logp, logp) and close(r.entropy, h)
    if k:
        # ties by index: a stable descending sort of the logits
        order = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :k]
        order = torch.where(live[:, None], order, -1)
        assert torch.equal(r.top_indices, order)
        want = torch.where(live[:, None], lp.gather(1, order.clamp_min(0)), 0.0)
        assert close(r.top_logprobs, want)
    return r


def check_grad(x, t, gp, gh, temperature=1.0, **kw):
    r = token_logprobs_and_grad(x, t, gp, gh, temperature=temperature, **kw)
    _, _, logp, h, _ = exact(x, t, temperature)
    want = exact_grad(x, t, gp, gh, temperature)
    assert close(r.logp, logp) and close(r.entropy, h)
    assert r.grad.shape == x.shape and r.grad.dtype == x.dtype
    most = want.abs().amax(1, keepdim=True)
    tol = 4e-5 * most + (want.abs() * 2 ** -8 if x.dtype == torch.bfloat16 else 0) + 1e-38
    assert bool(((r.grad.double() - want).abs() <= tol).all())
    return r


DTYPES = [torch.float32, torch.bfloat16]
VOCABS = [1, 2, 3, 5, 63, 64, 65, 255, 1000, 1024, 2049, 5003, 8192, 16411, 30522, 32000, 50257, 65537, 70001]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_sizes(vocab, dtype):
    print(f"[logprobs] vocab {vocab} {dtype}", flush=True)
    for rows, pad in ((1, 0), (7, 3), (40, 0)):
        x, t = logits_of(rows, vocab, dtype, vocab + rows, pad)
        check_values(x, t, min(vocab, 7))
        g = torch.Generator(device="cuda").manual_seed(1)
        gp, gh = torch.randn(2, rows, generator=g, device="cuda")
        check_grad(x, t, gp, gh)
        check_grad(x, t, gp, None, temperature=0.6)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [500, 1024, 2048, 4096, 9001, 16384, 24001, 32000, 50257, 70001])
def test_many_rows(vocab, dtype):
    """Enough rows that throughput decides the launch's form."""
    print(f"[logprobs] 200 rows of {vocab} {dtype}", flush=True)
    x, t = logits_of(200, vocab, dtype, vocab, 1)
    t[::7] = -100
    x[3, :] = NINF
    x[4, : vocab // 2] = NINF
    check_values(x, t, 0, 0.8)
    check_values(x, t, 11)
    g = torch.Generator(device="cuda").manual_seed(3)
    gp, gh = torch.randn(2, 200, generator=g, device="cuda")
    check_grad(x, t, gp, None)
    check_grad(x, t, gp, gh, 1.4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k", [1, 2, 20, 63, 64])
def test_alternatives(k, dtype):
    """Ties, few allowed tokens, the best ones side by side or at the ends."""
    print(f"[logprobs] k {k} {dtype}", flush=True)
    x, t = logits_of(12, 32000, dtype, k)
    x[0] = 1.5                                    # all equal
    x[1] = NINF
    x[1, [3, 31999, 17000]] = torch.tensor([1.0, 2.0, 1.0], device="cuda", dtype=dtype)
    x[2, 100:100 + 2 * k] = 30.0                  # more equal ones than asked for, in one place
    x[3] = torch.linspace(10, -10, 32000, device="cuda").to(dtype)
    x[4] = torch.linspace(-10, 10, 32000, device="cuda").to(dtype)
    x[5] = torch.where(torch.arange(32000, device="cuda") % 2 == 0, 0.0, -0.0).to(dtype)
    x[6] = torch.finfo(dtype).min
    x[6, 5:9] = 0.0
    x[7] = x[7].clamp_max(2.0)                    # thousands of equal ones at the top
    x[8] = -x[8].abs() - 100.0
    t[9] = -100
    x[10] = NINF
    x[11] = torch.finfo(dtype).min
    check_values(x, t, k)
    check_values(x[:, 1:], t.clamp_max(31998), k, 0.5)


@pytest.mark.parametrize("dtype", DTYPES)
def test_masks_and_ignored_rows(dtype):
    print(f"[logprobs] masks {dtype}", flush=True)
    x, t = logits_of(64, 5003, dtype, 3, 5)
    g = torch.Generator(device="cuda").manual_seed(2)
    x.masked_fill_(torch.rand(64, 5003, generator=g, device="cuda") < 0.5, NINF)
    x[3] = NINF                                   # nothing allowed
    x[4] = NINF
    x[4, 77] = -2.0                               # one token allowed
    x[5] = torch.finfo(dtype).min                 # all at the type's lowest value
    x[6, :4000] = torch.finfo(dtype).min
    t[4], t[7], t[8] = 77, -100, -100
    x[8] = math.nan                               # an ignored row is not looked at
    t[9] = int(torch.nonzero(x[9] == NINF)[0])    # a token that cannot occur
    gp, gh = torch.randn(2, 64, generator=g, device="cuda")
    gp[8] = math.nan
    for temperature in (1.0, 0.3, 2.5):
        y = torch.where(x.isnan(), 0.0, x).to(dtype)
        check_values(y, t, 9, temperature)
        r = check_values_ignoring(x, t, temperature)
        assert float(r.logp[8]) == 0 and float(r.entropy[8]) == 0 and float(r.logp[9]) == NINF
        check_grad(y, t, torch.where(gp.isnan(), 0.0, gp), gh, temperature)
        z = token_logprobs_and_grad(x, t, gp, gh, temperature=temperature)
        assert bool((z.grad[7:9] == 0).all()) and bool((z.grad[3] == 0).all())


def check_values_ignoring(x, t, temperature):
    r = token_logprobs(x, t, top_k=3, temperature=temperature)
    _, _, logp, h, _ = exact(torch.where(x.isnan(), 0.0, x), t, temperature)
    assert close(r.logp, logp) and close(r.entropy, h)
    assert torch.equal(r.top_indices[7:9], torch.full((2, 3), -1, device="cuda"))
    assert bool((r.top_logprobs[7:9] == 0).all())
    return r


@pytest.mark.parametrize("dtype", DTYPES)
def test_non_finite_rows_and_bad_targets(dtype):
    print(f"[logprobs] non-finite {dtype}", flush=True)
    x, t = logits_of(8, 3000, dtype, 4)
    clean = token_logprobs(x, t, top_k=4)
    x[1, 2999] = math.nan
    x[2, 0] = math.inf
    t[4], t[5] = 3000, -1
    r = token_logprobs(x, t, top_k=4)
    for i in (1, 2):
        assert math.isnan(float(r.logp[i])) and math.isnan(float(r.entropy[i]))
        assert bool(r.top_logprobs[i].isnan().all()) and bool((r.top_indices[i] == -1).all())
    for i in (4, 5):
        assert math.isnan(float(r.logp[i]))
        assert torch.equal(r.top_indices[i], clean.top_indices[i])
    for i in (0, 3, 6, 7):
        assert torch.equal(r.logp[i], clean.logp[i]) and torch.equal(r.top_logprobs[i], clean.top_logprobs[i])
    one = torch.ones(8, device="cuda")
    z = token_logprobs_and_grad(x, t, one, one)
    for i in range(8):
        assert bool(z.grad[i].isnan().all()) == (i in (1, 2, 4, 5))
        assert bool(z.grad[i].isnan().any()) == (i in (1, 2, 4, 5))


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_starts_and_in_place(dtype):
    print(f"[logprobs] strides {dtype}", flush=True)
    for off, pad in ((0, 1), (1, 0), (3, 24), (5, 8)):
        x, t = logits_of(9, 4001 + off, dtype, off, pad)
        x = x[:, off:]
        t = t.clamp_max(4000)
        gp = torch.full((9,), -1 / 9, device="cuda")
        gh = torch.full((9,), 0.1, device="cuda")
        r = check_grad(x, t, gp, gh)
        # another alignment than the logits'
        big = torch.full((9, 4013), 7.0, dtype=dtype, device="cuda")
        o = big[:, 2:4003]
        token_logprobs_and_grad(x, t, gp, gh, out=o)
        assert torch.equal(o, r.grad)
        assert bool((big[:, :2] == 7).all()) and bool((big[:, 4003:] == 7).all())
        y = torch.empty(9, 4001 + off + pad, dtype=dtype, device="cuda")[:, off:off + 4001]   # as x lies
        y.copy_(x)
        z = token_logprobs_and_grad(y, t, gp, gh, out=y)
        assert z.grad is y and torch.equal(y, r.grad) and torch.equal(z.logp, r.logp)
    x, t = logits_of(6, 100, dtype)
    r = token_logprobs(x.view(2, 3, 100), t.view(2, 3), top_k=2)
    assert r.logp.shape == (2, 3) and r.top_indices.shape == (2, 3, 2)
    r1 = token_logprobs(x[4], t[4])
    assert r1.logp.shape == () and torch.equal(r1.logp, r.logp[1, 1])
    e = token_logprobs(x[:0], t[:0], top_k=2)
    assert e.logp.shape == (0,) and e.top_indices.shape == (0, 2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab,pad", [(4000, 0), (4001, 0), (1003, 5), (70001, 0)])
def test_rows_in_groups(vocab, pad, dtype):
    """Views of a batch of sequences whose rows have no one stride."""
    print(f"[logprobs] groups {vocab} + {pad} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(vocab)
    base = (torch.randn(3, 9, vocab + pad, generator=g, device="cuda") * 3).to(dtype)[:, :, :vocab]
    for x in (base[:, :-1], base[:, 1:], base.transpose(0, 1), base[::2, ::3], base[:, None, :4], base[:2, 5:6]):
        lead = x.shape[:-1]
        t = torch.randint(0, vocab, lead, generator=g, device="cuda")
        gp, gh = torch.randn(2, *lead, generator=g, device="cuda")
        flat, ft = x.reshape(-1, vocab), t.reshape(-1)
        check_values(flat, ft, 5)
        r = token_logprobs(x, t, top_k=5)
        lp, _, logp, h, _ = exact(flat, ft)
        assert r.logp.shape == lead and close(r.logp.reshape(-1), logp) and close(r.entropy.reshape(-1), h)
        order = torch.sort(flat.float(), dim=1, descending=True, stable=True).indices[:, :5]
        assert torch.equal(r.top_indices.reshape(-1, 5), order)
        assert close(r.top_logprobs.reshape(-1, 5), lp.gather(1, order))
        out = torch.empty(x.shape, dtype=dtype, device="cuda")
        want = exact_grad(flat, ft, gp.reshape(-1), gh.reshape(-1))
        tol = 4e-5 * want.abs().amax(1, keepdim=True) + (want.abs() * 2 ** -8 if dtype == torch.bfloat16 else 0) + 1e-38
        for z in (token_logprobs_and_grad(x, t, gp, gh), token_logprobs_and_grad(x, t, gp, gh, out=out)):
            assert z.grad.shape == x.shape
            assert bool(((z.grad.reshape(-1, vocab).double() - want).abs() <= tol).all())
    # through autograd, the shift of a causal model's loss
    leaf = base.clone().requires_grad_()
    t = torch.randint(0, vocab, (3, 8), generator=g, device="cuda")
    token_logprobs(leaf[:, :-1], t).logp.sum().backward()
    assert bool((leaf.grad[:, -1] == 0).all())
    want = exact_grad(base[:, :-1].reshape(-1, vocab), t.reshape(-1), torch.ones(24, device="cuda"), None)
    tol = 4e-5 * want.abs().amax(1, keepdim=True) + (want.abs() * 2 ** -8 if dtype == torch.bfloat16 else 0) + 1e-38
    assert bool(((leaf.grad[:, :-1].reshape(-1, vocab).double() - want).abs() <= tol).all())
    x, t = base[:, :-1], t
    with pytest.raises(ValueError):
        token_logprobs_and_grad(x, t, torch.ones(3, 8, device="cuda"), out=x)   # in place takes one stride
    with pytest.raises(ValueError):
        token_logprobs(base[:, :, None].expand(3, 9, 2, vocab), torch.zeros(3, 9, 2, dtype=torch.int64, device="cuda"))
    four = base.clone().view(3, 3, 3, vocab)[:, :2, :2]
    with pytest.raises(ValueError):
        token_logprobs(four, torch.zeros(3, 2, 2, dtype=torch.int64, device="cuda"))


def test_rows_past_32_bits():
    """Row offsets above 2^31 elements."""
    print("[logprobs] long strides", flush=True)
    store = torch.zeros(2 ** 31 + 4096, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((2, 3000), (2 ** 31 + 8, 1))
    src, t = logits_of(2, 3000, torch.bfloat16, 5)
    x.copy_(src)
    gp = torch.ones(2, device="cuda")
    a = token_logprobs(x, t, top_k=5)
    b = token_logprobs(src, t, top_k=5)
    assert torch.equal(a.logp, b.logp) and torch.equal(a.top_indices, b.top_indices)
    want = token_logprobs_and_grad(src, t, gp).grad
    token_logprobs_and_grad(x, t, gp, out=x)
    assert torch.equal(x, want)


def test_autograd_and_differences():
    """The autograd path against the formula, and the formula's derivative
    against differences of binary64 losses."""
    print("[logprobs] autograd", flush=True)
    x, t = logits_of(5, 301, torch.float32, 8)
    t[2] = -100
    w = torch.tensor([0.3, -1.0, 2.0, 0.7, -0.2], device="cuda")
    leaf = x.detach().clone().requires_grad_()
    r = token_logprobs(leaf, t, top_k=3, temperature=1.7)
    assert not r.top_logprobs.requires_grad
    ((w * r.logp).sum() + 0.5 * (w * r.entropy).sum()).backward()
    want = exact_grad(x, t, w, 0.5 * w, 1.7)
    assert bool(((leaf.grad.double() - want).abs() <= 4e-5 * want.abs().amax(1, keepdim=True)).all())

    def loss(z):
        _, _, logp, h, _ = exact(z, t, 1.7)
        return float((w.double() * logp).sum() + 0.5 * (w.double() * h).sum())

    for i, v in ((0, int(t[0])), (1, 7), (2, 5), (4, 300), (3, int(t[3]))):
        step = 1e-4
        up, down = x.double().clone(), x.double().clone()
        up[i, v] += step
        down[i, v] -= step
        # central differences: error step^2 / 6 times a third derivative below 10, and 1e-15 / step
        assert abs((loss(up) - loss(down)) / (2 * step) - float(leaf.grad[i, v])) < 1e-5
    # only one of the two outputs used
    for pick in (0, 1):
        leaf.grad = None
        token_logprobs(leaf, t)[pick].sum().backward()
        one = torch.ones(5, device="cuda")
        want = exact_grad(x, t, one * (pick == 0), one * (pick == 1))
        assert bool(((leaf.grad.double() - want).abs() <= 4e-5 * want.abs().amax(1, keepdim=True) + 1e-38).all())


def test_streams_and_graph():
    print("[logprobs] streams and graph", flush=True)
    x, t = logits_of(33, 30522, torch.bfloat16, 9)
    gp = torch.full((33,), -1 / 33, device="cuda")
    a = token_logprobs_and_grad(x, t, gp)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = token_logprobs_and_grad(x, t, gp)
        top = token_logprobs(x, t, top_k=8)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a.grad, b.grad) and torch.equal(a.logp, b.logp)
    graph = torch.cuda.CUDAGraph()
    out = torch.empty_like(x)
    with torch.cuda.graph(graph):
        c = token_logprobs_and_grad(x, t, gp, out=out)
        d = token_logprobs(x, t, top_k=8)
    for i in range(3):
        y, _ = logits_of(33, 30522, torch.bfloat16, 20 + i)
        x.copy_(y)
        graph.replay()
        e = token_logprobs_and_grad(y, t, gp)
        f = token_logprobs(y, t, top_k=8)
        torch.cuda.synchronize()
        assert torch.equal(out, e.grad) and torch.equal(c.logp, e.logp)
        assert torch.equal(d.top_indices, f.top_indices) and torch.equal(d.top_logprobs, f.top_logprobs)


def test_refusals_with_tensors():
    x, t = logits_of(4, 50, torch.float32)
    gp = torch.ones(4, device="cuda")
    with pytest.raises(TypeError):
        token_logprobs(x.half(), t)
    with pytest.raises(TypeError):
        token_logprobs(x, t.int())
    with pytest.raises(ValueError):
        token_logprobs(x, t[:3])
    with pytest.raises(ValueError):
        token_logprobs(x.t(), t[:1].expand(50))
    with pytest.raises(ValueError):
        token_logprobs(x.cpu(), t.cpu())
    with pytest.raises(ValueError):
        token_logprobs_and_grad(x, t, gp[:2])
    with pytest.raises(ValueError):
        token_logprobs_and_grad(x, t, gp, out=x.bfloat16())
    with pytest.raises(ma.MicroAdamError) as e:
        token_logprobs(x, t, top_k=51)
    assert e.value.code == ma.MICROADAM_ERR_INVALID_ARG
    big, tb = logits_of(1, 100, torch.float32)
    with pytest.raises(ma.MicroAdamError) as e:
        token_logprobs(big, tb, top_k=65)
    assert e.value.code == ma.MICROADAM_ERR_UNSUPPORTED
    for temperature in (0.0, -1.0, math.nan, math.inf, 1e-60):
        with pytest.raises(ma.MicroAdamError):
            token_logprobs(x, t, temperature=temperature)
