"""Rows of millions of logits, up to the 2^24 that are accepted, and segmented
rows in place.

Logits are 0 or -1, so that the 64-bit values follow from two counts.
Tolerances, before any run: a thread adds at most 64 terms of a segment one
after another, 64 2^-24 = 3.8e-6 of the sum; segments add nothing (binary64),
threads and waves a tree of at most 14 levels, 8e-7; exponentials 2e-7.  That
is 4.8e-6 for s, and as much again for the sum of p d where |d| <= 1.  log s
comes within 2 units of 17 in binary32, 2e-6 2: logp is within 1e-5, the
entropy within 2e-5, a binary32 gradient's element within 1e-5 of itself (the
entropy's part apart: 4e-5)."""
import math

import pytest
import torch

from paper_2405_15593_amd.logprobs import token_logprobs, token_logprobs_and_grad

pytestmark = pytest.mark.gpu


def two_levels(rows, vocab, dtype):
    """Rows whose share of zeros differs, with their 64-bit (logp of a 0, entropy)."""
    g = torch.Generator(device="cuda").manual_seed(vocab + rows)
    x = torch.empty(rows, vocab, dtype=dtype, device="cuda")
    want = []
    for i in range(min(rows, 5)):
        line = (torch.rand(vocab, generator=g, device="cuda") < 0.1 + 0.2 * i)
        line[0] = True
        zeros = int(line.sum())
        s = zeros + (vocab - zeros) * math.exp(-1)
        want.append((-math.log(s), math.log(s) + (vocab - zeros) * math.exp(-1) / s))
        x[i::5] = (line.float() - 1.0).to(dtype)
    want = torch.tensor(want, dtype=torch.float64, device="cuda")
    return x, want[torch.arange(rows, device="cuda") % 5]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(1, 1 << 24), (5, 1 << 20), (130, 1 << 20), (130, 4_000_003), (130, 1 << 24)])
def test_long_rows(rows, vocab, dtype):
    if dtype == torch.float32 and rows * vocab > 1 << 30:
        rows = 1 + rows % 129   # 9 GB say no more than 4.5
    print(f"[logprobs] {rows} rows of {vocab} {dtype}", flush=True)
    x, want = two_levels(rows, vocab, dtype)
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    one = torch.ones(rows, device="cuda")
    for r in (token_logprobs(x, t), token_logprobs(x, t, top_k=3), token_logprobs_and_grad(x, t, one),
              token_logprobs_and_grad(x, t, one, one)):
        assert float((r.logp.double() - want[:, 0]).abs().max()) < 1e-5
        assert float((r.entropy.double() - want[:, 1]).abs().max()) < 2e-5
    del r
    if dtype == torch.float32:
        p = [want[:5, 0].exp(), (want[:5, 0] - 1.0).exp()]
        for gh in (None, 0.5 * one):
            grad = token_logprobs_and_grad(x, t, one, gh).grad
            for i in range(min(rows, 5)):
                for level in (0, 1):
                    exact = -float(p[level][i])
                    tol = 1e-5 * -exact
                    if gh is not None:
                        # lp + H: two numbers near 17 whose difference is below 1
                        exact -= 0.5 * float(p[level][i] * (want[i, 0] - level + want[i, 1]))
                        tol = 4e-5 * float(p[level][i])
                    at = x[i] == -level
                    at[0] = False
                    assert float((grad[i][at].double() - exact).abs().max()) < tol
            del grad


@pytest.mark.parametrize("rows", [1, 130])
def test_a_token_with_most_of_a_long_row(rows):
    """The others' sum, which is taken apart from the largest: all of it in the
    chunks of 16 bytes that one thread of 256 (or of 1024) holds with it."""
    print(f"[logprobs] most in one token, {rows} rows", flush=True)
    vocab = 1 << 24
    x = torch.full((rows, vocab), -math.inf, dtype=torch.bfloat16, device="cuda")
    x.view(rows, -1, 1024, 8)[:, :, 0] = 0.0
    x[:, 0] = 12.0
    others = vocab // 1024 - 1
    r = token_logprobs(x, torch.zeros(rows, dtype=torch.int64, device="cuda"))
    rest = others * math.exp(-12.0)
    assert float((r.logp.double() + math.log1p(rest)).abs().max()) < 1e-5 * rest


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(3, 70001), (140, 70008), (140, 200003)])
def test_segmented_rows_in_place(rows, vocab, dtype):
    """Rows that are read again for their gradient, which replaces them."""
    print(f"[logprobs] in place {rows} x {vocab} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = (torch.randn(rows, vocab, generator=g, device="cuda") * 3).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    x[1, int(t[1])] = 40.0                       # nearly all of the probability
    x[2] = -math.inf
    t[0] = -100
    gp, gh = torch.randn(2, rows, generator=g, device="cuda")
    for entropy in (None, gh):
        apart = token_logprobs_and_grad(x, t, gp, entropy)
        y = x.clone()
        here = token_logprobs_and_grad(y, t, gp, entropy, out=y)
        assert here.grad is y and torch.equal(y, apart.grad)
        assert torch.equal(here.logp, apart.logp) and torch.equal(here.entropy, apart.entropy)
        z = x.double()
        lp = torch.log_softmax(z, 1)
        p = lp.exp()
        h = -(p * lp.clamp_min(-1e30)).sum(1)
        want = -p * gp.double()[:, None]
        if entropy is not None:
            want -= entropy.double()[:, None] * p * (lp.clamp_min(-1e30) + h[:, None])
        want[torch.arange(rows), t.clamp_min(0)] += gp.double()
        want[0] = 0.0
        want[2] = 0.0
        most = want.abs().amax(1, keepdim=True)
        tol = 4e-5 * most + (want.abs() * 2 ** -8 if dtype == torch.bfloat16 else 0) + 1e-38
        assert bool(((y.double() - want).abs() <= tol).all())
        del apart, here, y, z, lp, p, want
