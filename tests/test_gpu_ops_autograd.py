"""What the loss and matrix-update functions do to autograd: writes in place
are seen by it, derivatives that they do not have are refused, and their
outputs are tensors of their own."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.logprobs import token_logprobs, token_logprobs_and_grad
from paper_2405_15593_amd.muon import Muon, muon_step, orthogonalize

pytestmark = pytest.mark.gpu

CHANGED = "modified by an inplace operation"


def rows(n=6, vocab=101, dtype=torch.float32, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, vocab, generator=g, device="cuda").to(dtype)
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    return x, t, torch.full((n,), -1.0 / n, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_saved_logits_that_the_gradient_replaces(dtype):
    """A soft-capped head's tanh saves its output, token_logprobs its logits:
    once the gradient stands in their place, their backward raises."""
    print(f"[autograd] gradient in place {dtype}", flush=True)
    x, t, gp = rows(dtype=dtype)
    leaf = x.clone().requires_grad_()
    logits = torch.tanh(leaf)
    token_logprobs_and_grad(logits, t, gp, out=logits)
    with pytest.raises(RuntimeError, match=CHANGED):
        logits.backward(torch.ones_like(logits))
    logits = leaf * 2.0
    r = token_logprobs(logits, t)
    token_logprobs_and_grad(logits, t, gp, out=logits)
    with pytest.raises(RuntimeError, match=CHANGED):
        r.logp.sum().backward()
    # a view of what was saved
    whole = torch.tanh(leaf)
    token_logprobs_and_grad(whole[2:], t[2:], gp[2:], out=whole[2:])
    with pytest.raises(RuntimeError, match=CHANGED):
        whole.sum().backward()


def test_a_producer_that_saved_nothing():
    """In place on a product's result is what out=logits is for."""
    print("[autograd] gradient in place of a product", flush=True)
    x, t, gp = rows()
    w = torch.randn(101, 101, device="cuda")
    grads = []
    for in_place in (False, True):
        leaf = x.clone().requires_grad_()
        logits = leaf @ w
        r = token_logprobs_and_grad(logits, t, gp, out=logits if in_place else None)
        logits.backward(r.grad)
        grads.append(leaf.grad)
    assert torch.equal(*grads)


def test_leaves_are_not_overwritten():
    print("[autograd] leaves", flush=True)
    x, t, gp = rows()
    leaf = x.clone().requires_grad_()
    view = leaf[:]
    for out in (leaf, view):
        with pytest.raises(ValueError, match="leaf"):
            token_logprobs_and_grad(x, t, gp, out=out)
    with pytest.raises(ValueError, match="requires grad"):
        orthogonalize(x, out=leaf)
    assert torch.equal(leaf.detach(), x)
    with torch.no_grad():
        assert torch.equal(token_logprobs_and_grad(x, t, gp, out=leaf).grad, token_logprobs_and_grad(x, t, gp).grad)
        assert torch.equal(orthogonalize(x, out=leaf), orthogonalize(x))


def test_what_is_written_gets_a_new_version():
    print("[autograd] versions", flush=True)
    x, t, gp = rows()
    p, g, v, o = x.clone(), x.clone(), torch.zeros_like(x), torch.empty_like(x)

    def versions():
        return [i._version for i in (p, g, v, o, x)]

    before = versions()
    muon_step([p], [g], [v], lr=0.1)
    orthogonalize(g, out=o)
    token_logprobs(x, t)
    token_logprobs_and_grad(x, t, gp)
    assert [a > b for a, b in zip(versions(), before)] == [True, False, True, True, False]
    before = versions()
    with pytest.raises(ma.MicroAdamError):
        token_logprobs_and_grad(x, t, gp, out=o, temperature=0.0)
    with pytest.raises(ma.MicroAdamError):
        muon_step([p], [g], [v], lr=float("nan"))
    assert versions() == before
    # where autograd keeps no versions
    with torch.inference_mode():
        y = x.clone()
        token_logprobs_and_grad(y, t, gp, out=y)
        muon_step([x.clone()], [g], [torch.zeros_like(x)], lr=0.1)
        assert torch.equal(y, token_logprobs_and_grad(x, t, gp).grad)


def test_backward_after_the_step():
    """A retained graph that saved the weights raises after Muon's step."""
    print("[autograd] retained graph", flush=True)
    w = torch.nn.Parameter(rows(16, 24)[0])
    x = rows(8, 16, seed=1)[0].requires_grad_()
    opt = Muon([w], lr=0.1)
    loss = (x @ w).sum()
    loss.backward(retain_graph=True)
    opt.step()
    with pytest.raises(RuntimeError, match=CHANGED):
        loss.backward()


def test_tangents_are_refused():
    """No derivative in forward mode: an error, not a result without a tangent."""
    print("[autograd] tangents", flush=True)
    x, t, gp = rows()
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        dual_gp = forward_ad.make_dual(gp, torch.ones_like(gp))
        calls = (lambda: token_logprobs(dual, t, top_k=2), lambda: token_logprobs_and_grad(dual, t, gp),
                 lambda: token_logprobs_and_grad(x, t, dual_gp), lambda: token_logprobs_and_grad(x, t, gp, dual_gp),
                 lambda: token_logprobs_and_grad(x, t, gp, out=dual), lambda: orthogonalize(dual),
                 lambda: orthogonalize(x, out=dual), lambda: muon_step([dual], [x], [gp], lr=0.1),
                 lambda: muon_step([x.clone()], [dual], [torch.zeros_like(x)], lr=0.1))
        for call in calls:
            with pytest.raises(NotImplementedError, match="forward mode"):
                call()
        with torch.no_grad(), pytest.raises(NotImplementedError, match="forward mode"):
            token_logprobs(dual, t)
        # others in the same level go on
        plain = token_logprobs(x, t)
    assert torch.equal(plain.logp, token_logprobs(x, t).logp)
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda z: token_logprobs(z, t).logp, (x,), (x,))


def test_orthogonalize_has_no_derivative():
    """A tensor that requires grad is refused where its graph would be lost."""
    print("[autograd] orthogonalize", flush=True)
    x = rows()[0]
    leaf = x.clone().requires_grad_()
    for t in (leaf, leaf * 2.0):
        with pytest.raises(NotImplementedError, match="no derivative"):
            orthogonalize(t)
        with torch.no_grad():
            orthogonalize(t)
    assert torch.equal(orthogonalize(leaf.detach()), orthogonalize(x))
    # a step is not recorded
    muon_step([leaf], [x.clone().requires_grad_()], [torch.zeros_like(x)], lr=0.1)
    assert leaf.is_leaf and not torch.equal(leaf, x)


@pytest.mark.parametrize("lead", [(), (6,), (2, 3)], ids=str)
def test_outputs_are_tensors_of_their_own(lead):
    """Each can be changed in place without touching the others' backward."""
    print(f"[autograd] outputs {lead}", flush=True)
    x, t, _ = rows()
    n = 6 if lead else 1
    x, t = x[:n].reshape(*lead, 101), t[:n].reshape(lead)
    keep = torch.arange(n, device="cuda").reshape(lead) % 2 == 0

    def grad(change):
        leaf = x.clone().requires_grad_()
        r = token_logprobs(leaf, t, top_k=2)
        change(r)
        return leaf.grad

    def in_place(r):
        r.logp.masked_fill_(~keep, 0.0).mul_(3.0)
        r.entropy.add_(r.logp.detach())
        r.top_logprobs.exp_()
        r.top_indices.add_(1)
        (r.logp.sum() + r.entropy.sum()).backward()

    def plain(r):
        ((r.logp * keep).sum() * 3.0 + r.entropy.sum()).backward()

    assert torch.equal(grad(in_place), grad(plain))

    def saved(r):
        loss = r.logp.square().sum()      # saves logp
        with torch.no_grad():
            r.entropy.mul_(2.0)
            r.top_logprobs.zero_()
        loss.backward()

    assert torch.equal(grad(saved), grad(lambda r: r.logp.square().sum().backward()))
    g = token_logprobs_and_grad(x, t, torch.ones(lead, device="cuda"))
    version = g.logp._version
    g.entropy.mul_(2.0)
    assert g.logp._version == version and g.logp.shape == g.entropy.shape == lead
