"""layer_norm, attention and the clipping functions towards autograd and torch's
modes: which gradients are asked for, saved tensors, graphs of the backward
pass, inference mode."""
import pytest
import torch

from paper_2405_15593_amd.attention import attention
from paper_2405_15593_amd.clip import clip_grads, grad_norm
from paper_2405_15593_amd.norm import layer_norm

pytestmark = pytest.mark.gpu


def tensors(*shapes, dtype=torch.float32, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(s, generator=g, device="cuda").to(dtype) for s in shapes]


def norm_case():
    return (lambda x, w, b: layer_norm(x, w, b)), tensors((5, 33, 72), (72,), (72,))


def attention_case():
    return (lambda q, k, v: attention(q, k, v, causal=True)), tensors((2, 33, 4, 32), (2, 40, 2, 32), (2, 40, 2, 32))


CASES = {"norm": norm_case, "attention": attention_case}


@pytest.mark.parametrize("name", CASES)
def test_each_set_of_gradients(name):
    """Whatever is asked for, by grad and by backward, has the bits of the whole."""
    print(f"[nodes] sets {name}", flush=True)
    f, given = CASES[name]()
    dy = torch.randn_like(given[0])
    leaves = [t.clone().requires_grad_() for t in given]
    whole = torch.autograd.grad(f(*leaves), leaves, dy)
    for which in range(1, 8):
        some = [t.clone().requires_grad_(bool(which >> i & 1)) for i, t in enumerate(given)]
        y = f(*some)
        assert y.requires_grad and y.dtype == given[0].dtype
        y.backward(dy)
        for i, t in enumerate(some):
            assert torch.equal(t.grad, whole[i]) if which >> i & 1 else t.grad is None
        asked = [i for i in range(3) if which >> i & 1]
        got = torch.autograd.grad(f(*leaves), [leaves[i] for i in asked], dy)
        assert all(torch.equal(g, whole[i]) for g, i in zip(got, asked))
    assert not f(*given).requires_grad
    with torch.no_grad():
        assert not f(*leaves).requires_grad


def test_norm_with_a_bias_alone():
    print("[nodes] a bias alone", flush=True)
    x, b, dy = tensors((9, 40), (40,), (9, 40))
    leaves = [t.clone().requires_grad_() for t in (x, b)]
    got = torch.autograd.grad(layer_norm(leaves[0], None, leaves[1]), leaves, dy)
    ones = torch.ones_like(b)
    both = [t.clone().requires_grad_() for t in (x, b)]
    want = torch.autograd.grad(layer_norm(both[0], ones, both[1]), both, dy)
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    only = b.clone().requires_grad_()
    assert torch.equal(torch.autograd.grad(layer_norm(x, None, only), only, dy)[0], want[1])


@pytest.mark.parametrize("name", CASES)
def test_saved_tensors(name):
    """Through hooks (kept on the CPU between), twice with the graph kept, and no
    second time without."""
    print(f"[nodes] saved {name}", flush=True)
    f, given = CASES[name]()
    dy = torch.randn_like(given[0])
    leaves = [t.clone().requires_grad_() for t in given]
    y = f(*leaves)
    want = torch.autograd.grad(y, leaves, dy, retain_graph=True)
    again = torch.autograd.grad(y, leaves, dy)
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    with pytest.raises(RuntimeError):
        torch.autograd.grad(y, leaves, dy)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.cpu(), lambda t: t.cuda()):
        y = f(*leaves)
    assert all(torch.equal(a, b) for a, b in zip(want, torch.autograd.grad(y, leaves, dy)))


@pytest.mark.parametrize("name", CASES)
def test_no_second_derivative(name):
    """The gradients of a graph that is kept have the same bits, and raise when
    they are differentiated, also where only some are asked for."""
    print(f"[nodes] second derivative {name}", flush=True)
    f, given = CASES[name]()
    dy = torch.randn_like(given[0])
    leaves = [t.clone().requires_grad_() for t in given]
    want = torch.autograd.grad(f(*leaves), leaves, dy)
    for i in range(3):
        (g,) = torch.autograd.grad(f(*leaves), leaves[i], dy, create_graph=True)
        assert torch.equal(g, want[i]) and g.requires_grad
        with pytest.raises(RuntimeError, match="no derivative"):
            g.square().sum().backward()


def test_inference_mode():
    print("[nodes] inference mode", flush=True)
    for case in CASES.values():
        f, given = case()
        want = f(*given)
        with torch.inference_mode():
            assert torch.equal(f(*given), want)
            made = [t.clone() for t in given]
            assert torch.equal(f(*made), want)
    with torch.inference_mode():
        grads = tensors((300,), (7, 5))
        norm = grad_norm(grads)
        assert torch.equal(clip_grads(grads, 0.5), norm)
        assert abs(float(grad_norm(grads)) - 0.5) < 1e-5


def test_clipping_counts_as_a_change():
    """A gradient that a graph has saved is not scaled behind its back."""
    print("[nodes] version", flush=True)
    (g,) = tensors((50,))
    leaf = torch.ones(50, device="cuda", requires_grad=True)
    y = leaf * g
    clip_grads([g], 1e-3)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.parametrize("name", CASES)
def test_another_stream(name):
    """Forward on a stream of its own; backward follows it there."""
    print(f"[nodes] stream {name}", flush=True)
    f, given = CASES[name]()
    dy = torch.randn_like(given[0])
    leaves = [t.clone().requires_grad_() for t in given]
    want = torch.autograd.grad(f(*leaves), leaves, dy)
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            y = f(*(t * 1.0 for t in leaves))
        torch.cuda.current_stream().wait_stream(side)
        got = torch.autograd.grad(y, leaves, dy)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
