"""torch's tracers record its own operators: of layer_norm, attention and the
clipping functions they would record the allocations alone.  Each refuses to be
recorded, forward and backward."""
import os

import pytest
import torch
from torch.fx.experimental.proxy_tensor import make_fx
from torch.utils._python_dispatch import TorchDispatchMode

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.attention import attention
from paper_2405_15593_amd.clip import clip_grad_norm, clip_grads, grad_norm
from paper_2405_15593_amd.norm import layer_norm

X, Q = (3, 8), (1, 3, 2, 8)
CALLS = {"layer_norm": (X, lambda x: layer_norm(x)), "attention": (Q, lambda q: attention(q, q, q)),
         "grad_norm": (X, lambda x: grad_norm([x])), "clip_grads": (X, lambda x: clip_grads([x], 1.0))}
TRACERS = {"jit": lambda f, t: torch.jit.trace(f, t), "real": lambda f, t: make_fx(f)(t),
           "before_dispatch": lambda f, t: make_fx(f, pre_dispatch=True)(t),
           "symbolic": lambda f, t: make_fx(f, tracing_mode="symbolic")(t)}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ma.LIBRARY):
        from paper_2405_15593_amd import _build
        _build.build()
    return ma.operators()


def refuse(name, tracer, device):
    shape, f = CALLS[name]
    with pytest.raises(NotImplementedError, match=f"{name}: not recorded"):
        TRACERS[tracer](f, torch.ones(shape, device=device))


@pytest.mark.parametrize("tracer", TRACERS)
@pytest.mark.parametrize("name", CALLS)
def test_tracers_are_refused(name, tracer):
    refuse(name, tracer, "cpu")
    # not once the tracer is gone
    shape, f = CALLS[name]
    with pytest.raises(ValueError, match="ROCm"):
        f(torch.ones(shape))


@pytest.mark.gpu
@pytest.mark.parametrize("tracer", TRACERS)
@pytest.mark.parametrize("name", CALLS)
def test_tracers_are_refused_on_the_device(name, tracer):
    print(f"[tracing] {name} {tracer}", flush=True)
    refuse(name, tracer, "cuda")
    CALLS[name][1](torch.ones(CALLS[name][0], device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["layer_norm", "attention"])
def test_backward_passes_are_refused(name):
    """... of a forward pass that was made outside of the tracer, and is whole after."""
    print(f"[tracing] backward {name}", flush=True)
    shape, f = CALLS[name]
    leaf = torch.randn(shape, device="cuda", requires_grad=True)
    dy = torch.randn(shape, device="cuda")
    (want,) = torch.autograd.grad(f(leaf), leaf, dy)
    for pre_dispatch in (False, True):
        y = f(leaf)
        with pytest.raises(NotImplementedError, match=f"{name}: the backward pass is not recorded"):
            make_fx(lambda d: torch.autograd.grad(y, leaf, d, retain_graph=True)[0], pre_dispatch=pre_dispatch)(dy)
        assert torch.equal(torch.autograd.grad(y, leaf, dy)[0], want)


@pytest.mark.gpu
def test_modes_that_watch_are_not():
    """Any other dispatch mode sees the allocations, and results are right."""
    print("[tracing] watching", flush=True)

    class Watch(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))

    given = {name: torch.randn(shape, device="cuda") for name, (shape, _) in CALLS.items()}
    wants = {name: CALLS[name][1](t.clone()) for name, t in given.items()}
    with Watch():
        gots = {name: CALLS[name][1](t.clone()) for name, t in given.items()}
    assert all(torch.equal(gots[name], w) for name, w in wants.items())


@pytest.mark.gpu
def test_compiled_functions_break_their_graph():
    """torch.compile calls them between its graphs."""
    print("[tracing] compile", flush=True)

    def f(x):
        return layer_norm(x * 2.0) + 1.0

    x = torch.randn(X, device="cuda")
    assert torch.equal(torch.compile(f, backend="eager")(x), f(x))
    leaf = torch.nn.Parameter(x.clone())
    leaf.grad = x.clone()
    assert torch.equal(clip_grad_norm([leaf], 1.0), grad_norm([x]))
