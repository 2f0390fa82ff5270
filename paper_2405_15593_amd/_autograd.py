"""What the tensor functions share: checks on autograd's behalf, and the stream."""
from __future__ import annotations

import torch
import torch.autograd.forward_ad as forward_ad


def refuse_tangents(what: str, tensors) -> None:
    """A kernel takes addresses and would drop a dual tensor's tangent: the
    derivative would be zero without an error.  (None among the tensors is
    allowed.)"""
    if forward_ad._current_level < 0:   # no dual tensors outside a dual level
        return
    for t in tensors:
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise NotImplementedError(f"{what}: no derivatives in forward mode")


def _public_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


# The current stream's handle.  torch's own short way to it where there is one:
# autograd runs a backward function on a thread of its own, where every Python
# object that it touches comes from another core's cache.
stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or _public_stream


def once_differentiable(function):
    """A backward function without a derivative: itself where no graph of the
    backward pass is made; where one is, in torch's wrapper, whose results raise
    when they are differentiated."""
    wrapped = torch.autograd.function.once_differentiable(function)

    def backward(ctx, *grads):
        return wrapped(ctx, *grads) if torch.is_grad_enabled() else function(ctx, *grads)

    return staticmethod(backward)
