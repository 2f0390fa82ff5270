"""The norm over a list of gradients, and clipping by it, over the C ABI
(``microadam_grad_norm``, ``microadam_clip_grads``).

``clip_grad_norm`` takes a model's parameters, between backward and the
optimizers' steps; ``grad_norm`` and ``clip_grads`` take the gradients
themselves.  The norm stays on the device: nothing waits for it.

Gradients are float32 or bfloat16 on one ROCm device, mixed as they come, of
any shape, without gaps or overlaps in memory.  Work is queued on torch's
current stream.  Tracers that record torch's own operators (torch.jit.trace,
make_fx) are refused.
"""
from __future__ import annotations

from typing import Iterable, Optional

import torch

from . import microadam_clip_workspace, operators


def workspace_bytes() -> int:
    """Bytes of workspace that a call takes, however long its list."""
    return microadam_clip_workspace()


def grad_norm(grads: Iterable[torch.Tensor], *, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The 2-norm over all elements of the list, a float32 scalar on the
    device.  It has no derivative."""
    return operators().grad_norm(list(grads), workspace)


def clip_grads(grads: Iterable[torch.Tensor], max_norm: float, *, eps: float = 1e-6,
               workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Multiplies the gradients in place by ``max_norm / (norm + eps)`` where
    that is below 1, and returns the norm that they had, a float32 scalar on
    the device.  A norm of NaN makes all of them NaN, an infinite one makes
    the finite elements zero."""
    return operators().clip_grads(list(grads), max_norm, eps, workspace)


@torch.no_grad()
def clip_grad_norm(params, max_norm: float, *, eps: float = 1e-6,
                   workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``clip_grads`` over the gradients of a model's parameters (one parameter
    or several; those without a gradient are left out)."""
    params = [params] if isinstance(params, torch.Tensor) else list(params)
    grads = [p.grad for p in params if p.grad is not None]
    if not grads:
        return torch.zeros((), dtype=torch.float32, device=params[0].device if params else "cpu")
    return clip_grads(grads, max_norm, eps=eps, workspace=workspace)
