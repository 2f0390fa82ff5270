"""The norm over a list of gradients, and clipping by it, over the C ABI
(``microadam_grad_norm``, ``microadam_clip_grads``).

``clip_grad_norm`` takes a model's parameters, between backward and the
optimizers' steps; ``grad_norm`` and ``clip_grads`` take the gradients
themselves.  The norm stays on the device: nothing waits for it.

Gradients are float32 or bfloat16 on one ROCm device, mixed as they come, of
any shape, without gaps or overlaps in memory.  Work is queued on torch's
current stream.
"""
from __future__ import annotations

import contextlib
from array import array
from operator import attrgetter
from typing import Iterable, Optional

import torch
from torch.autograd.graph import increment_version

from . import MICROADAM_BF16, MICROADAM_F32, microadam_clip_grads, microadam_clip_workspace, microadam_grad_norm
from ._autograd import refuse_tangents, stream_of

_HERE = contextlib.nullcontext()
_DTYPES = {torch.float32: MICROADAM_F32, torch.bfloat16: MICROADAM_BF16}


def _on(device):
    """The device as the current one; nothing to do where it is."""
    return _HERE if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def workspace_bytes() -> int:
    """Bytes of workspace that a call takes, however long its list."""
    return microadam_clip_workspace()


def _dense(t: torch.Tensor) -> bool:
    """Whether t's elements fill one run of memory, each place once, in any
    order of the dimensions."""
    want = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != want and t.numel():
            return False
        want *= size
    return True


# (per tensor of a list of hundreds, whose host time is the call's: mapped, not looped over)
_data_ptr, _numel, _get_device, _is_contiguous = (torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.get_device,
                                                  torch.Tensor.is_contiguous)
_dtype, _requires_grad = attrgetter("dtype"), attrgetter("requires_grad")


def _listed(what: str, grads: list):
    """The addresses, numels and dtype codes as arrays."""
    if set(map(_get_device, grads)) != {grads[0].device.index} or not grads[0].is_cuda:
        raise ValueError(f"{what}: tensors on one ROCm device")
    try:
        codes = array("i", map(_DTYPES.__getitem__, map(_dtype, grads)))
    except KeyError as e:
        raise TypeError(f"{what}: float32 or bfloat16, not {e.args[0]}") from None
    if torch.is_grad_enabled() and any(map(_requires_grad, grads)):
        raise NotImplementedError(f"{what}: no derivative; a gradient requires grad")
    if not all(map(_is_contiguous, grads)) and not all(map(_dense, grads)):
        raise ValueError(f"{what}: a gradient with gaps or overlaps in memory")
    return array("Q", map(_data_ptr, grads)), array("q", map(_numel, grads)), codes


def _workspace(device, workspace):
    """(address, bytes, the tensor that holds it): the caller's, or one from
    torch's allocator."""
    if workspace is None:
        workspace = torch.empty(workspace_bytes(), dtype=torch.uint8, device=device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != device:
        raise ValueError("workspace: a contiguous uint8 tensor on the gradients' device")
    return workspace.data_ptr(), workspace.numel(), workspace


def grad_norm(grads: Iterable[torch.Tensor], *, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The 2-norm over all elements of the list, a float32 scalar on the
    device.  It has no derivative."""
    grads = list(grads)
    if not grads:
        raise ValueError("grads: at least one tensor")
    refuse_tangents("grad_norm", grads)
    arrays = _listed("grads", grads)
    given = [a.buffer_info()[0] for a in arrays]
    device = grads[0].device
    with _on(device):
        norm = torch.empty((), dtype=torch.float32, device=device)
        address, size, keep = _workspace(device, workspace)
        microadam_grad_norm(*given, len(grads), norm.data_ptr(), address, size,
                            stream_of(device.index))
    return norm


def clip_grads(grads: Iterable[torch.Tensor], max_norm: float, *, eps: float = 1e-6,
               workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Multiplies the gradients in place by ``max_norm / (norm + eps)`` where
    that is below 1, and returns the norm that they had, a float32 scalar on
    the device.  A norm of NaN makes all of them NaN, an infinite one makes
    the finite elements zero."""
    grads = list(grads)
    if not grads:
        raise ValueError("grads: at least one tensor")
    refuse_tangents("clip_grads", grads)
    arrays = _listed("grads", grads)
    given = [a.buffer_info()[0] for a in arrays]
    device = grads[0].device
    with _on(device):
        norm = torch.empty((), dtype=torch.float32, device=device)
        address, size, keep = _workspace(device, workspace)
        microadam_clip_grads(*given, len(grads), max_norm, eps, norm.data_ptr(), address, size,
                             stream_of(device.index))
    increment_version(grads)
    return norm


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
