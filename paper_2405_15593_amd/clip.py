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
import ctypes
from typing import Iterable, Optional

import torch
from torch.autograd.graph import increment_version

from . import MICROADAM_BF16, MICROADAM_F32, microadam_clip_grads, microadam_clip_workspace, microadam_grad_norm
from ._autograd import refuse_tangents

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


def _listed(what: str, grads: list):
    """(addresses, numels, dtype codes) as arrays."""
    device = grads[0].device
    if device.type != "cuda":
        raise ValueError(f"{what}: tensors on a ROCm device")
    codes = []
    differentiable = torch.is_grad_enabled()
    for g in grads:
        code = _DTYPES.get(g.dtype)
        if code is None:
            raise TypeError(f"{what}: float32 or bfloat16, not {g.dtype}")
        codes.append(code)
        if g.device != device:
            raise ValueError(f"{what}: one device")
        if differentiable and g.requires_grad:
            raise NotImplementedError(f"{what}: no derivative; a gradient requires grad")
        if not g.is_contiguous() and not _dense(g):
            raise ValueError(f"{what}: a gradient with gaps or overlaps in memory")
    n = len(grads)
    return ((ctypes.c_void_p * n)(*[g.data_ptr() for g in grads]), (ctypes.c_int64 * n)(*[g.numel() for g in grads]),
            (ctypes.c_int32 * n)(*codes), n)


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
    given = _listed("grads", grads)
    device = grads[0].device
    with _on(device):
        norm = torch.empty((), dtype=torch.float32, device=device)
        address, size, keep = _workspace(device, workspace)
        microadam_grad_norm(*given, norm.data_ptr(), address, size,
                            torch.cuda.current_stream(device.index).cuda_stream)
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
    given = _listed("grads", grads)
    device = grads[0].device
    with _on(device):
        norm = torch.empty((), dtype=torch.float32, device=device)
        address, size, keep = _workspace(device, workspace)
        microadam_clip_grads(*given, max_norm, eps, norm.data_ptr(), address, size,
                             torch.cuda.current_stream(device.index).cuda_stream)
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
