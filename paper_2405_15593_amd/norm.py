"""Layer norm over the last dimension, over the C ABI
(``microadam_layer_norm``, ``microadam_layer_norm_grad``).

``layer_norm`` is differentiable in the input, the weight and the bias.  The
input is float32 or bfloat16 on a ROCm device, weight and bias are of one of
these dtypes too, the input's or the other (float32 weights of bfloat16
activations).  Rows at one stride are read where they lie; any other layout is
copied first.  Work is queued on torch's current stream.
"""
from __future__ import annotations

import contextlib
import functools
from typing import Optional

import torch

from . import (MICROADAM_BF16, MICROADAM_F32, microadam_layer_norm, microadam_layer_norm_grad,
               microadam_layer_norm_workspace, microadam_rows)
from ._autograd import once_differentiable, refuse_tangents, stream_of

_HERE = contextlib.nullcontext()
_DTYPES = {torch.float32: MICROADAM_F32, torch.bfloat16: MICROADAM_BF16}


def _on(device):
    """The device as the current one; nothing to do where it is."""
    return _HERE if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _matrix(t: torch.Tensor):
    """(t, or a copy of it, that lies in rows at one stride; rows; row stride)."""
    cols = t.shape[-1]
    rows = t.numel() // cols
    if t.is_contiguous():
        return t, rows, cols
    if cols == 1 or t.stride(-1) == 1:
        lead = [(n, s) for n, s in zip(t.shape[:-1], t.stride()[:-1]) if n != 1]
        if not lead:
            return t, rows, cols
        if lead[-1][1] >= cols and all(a[1] == b[0] * b[1] for a, b in zip(lead, lead[1:])):
            return t, rows, lead[-1][1]
    return t.contiguous(), rows, cols


def _check(x, weight, bias):
    code = _DTYPES.get(x.dtype)
    if code is None:
        raise TypeError(f"x: float32 or bfloat16, not {x.dtype}")
    if not x.is_cuda:
        raise ValueError("x: a tensor on a ROCm device")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x: at least one element in the last dimension")
    side = None
    for t, what in ((weight, "weight"), (bias, "bias")):
        if t is None:
            continue
        if t.dtype not in _DTYPES:
            raise TypeError(f"{what}: float32 or bfloat16, not {t.dtype}")
        if side is not None and t.dtype is not side:
            raise TypeError("weight and bias: one dtype")
        side = t.dtype
        if t.shape != x.shape[-1:] or t.device != x.device:
            raise ValueError(f"{what}: one element for each of x's last dimension, on x's device")
    return code, code if side is None else _DTYPES[side]


@functools.lru_cache(maxsize=256)
def _workspace_bytes(rows, cols, code):
    return microadam_layer_norm_workspace(microadam_rows(None, None, None, rows, cols, cols, 0.0, code, code))


def _address(t):
    return None if t is None else t.data_ptr()


def _forward(x, weight, bias, eps, keep):
    """(y, the statistics or None, rows, dtype codes)."""
    codes = _check(x, weight, bias)
    given, rows, ld = _matrix(x)
    w, b = (t if t is None or t.is_contiguous() else t.contiguous() for t in (weight, bias))
    cols, dev = x.shape[-1], x.device
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    stats = torch.empty(2 * rows, dtype=torch.float32, device=dev) if keep else None   # means, then rstds
    mean = None if stats is None else stats.data_ptr()
    with _on(dev):
        r = microadam_rows(given.data_ptr(), _address(w), _address(b), rows, cols, ld, eps, *codes)
        microadam_layer_norm(r, y.data_ptr(), cols, mean, mean and mean + 4 * rows, stream_of(dev.index))
    return y, stats, rows, codes


def _backward(ctx, dy):
    """(autograd calls this on a thread of its own: what can be known before is
    in ctx.settings, and the usual layouts take the short way)"""
    x, weight, stats = ctx.saved_tensors
    want_x, want_w, want_b, _ = ctx.needs_input_grad
    rows, cols, eps, codes, side, need = ctx.settings
    plain, ld = x.is_contiguous(), cols
    if not plain:
        x, _, ld = _matrix(x)
    if not dy.is_contiguous():
        dy, _, dy_ld = _matrix(dy)
    else:
        dy_ld = cols
    w = weight if weight is None or weight.is_contiguous() else weight.contiguous()
    dx = (torch.empty_like(x) if plain else x.new_empty(x.shape)) if want_x else None
    dw = stats.new_empty(cols, dtype=side) if want_w else None
    db = stats.new_empty(cols, dtype=side) if want_b else None
    workspace = stats.new_empty(need) if need else None
    r = microadam_rows(x.data_ptr(), None if w is None else w.data_ptr(), None, rows, cols, ld, eps, *codes)
    mean, dev = stats.data_ptr(), x.device
    with _on(dev):
        microadam_layer_norm_grad(r, mean, mean + 4 * rows, dy.data_ptr(), dy_ld, None if dx is None else dx.data_ptr(),
                                  cols, None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(),
                                  None if workspace is None else workspace.data_ptr(), 4 * need, stream_of(dev.index))
    return dx, dw, db, None


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, stats, rows, codes = _forward(x, weight, bias, eps, True)
        ctx.save_for_backward(x, weight, stats)
        cols = x.shape[-1]
        side = weight.dtype if weight is not None else bias.dtype if bias is not None else x.dtype
        need = _workspace_bytes(rows, cols, codes[0]) if ctx.needs_input_grad[1] or ctx.needs_input_grad[2] else 0
        ctx.settings = (rows, cols, eps, codes, side, need // 4)
        return y

    backward = once_differentiable(_backward)


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
               eps: float = 1e-5) -> torch.Tensor:
    """Rows (the last dimension) of ``x`` with their mean taken off, divided by
    the root of their variance plus ``eps``, times ``weight``, plus ``bias``; of
    x's shape and dtype.  There is no derivative of the backward pass, nor one
    in forward mode."""
    refuse_tangents("layer_norm", (x, weight, bias))
    if torch.is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad) or
                                    (bias is not None and bias.requires_grad)):
        return _LayerNorm.apply(x, weight, bias, eps)
    return _forward(x, weight, bias, eps, False)[0]
