"""Softmax attention, over the C ABI (``microadam_attention_forward``,
``microadam_attention_grad``).

``attention`` takes queries, keys and values as (batch, positions, heads, dim),
as a projection leaves them: views of one packed projection need no copy.  It
is differentiable in all three; the scores are not kept for that but computed
again.  Query heads may share key heads.  A batch of single queries over long
keys (generation) and prompts go through the same call.

Tensors are float32 or bfloat16 on a ROCm device, the dim a multiple of 8 up to
128.  Work is queued on torch's current stream.
"""
from __future__ import annotations

import contextlib
import functools
import math
from typing import Optional

import torch

from . import (MICROADAM_BF16, MICROADAM_F32, microadam_attention, microadam_attention_forward,
               microadam_attention_grad, microadam_attention_saved, microadam_attention_workspace, microadam_heads)
from ._autograd import once_differentiable, refuse_tangents, stream_of

_HERE = contextlib.nullcontext()
_DTYPES = {torch.float32: MICROADAM_F32, torch.bfloat16: MICROADAM_BF16}


def _on(device):
    """The device as the current one; nothing to do where it is."""
    return _HERE if device.index == torch.cuda.current_device() else torch.cuda.device(device)


_FAR = 1 << 23


def _rows(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy where its rows are not contiguous, share elements or lie
    further apart than the C ABI takes."""
    _, pos, _, one = t.stride()
    return t if one == 1 and (t.shape[3] <= pos <= _FAR or t.shape[1] <= 1) else t.contiguous()


def _heads(t: torch.Tensor) -> microadam_heads:
    b, p, h, _ = t.stride()
    return microadam_heads(t.data_ptr(), b, p, h)


def _check(q, k, v, key_lengths):
    for t, what in ((q, "q"), (k, "k"), (v, "v")):
        if t.dtype not in _DTYPES:
            raise TypeError(f"{what}: float32 or bfloat16, not {t.dtype}")
        if t.dim() != 4:
            raise ValueError(f"{what}: (batch, positions, heads, dim)")
        if not t.is_cuda or t.device != q.device:
            raise ValueError("q, k and v: tensors on one ROCm device")
        if t.dtype is not q.dtype:
            raise TypeError("q, k and v: one dtype")
    if k.shape != v.shape or k.shape[0] != q.shape[0] or k.shape[3] != q.shape[3]:
        raise ValueError("k and v: one shape, with q's batch and dim")
    if key_lengths is not None:
        if key_lengths.dtype is not torch.int32:
            raise TypeError(f"key_lengths: int32, not {key_lengths.dtype}")
        if key_lengths.shape != q.shape[:1] or key_lengths.device != q.device:
            raise ValueError("key_lengths: one for each sequence, on q's device")


def _struct(q, k, v, key_lengths, causal, scale):
    b, sq, h, d = q.shape
    return microadam_attention(_heads(q), _heads(k), _heads(v), None if key_lengths is None else key_lengths.data_ptr(),
                               b, sq, k.shape[1], h, k.shape[2], d, scale, _DTYPES[q.dtype], 1 if causal else 0)


@functools.lru_cache(maxsize=256)
def _sizes(b, sq, sk, h, hk, d, code):
    """(workspace forward, workspace of the gradients, saved) bytes."""
    none = microadam_heads(None, 0, 0, 0)
    given = microadam_attention(none, none, none, None, b, sq, sk, h, hk, d, 1.0, code, 0)
    return (microadam_attention_workspace(given, False), microadam_attention_workspace(given, True),
            microadam_attention_saved(given))


def _sizes_of(q, k):
    b, sq, h, d = q.shape
    return _sizes(b, sq, k.shape[1], h, k.shape[2], d, _DTYPES[q.dtype])


def _bytes(need, device):
    """(the tensor that holds them, address) of so many bytes at a multiple of
    256, where torch's allocator puts a tensor of its own."""
    if not need:
        return None, None
    store = torch.empty(need, dtype=torch.uint8, device=device)
    return store, store.data_ptr()


def _forward(q, k, v, key_lengths, causal, scale, keep):
    """(out, what the backward pass takes besides or None)."""
    dev = q.device
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    given = _struct(q, k, v, key_lengths, causal, scale)
    need, _, kept = _sizes_of(q, k)
    if not keep:
        kept = 0
    with _on(dev):
        store, address = _bytes(need, dev)
        saved, at = _bytes(kept, dev)
        microadam_attention_forward(given, _heads(out), at, kept, address, need, stream_of(dev.index))
    return out, saved


def _backward(ctx, dout):
    """(autograd calls this on a thread of its own: what can be known before is
    in ctx.settings)"""
    q, k, v, key_lengths, out, saved = ctx.saved_tensors
    causal, scale, need, kept = ctx.settings
    q, k, v, dout = _rows(q), _rows(k), _rows(v), _rows(dout)
    dq = torch.empty_like(q, memory_format=torch.contiguous_format)
    dk = torch.empty_like(k, memory_format=torch.contiguous_format)
    dv = torch.empty_like(v, memory_format=torch.contiguous_format)
    given = _struct(q, k, v, key_lengths, causal, scale)
    dev = q.device
    with _on(dev):
        store, address = _bytes(need, dev)
        microadam_attention_grad(given, _heads(out), None if saved is None else saved.data_ptr(), kept, _heads(dout),
                                 _heads(dq), _heads(dk), _heads(dv), address, need, stream_of(dev.index))
    return dq, dk, dv, None, None, None


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, key_lengths, causal, scale):
        out, saved = _forward(_rows(q), _rows(k), _rows(v), key_lengths, causal, scale, True)
        ctx.save_for_backward(q, k, v, key_lengths, out, saved)
        _, need, kept = _sizes_of(q, k)
        ctx.settings = (causal, scale, need, kept)
        return out

    backward = once_differentiable(_backward)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, causal: bool = False,
              scale: Optional[float] = None, key_lengths: Optional[torch.Tensor] = None) -> torch.Tensor:
    """softmax(scale q k) v of (batch, queries, heads, dim) over (batch, keys,
    kv_heads, dim), of q's shape and dtype.  kv_heads divides heads, and
    consecutive query heads share a key head.  ``scale`` is 1 / sqrt(dim)
    unless given.  ``key_lengths`` (int32, one per sequence): how many of the
    first keys there are; what lies past them is not read.  ``causal``: the
    last query sees the last of the keys, each one before it one key less; what
    it hides is multiplied by zero, and expected to be finite.  A query without
    a key gives zeros.  There is no derivative of the backward pass, nor one in
    forward mode."""
    refuse_tangents("attention", (q, k, v))
    _check(q, k, v, key_lengths)
    scale = 1.0 / math.sqrt(q.shape[3]) if scale is None and q.shape[3] else scale if scale is not None else 1.0
    if key_lengths is not None:
        key_lengths = key_lengths.contiguous()
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad):
        return _Attention.apply(q, k, v, key_lengths, causal, float(scale))
    return _forward(_rows(q), _rows(k), _rows(v), key_lengths, causal, float(scale), False)[0]
