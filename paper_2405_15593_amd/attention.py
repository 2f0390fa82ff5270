"""Softmax attention, over the C ABI (``microadam_attention_forward``,
``microadam_attention_grad``).

``attention`` takes queries, keys and values as (batch, positions, heads, dim),
as a projection leaves them: views of one packed projection need no copy.  It
is differentiable in all three; the scores are not kept for that but computed
again.  Query heads may share key heads.  A batch of single queries over long
keys (generation) and prompts go through the same call.

Tensors are float32 or bfloat16 on a ROCm device, the dim a multiple of 8 up to
128.  Work is queued on torch's current stream.  A backward pass can be captured
into a graph together with its forward pass; as with torch's own operators no
eager graph of the same leaves may be alive then.  Tracers that record torch's own
operators (torch.jit.trace, make_fx) are refused; torch.compile calls it between
its graphs.
"""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import operators


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
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1]) if q.dim() and q.shape[-1] else 1.0
    return operators().attention(q, k, v, causal, scale, key_lengths)
