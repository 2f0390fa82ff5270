"""Layer norm over the last dimension, over the C ABI
(``microadam_layer_norm``, ``microadam_layer_norm_grad``).

``layer_norm`` is differentiable in the input, the weight and the bias.  The
input is float32 or bfloat16 on a ROCm device, weight and bias are of one of
these dtypes too, the input's or the other (float32 weights of bfloat16
activations).  Rows at one stride are read where they lie; any other layout is
copied first.  Work is queued on torch's current stream.  A backward pass can be
captured into a graph together with its forward pass; as with torch's own
operators no eager graph of the same leaves may be alive then.  Tracers that record
torch's own operators (torch.jit.trace, make_fx) are refused; torch.compile calls it
between its graphs.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import operators


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
               eps: float = 1e-5) -> torch.Tensor:
    """Rows (the last dimension) of ``x`` with their mean taken off, divided by
    the root of their variance plus ``eps``, times ``weight``, plus ``bias``; of
    x's shape and dtype.  The backward pass takes the mean as it was saved, rounded
    to float32: of rows whose mean lies more than some 64 standard deviations from
    zero gradients have fewer bits than the result.  There is no derivative of the
    backward pass, nor one in forward mode."""
    return operators().layer_norm(x, weight, bias, eps)
