"""Checks on autograd's behalf that the tensor functions share."""
from __future__ import annotations

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
