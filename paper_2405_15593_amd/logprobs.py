"""Log probabilities of given tokens from logits, with the distribution's
entropy, the most probable alternatives and the gradient, over the C ABI
(``microadam_token_logprobs``, ``microadam_token_logprobs_grad``).

``token_logprobs`` is differentiable in the logits through ``logp`` and
``entropy``; a loss made of them (``-logp.mean()``, a policy gradient, an
entropy bonus) trains as usual.  Where the loss's weight of every token is
known before the call, ``token_logprobs_and_grad`` gives the values and the
gradient in one pass over the logits.

Logits are float32 or bfloat16 on a ROCm device, (..., vocab) with contiguous
rows at one stride, or at two (``logits[:, :-1]`` of a batch of sequences);
targets are int64 of the leading shape, with
``ignore_index`` for rows to leave out.  Work is queued on torch's current
stream.
"""
from __future__ import annotations

import contextlib
from typing import NamedTuple, Optional

import torch
from torch.autograd.graph import increment_version

from . import (MICROADAM_BF16, MICROADAM_F32, microadam_logits, microadam_token_logprobs,
               microadam_token_logprobs_grad)
from ._autograd import refuse_tangents

_HERE = contextlib.nullcontext()
_DTYPES = {torch.float32: MICROADAM_F32, torch.bfloat16: MICROADAM_BF16}


class TokenLogprobs(NamedTuple):
    logp: torch.Tensor                        # (...) float32
    entropy: torch.Tensor                     # (...) float32
    top_logprobs: Optional[torch.Tensor]      # (..., top_k) float32, or None
    top_indices: Optional[torch.Tensor]       # (..., top_k) int64, or None


class TokenLogprobsGrad(NamedTuple):
    logp: torch.Tensor
    entropy: torch.Tensor
    grad: torch.Tensor                        # of the logits' shape and dtype


def _joined(lead):
    """Leading (size, stride) with neighbours joined where one stride serves
    both; a single empty dimension if any is."""
    if any(n == 0 for n, _ in lead):
        return [(0, 0)]
    out = [lead[0]]
    for n, s in lead[1:]:
        if out[-1][1] == n * s:
            out[-1] = (out[-1][0] * n, s)
        else:
            out.append((n, s))
    return out


def _rows(logits: torch.Tensor, targets: torch.Tensor):
    """(dtype code, address, rows, vocab, row stride, rows of a group or 0, stride
    of groups, targets as [rows])."""
    code = _DTYPES.get(logits.dtype)
    if code is None:
        raise TypeError(f"logits: float32 or bfloat16, not {logits.dtype}")
    if targets.dtype != torch.int64:
        raise TypeError(f"targets: int64, not {targets.dtype}")
    if not logits.is_cuda or targets.device != logits.device:
        raise ValueError("logits and targets: tensors on one ROCm device")
    if logits.dim() < 1 or targets.shape != logits.shape[:-1]:
        raise ValueError("targets: the shape of logits without its last dimension")
    vocab = logits.shape[-1]
    if vocab > 1 and logits.stride(-1) != 1:
        raise ValueError("logits: contiguous rows")
    lead = [(n, s) for n, s in zip(logits.shape[:-1], logits.stride()[:-1]) if n != 1] if logits.dim() != 2 else \
        ((logits.shape[0], logits.stride(0)),)
    if len(lead) > 1:
        lead = _joined(lead)
    rows, ld, group, group_stride = 1, max(1, vocab), 0, 0
    if lead:
        rows, stride = lead[-1]
        if rows > 1:
            ld = stride
            if ld < vocab:
                raise ValueError("logits: rows must not overlap")
        if len(lead) == 2 and rows:
            group, group_stride = rows, lead[0][1]
            rows *= lead[0][0]
        elif len(lead) > 1:
            raise ValueError("logits: rows at one stride, or in groups at a second")
    if targets.dim() != 1 or not targets.is_contiguous():
        targets = targets.reshape(-1).contiguous()
    return code, logits.data_ptr(), rows, vocab, ld, group, group_stride, targets


def _on(device):
    """The device as the current one; nothing to do where it is."""
    return _HERE if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _struct(rows, ignore_index, temperature):
    code, address, n, vocab, ld, group, group_stride, targets = rows
    return microadam_logits(address, targets.data_ptr(), n, vocab, ld, int(ignore_index), float(temperature), code, 0,
                            group, group_stride)


def _outputs(targets):
    """logp and entropy: tensors of their own, no views, since what the autograd
    function returns may be changed in place."""
    return (torch.empty_like(targets, dtype=torch.float32, memory_format=torch.contiguous_format),
            torch.empty_like(targets, dtype=torch.float32, memory_format=torch.contiguous_format))


def _values(logits, targets, top_k, temperature, ignore_index):
    given = _rows(logits, targets)
    lead, dev = targets.shape, logits.device
    logp, entropy = _outputs(targets)
    top_v = top_i = None
    if top_k:
        top_v = torch.empty((*lead, top_k), dtype=torch.float32, device=dev)
        top_i = torch.empty((*lead, top_k), dtype=torch.int64, device=dev)
    with _on(dev):
        microadam_token_logprobs(_struct(given, ignore_index, temperature), int(top_k), logp.data_ptr(),
                                 entropy.data_ptr(), top_v.data_ptr() if top_k else None,
                                 top_i.data_ptr() if top_k else None, torch.cuda.current_stream(dev.index).cuda_stream)
    return TokenLogprobs(logp, entropy, top_v, top_i)


def _grad_rows(logits: torch.Tensor, given) -> torch.Tensor:
    """[rows, vocab] for the gradient, whose rows start at the same place in 16
    bytes as the logits' rows: at most 15 bytes of a row and of the start are
    left unused, none where the logits are dense and start aligned.  Rows in
    groups: only as far as the groups' stride allows.  Of logits[:, :-1] with a
    vocabulary that is no multiple of 16 bytes most groups start elsewhere, and
    their gradient is stored element by element (4 x 2047 x 50257 bf16: 446 us;
    of a dense copy 396, and 272 for the copy)."""
    _, address, rows, vocab, ld = given[:5]
    size = logits.element_size()
    per = 16 // size
    start = address % 16 // size
    gld = vocab + (ld - vocab) % per
    if not start and gld == vocab:
        return torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device)
    store = torch.empty(start + rows * gld, dtype=logits.dtype, device=logits.device)
    return store.as_strided((rows, vocab), (gld, 1), start)


def _upstream(g, lead, what):
    if g.shape != lead:
        raise ValueError(f"{what}: the targets' shape")
    if g.dtype is not torch.float32 or g.dim() != 1 or not g.is_contiguous():
        g = g.reshape(-1).to(torch.float32).contiguous()
    return g


def token_logprobs_and_grad(logits: torch.Tensor, targets: torch.Tensor, grad_logp: torch.Tensor,
                            grad_entropy: Optional[torch.Tensor] = None, *, temperature: float = 1.0,
                            ignore_index: int = -100, out: Optional[torch.Tensor] = None) -> TokenLogprobsGrad:
    """Log probabilities, entropies and, in the same pass, the gradient with
    respect to the logits of sum(grad_logp * logp + grad_entropy * entropy).
    For the mean negative log likelihood of n tokens, grad_logp is -1/n.
    ``out``: where the gradient goes (``logits`` itself is allowed; autograd
    sees the write as one in place, so a backward that saved what was there
    raises).  Nothing else is recorded for autograd."""
    refuse_tangents("token_logprobs_and_grad", (logits, grad_logp, grad_entropy, out))
    if logits.requires_grad:
        logits = logits.detach()
    given = _rows(logits, targets)
    lead, dev = targets.shape, logits.device
    gp = _upstream(grad_logp, lead, "grad_logp")
    ge = None if grad_entropy is None else _upstream(grad_entropy, lead, "grad_entropy")
    for g in (gp, ge):
        if g is not None and g.device != dev:
            raise ValueError("grad_logp and grad_entropy: the logits' device")
    if out is None:
        grad = _grad_rows(logits, given)
        gld, shaped = grad.stride(0), grad if logits.dim() == 2 else grad.view(logits.shape)
        grad_address = grad.data_ptr()
    else:
        if out.shape != logits.shape or out.dtype != logits.dtype:
            raise ValueError("out: the logits' shape and dtype")
        if torch.is_grad_enabled() and out.requires_grad and (out if out._base is None else out._base).is_leaf:
            raise ValueError("out: a leaf that requires grad, or a view of one")
        _, grad_address, _, _, gld, group, _, _ = _rows(out, targets)
        if group:
            raise ValueError("out: rows at one stride")
        shaped = out
    logp, entropy = _outputs(targets)
    with _on(dev):
        microadam_token_logprobs_grad(_struct(given, ignore_index, temperature), gp.data_ptr(),
                                      None if ge is None else ge.data_ptr(), logp.data_ptr(), entropy.data_ptr(),
                                      grad_address, gld, torch.cuda.current_stream(dev.index).cuda_stream)
    if out is not None:
        increment_version(out)
    return TokenLogprobsGrad(logp, entropy, shaped)


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, top_k, temperature, ignore_index):
        r = _values(logits, targets, top_k, temperature, ignore_index)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(logits, targets)
        ctx.settings = (temperature, ignore_index)
        if top_k:
            ctx.mark_non_differentiable(r.top_logprobs, r.top_indices)
        return tuple(r)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_logp, g_entropy, *_):
        logits, targets = ctx.saved_tensors
        temperature, ignore_index = ctx.settings
        if g_logp is None and g_entropy is None:
            return None, None, None, None, None
        if g_logp is None:
            g_logp = torch.zeros_like(g_entropy)
        return token_logprobs_and_grad(logits, targets, g_logp, g_entropy, temperature=temperature,
                                       ignore_index=ignore_index).grad, None, None, None, None


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, *, top_k: int = 0, temperature: float = 1.0,
                   ignore_index: int = -100) -> TokenLogprobs:
    """Per row of logits: the log probability of its target token, the entropy
    of the distribution and, with ``top_k`` > 0 (at most 64), the ``top_k`` most
    probable tokens with their log probabilities, ties to the lowest index.
    Ignored rows give zeros (alternatives 0 and -1) and no gradient.  The
    alternatives carry no gradient, and there is no derivative in forward mode."""
    refuse_tangents("token_logprobs", (logits,))
    if torch.is_grad_enabled() and logits.requires_grad:
        return TokenLogprobs(*_TokenLogprobs.apply(logits, targets, top_k, temperature, ignore_index))
    return _values(logits, targets, top_k, temperature, ignore_index)
