"""Matrix updates: orthogonalisation by Newton-Schulz products and the Muon
step, over the C ABI (``microadam_orthogonalize``, ``microadam_muon_step``).

``Muon`` is the ``torch.optim`` front-end for a model's weight matrices; its
other parameters (embeddings, norms, biases, the head) go to ``MicroAdamW``.
``orthogonalize`` and ``muon_step`` are the functions under it, for training
loops that keep their own lists.

Tensors are float32 or bfloat16 on a ROCm device, two-dimensional (rows,
cols) or stacks of matrices (..., rows, cols) with contiguous rows; a row
stride is allowed.  Every product runs in the library's kernels, on torch's
current stream, in a workspace that the call takes from torch's allocator
unless it is given one.
"""
from __future__ import annotations

import contextlib

import torch
from torch.autograd.graph import increment_version

from . import (MICROADAM_BF16, MICROADAM_F32, MICROADAM_PRECISION_AUTO, MICROADAM_PRECISION_F16,
               MICROADAM_PRECISION_SPLIT, MICROADAM_SCALE_MATCH_RMS, MICROADAM_SCALE_NONE, MICROADAM_SCALE_SPECTRAL,
               make_schulz_config, microadam_matrix, microadam_matrix_workspace, microadam_muon_config,
               microadam_muon_step, microadam_orthogonalize)
from ._autograd import refuse_tangents

_DTYPES = {torch.float32: MICROADAM_F32, torch.bfloat16: MICROADAM_BF16}
_PRECISIONS = {"auto": MICROADAM_PRECISION_AUTO, "f16": MICROADAM_PRECISION_F16, "split": MICROADAM_PRECISION_SPLIT}
_SCALES = {"match_rms": MICROADAM_SCALE_MATCH_RMS, "spectral": MICROADAM_SCALE_SPECTRAL,
           "none": MICROADAM_SCALE_NONE}


_HERE = contextlib.nullcontext()


def _on(device):
    """The device as the current one; nothing to do where it is."""
    return _HERE if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _code(t: torch.Tensor, what: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what}: float32 or bfloat16, not {t.dtype}")
    return code


def _schulz(steps, coefficients, eps, precision):
    if precision not in _PRECISIONS:
        raise ValueError(f"precision must be one of {sorted(_PRECISIONS)}")
    return make_schulz_config(steps, coefficients, eps, _PRECISIONS[precision])


def _matrices(t: torch.Tensor, what: str, written: bool = True) -> list:
    """(address, row stride) of each matrix of `t`.  Matrices that are written
    may lie between each other's rows, but not on each other: the library
    decides that for the whole list."""
    if t.dim() < 2:
        raise ValueError(f"{what}: a matrix or a stack of matrices, not {t.dim()} dimensions")
    r, c = t.shape[-2:]
    if (c > 1 and t.stride(-1) != 1) or (r > 1 and t.stride(-2) < c):
        raise ValueError(f"{what}: rows must be contiguous and not overlap")
    ld = t.stride(-2) if r > 1 else c
    if written and any(s == 0 and n > 1 for s, n in zip(t.stride()[:-2], t.shape[:-2])):
        raise ValueError(f"{what}: one matrix more than once in a stack")
    base, size = t.data_ptr(), t.element_size()
    if t.dim() == 2:
        return [(base, ld)]
    if t.dim() == 3:
        step = t.stride(0) * size
        return [(base + i * step, ld) for i in range(t.shape[0])]
    at = [0]
    for n, s in zip(t.shape[:-2], t.stride()[:-2]):
        at = [o + i * s * size for o in at for i in range(n)]
    return [(base + o, ld) for o in at]


def _workspace(cfg, array, n, out_dtype, device, workspace):
    """(address, bytes, the tensor that holds it): the caller's, or one of the
    useful size from torch's allocator."""
    if workspace is None:
        useful = microadam_matrix_workspace(cfg, array, n, out_dtype)[1]
        workspace = torch.empty(useful + 256, dtype=torch.uint8, device=device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != device:
        raise ValueError("workspace: a contiguous uint8 tensor on the matrices' device")
    off = (-workspace.data_ptr()) % 256
    return workspace.data_ptr() + off, max(0, workspace.numel() - off), workspace


def workspace_bytes(shapes, dtype: torch.dtype = torch.bfloat16, precision: str = "auto") -> tuple:
    """(least, useful) bytes of workspace for matrices of these (rows, cols)
    and results (parameters) of `dtype`, 256 bytes for alignment included."""
    shapes = list(shapes)
    array = (microadam_matrix * max(1, len(shapes)))()
    for a, (r, c) in zip(array, shapes):
        a.rows, a.cols = r, c
    lo, hi = microadam_matrix_workspace(_schulz(5, None, 1e-7, precision), array, len(shapes), _DTYPES[dtype])
    return lo + 256, hi + 256


def orthogonalize(grad: torch.Tensor, *, steps: int = 5, coefficients=None, eps: float = 1e-7,
                  precision: str = "auto", out: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None) -> torch.Tensor:
    """The orthogonalised matrix (or stack of matrices) of `grad`, in `out` if
    given (float32 or bfloat16; `grad` itself is allowed; autograd sees a write
    in place), else in a new tensor of grad's dtype.  It has no derivative:
    detach a tensor that requires grad."""
    refuse_tangents("orthogonalize", (grad, out))
    cfg = _schulz(steps, coefficients, eps, precision)
    gcode = _code(grad, "grad")
    if not grad.is_cuda:
        raise ValueError("grad: a tensor on a ROCm device")
    if grad.requires_grad and torch.is_grad_enabled():
        raise NotImplementedError("orthogonalize: no derivative; grad requires grad")
    if out is None:
        out = torch.empty(grad.shape, dtype=grad.dtype, device=grad.device)
    elif out.shape != grad.shape or out.device != grad.device:
        raise ValueError("out: grad's shape and device")
    elif out.requires_grad and torch.is_grad_enabled():
        raise ValueError("out: a tensor that requires grad")
    ocode = _code(out, "out")
    g, o = _matrices(grad, "grad", written=False), _matrices(out, "out")
    if grad.numel() == 0:
        return out
    r, c = grad.shape[-2:]
    array = (microadam_matrix * len(g))(*[(gp, None, op, r, c, gl, 0, ol) for (gp, gl), (op, ol) in zip(g, o)])
    with _on(grad.device):
        ptr, size, keep = _workspace(cfg, array, len(g), ocode, grad.device, workspace)
        microadam_orthogonalize(cfg, array, len(g), gcode, ocode, ptr, size,
                                torch.cuda.current_stream(grad.device.index).cuda_stream)
    increment_version(out)
    return out


def muon_step(params, grads, momenta, *, lr: float, momentum: float = 0.95, nesterov: bool = True,
              weight_decay: float = 0.0, scale: str = "match_rms", steps: int = 5, coefficients=None,
              eps: float = 1e-7, precision: str = "auto", workspace: torch.Tensor | None = None) -> None:
    """One Muon step: `params` and `momenta` (zeros before the first step) are
    updated in place from `grads`.  Three lists of equal length and shapes;
    one dtype per list.  Like an optimizer's step it is not recorded for
    autograd, whether the parameters require grad or not; a backward that saved
    what a parameter was before raises."""
    params, grads, momenta = list(params), list(grads), list(momenta)
    if not params or not len(params) == len(grads) == len(momenta):
        raise ValueError("params, grads and momenta: three lists of equal length")
    refuse_tangents("muon_step", params + grads + momenta)
    if scale not in _SCALES:
        raise ValueError(f"scale must be one of {sorted(_SCALES)}")
    cfg = microadam_muon_config(_schulz(steps, coefficients, eps, precision), float(momentum), float(weight_decay),
                                1 if nesterov else 0, _SCALES[scale])
    device = params[0].device
    if not params[0].is_cuda:
        raise ValueError("params: tensors on a ROCm device")
    codes = _code(grads[0], "grads"), _code(momenta[0], "momenta"), _code(params[0], "params")
    dtypes = grads[0].dtype, momenta[0].dtype, params[0].dtype
    rows = []
    for p, g, v in zip(params, grads, momenta):
        shape = p.shape
        if shape != g.shape or shape != v.shape:
            raise ValueError("a gradient or momentum has another shape than its parameter")
        if (g.dtype, v.dtype, p.dtype) != dtypes:
            raise TypeError("params, grads and momenta: one dtype per list")
        if not p.device == g.device == v.device == device:
            raise ValueError("params, grads and momenta: one device")
        if p.numel() == 0:
            raise ValueError("an empty matrix")
        if len(shape) == 2 and p.is_contiguous() and g.is_contiguous() and v.is_contiguous():
            r, c = shape
            rows.append((g.data_ptr(), v.data_ptr(), p.data_ptr(), r, c, c, c, c))
            continue
        r, c = shape[-2:] if len(shape) >= 2 else (0, 0)
        for (pp, pl), (gp, gl), (vp, vl) in zip(_matrices(p, "params"), _matrices(g, "grads", written=False),
                                                _matrices(v, "momenta")):
            rows.append((gp, vp, pp, r, c, gl, vl, pl))
    array = (microadam_matrix * len(rows))(*rows)
    with _on(device):
        ptr, size, keep = _workspace(cfg.schulz, array, len(rows), codes[2], device, workspace)
        microadam_muon_step(cfg, array, len(rows), *codes, lr, ptr, size,
                            torch.cuda.current_stream(device.index).cuda_stream)
    increment_version(params)
    increment_version(momenta)


class Muon(torch.optim.Optimizer):
    """Muon for weight matrices on a ROCm device (float32 or bfloat16, two or
    more dimensions; a parameter with more than two is a stack of matrices over
    its last two).  A convolution's weight is not such a stack, and nothing
    tells the two apart: its kernels would be orthogonalised one by one.  Give
    it to another optimizer.  ``momentum_dtype`` is the dtype of the one state tensor per
    parameter (None: the parameter's)."""

    def __init__(self, params, lr: float = 1e-3, momentum: float = 0.95, nesterov: bool = True,
                 weight_decay: float = 0.0, scale: str = "match_rms", steps: int = 5, coefficients=None,
                 eps: float = 1e-7, precision: str = "auto", momentum_dtype: torch.dtype | None = None):
        if not lr >= 0.0:
            raise ValueError(f"invalid lr {lr}")
        if not 0.0 <= momentum < 1.0:
            raise ValueError(f"invalid momentum {momentum}")
        if not weight_decay >= 0.0:
            raise ValueError(f"invalid weight_decay {weight_decay}")
        if not eps > 0.0:
            raise ValueError(f"invalid eps {eps}")
        if not 1 <= steps <= 16:
            raise ValueError(f"invalid steps {steps}")
        if scale not in _SCALES:
            raise ValueError(f"scale must be one of {sorted(_SCALES)}")
        if momentum_dtype is not None and momentum_dtype not in _DTYPES:
            raise ValueError("momentum_dtype must be float32, bfloat16 or None")
        _schulz(steps, coefficients, eps, precision)
        defaults = dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, scale=scale,
                        steps=steps, coefficients=coefficients, eps=eps, precision=precision,
                        momentum_dtype=momentum_dtype)
        super().__init__(params, defaults)
        for group in self.param_groups:
            for p in group["params"]:
                if p.dim() < 2:
                    raise ValueError("Muon takes matrices: give vectors and scalars to another optimizer")

    def state_bytes(self) -> int:
        """Bytes of the momenta held so far."""
        return sum(s["momentum"].numel() * s["momentum"].element_size() for s in self.state.values())

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            by_kind: dict = {}
            for p in group["params"]:
                if p.grad is None:
                    continue
                if p.dtype not in _DTYPES:
                    raise TypeError(f"Muon supports float32 and bfloat16 parameters, not {p.dtype}")
                state = self.state[p]
                if "momentum" not in state:
                    state["momentum"] = torch.zeros(p.shape, dtype=group["momentum_dtype"] or p.dtype,
                                                    device=p.device)
                g, v = p.grad, state["momentum"]
                if g.dtype not in _DTYPES:
                    g = g.float()
                by_kind.setdefault((p.device, p.dtype, g.dtype, v.dtype), []).append((p, g.contiguous(), v))
            for kind in by_kind.values():
                ps, gs, vs = zip(*kind)
                muon_step(ps, gs, vs, **{k: group[k] for k in ("lr", "momentum", "nesterov", "weight_decay", "scale",
                                                               "steps", "coefficients", "eps", "precision")})
        return loss

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)
        # torch casts floating state to the parameter's dtype: back to the saved one
        saved = [i for g in state_dict["param_groups"] for i in g["params"]]
        own = [p for g in self.param_groups for p in g["params"]]
        for i, p in zip(saved, own):
            if i in state_dict["state"]:
                self.state[p]["momentum"] = state_dict["state"][i]["momentum"].detach().to(p.device, copy=True)
