"""Attention and its gradients in binary64 on the CPU, with how far a kernel of
binary32 accumulators and products of the operands' dtype may be off.

With u = 2^-24 and h half a step of the dtype (2^-8 for bfloat16, u for binary32):
a score is a chain of dim products, off by (dim + 2) u scale |q| |k|; in a
probability that error counts once in the exponent and once in the sum, as do
the roundings of the exponent's argument (3 u of its size, in units of ln 2),
and the sum's chain of at most `keys` terms with its factors adds (keys + 16) u.
p and ds are rounded to the dtype before their products (h each), the products
summed in chains of at most `keys` (or rows) terms.  delta = sum dout out takes
out with what its rounding left over, which is rounded itself (h of h).  Results are rounded once (h).

Below binary32's normal range 2^-126 there are no relative errors: the
exponential gives zero there, and the matrix cores take smaller operands as
zeros.  So every p, every ds and every result may be off by TINY = 2^-126 besides
(seen in dv at scores 100 below the largest: 2.9e-41 more than the relative terms).
"""
import math

import torch

U = 2.0 ** -24
TINY = 2.0 ** -126
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def reference(q, k, v, dout, causal, lengths, scale, dtype):
    """((out, dq, dk, dv), their tolerances)."""
    h = HALF[dtype]
    q, k, v, dout = (t.detach().cpu().double().transpose(1, 2).contiguous() for t in (q, k, v, dout))
    b, nh, sq, d = q.shape
    hk, sk = k.shape[1:3]
    group = nh // hk
    k, v = k.clone(), v.clone()
    seen = torch.ones(b, 1, sq, sk, dtype=torch.bool)
    if causal:
        seen &= torch.ones(sq, sk, dtype=torch.bool).tril(sk - sq)
    if lengths is not None:
        there = torch.arange(sk) < lengths.cpu()[:, None]
        seen = seen & there[:, None, None, :]
        for t in (k, v):
            t.masked_fill_(~there[:, None, :, None], 0.0)     # what lies there is not read
    kk, vv = (t.repeat_interleave(group, 1) for t in (k, v))
    z = (q @ kk.transpose(2, 3)) * scale
    size = (q.abs() @ kk.abs().transpose(2, 3)) * scale
    z = z.masked_fill(~seen, -math.inf)
    top = z.amax(3, keepdim=True) if sk else torch.full((b, nh, sq, 1), -math.inf, dtype=z.dtype)
    some = top != -math.inf
    p = torch.exp(z - torch.where(some, top, torch.zeros_like(top)))
    total = p.sum(3, keepdim=True)
    p = p / torch.where(some, total, torch.ones_like(total))
    out = p @ vv
    zs = torch.where(seen, z.abs(), torch.zeros_like(z))
    most = zs.amax(3, keepdim=True) if sk else torch.zeros_like(top)
    es = torch.where(seen, size, torch.zeros_like(size)) * (d + 2) * U
    ep = p * (2 * (es + (es.amax(3, keepdim=True) if sk else 0)) + U * (sk + 16 + 3 * 1.45 * (zs + most))) + TINY
    eout = (ep + h * p) @ vv.abs() + sk * U * (p @ vv.abs())
    dp = dout @ vv.transpose(2, 3)
    delta = (dout * out).sum(3, keepdim=True)
    ds = p * (dp - delta)
    edelta = (dout.abs() * (eout + h * h * (out.abs() + eout) * 1.01 + 2 * d * U * out.abs())).sum(3, keepdim=True)
    eds = ep * (dp - delta).abs() + (p + ep) * (edelta + (d + 2) * U * (dout.abs() @ vv.abs().transpose(2, 3)) +
                                                2 * U * (dp - delta).abs())
    eds = eds + h * (ds.abs() + eds) + TINY
    rows = group * sq
    dq, edq = scale * (ds @ kk), scale * ((eds + sk * U * ds.abs()) @ kk.abs())
    dk, edk = scale * (ds.transpose(2, 3) @ q), scale * ((eds + rows * U * ds.abs()).transpose(2, 3) @ q.abs())
    dv, edv = p.transpose(2, 3) @ dout, (ep + h * (p + ep) + rows * U * p).transpose(2, 3) @ dout.abs()

    def shared(t):
        return t.reshape(b, hk, group, sk, d).sum(2)

    results = (out, dq, shared(dk), shared(dv))
    errors = (eout, edq, shared(edk), shared(edv))
    return tuple(t.transpose(1, 2) for t in results), tuple(t.transpose(1, 2) for t in errors)


def check(got, want, tolerance, dtype, what=("out", "dq", "dk", "dv")):
    for name, g, w, t in zip(what, got, want, tolerance):
        assert g.dtype == dtype and g.shape == w.shape, name
        g = g.detach().cpu().double()
        off = (g - w).abs()
        allowed = t + HALF[dtype] * (w.abs() + t) * 1.01 + TINY
        assert bool((off <= allowed).all()), (name, float((off - allowed).max()), float(off.max()))
