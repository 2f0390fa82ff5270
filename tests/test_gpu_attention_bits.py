"""bfloat16 attention of few rows and of few keys: probabilities and the scores'
gradients enter their products with 16 bits, so that the results' own rounding is
nearly all of the error.

Tolerances as in attention_reference.py, apart from the products' operands: what
bfloat16's rounding of p leaves over (2^-8 of it) is rounded in turn, 2^-16 of p in
all.  out as delta = sum dout out takes it is out with what its rounding left over,
2^-16 too.  Keys are few, so that the chains' and the scores' terms are smaller than
that; where results are small beside their terms a p of 8 bits is off by ten times
the tolerance and more.
"""
import pytest
import torch

from attention_reference import HALF, TINY, U, reference
from paper_2405_15593_amd.attention import attention
from test_gpu_attention import inputs, run

pytestmark = pytest.mark.gpu

TWO = 2.0 ** -16


def tolerances(q, k, v, dout, causal, scale):
    """Of out, dq, dk and dv before their last rounding."""
    q, k, v, dout = (t.cpu().double().transpose(1, 2).contiguous() for t in (q, k, v, dout))
    b, h, sq, d = q.shape
    hk, sk = k.shape[1:3]
    kk, vv = (t.repeat_interleave(h // hk, 1) for t in (k, v))
    seen = torch.ones(sq, sk, dtype=torch.bool)
    if causal:
        seen = seen.tril(sk - sq)
    z = (q @ kk.transpose(2, 3) * scale).masked_fill(~seen, -torch.inf)
    p = torch.where(seen.any(1, keepdim=True), torch.softmax(z, 3), torch.zeros(())).nan_to_num(0.0)
    size = torch.where(seen, q.abs() @ kk.abs().transpose(2, 3) * scale, torch.zeros(()))
    zs = torch.where(seen, z, torch.zeros(())).abs()
    es = size * (d + 2) * U
    ep = p * (2 * (es + es.amax(3, keepdim=True)) + U * (sk + 16 + 4.4 * (zs + zs.amax(3, keepdim=True)))) + TINY
    out, eout = p @ vv, (ep + (TWO + sk * U) * p) @ vv.abs()
    dp = dout @ vv.transpose(2, 3)
    delta = (dout * out).sum(3, keepdim=True)
    ds = p * (dp - delta)
    edelta = (dout.abs() * (eout + TWO * (out.abs() + eout) * 1.01 + 2 * d * U * out.abs())).sum(3, keepdim=True)
    eds = ep * (dp - delta).abs() + (p + ep) * (edelta + (d + 2) * U * (dout.abs() @ vv.abs().transpose(2, 3)) +
                                                2 * U * (dp - delta).abs())
    eds = eds + TWO * (ds.abs() + eds) + TINY
    rows = h // hk * sq
    edq = scale * ((eds + sk * U * ds.abs()) @ kk.abs())
    edk = scale * ((eds + rows * U * ds.abs()).transpose(2, 3) @ q.abs())
    edv = (ep + TWO * (p + ep) + rows * U * p).transpose(2, 3) @ dout.abs()
    edk, edv = (t.reshape(b, hk, h // hk, sk, d).sum(2) for t in (edk, edv))
    return [t.transpose(1, 2) for t in (eout, edq, edk, edv)]


def check(got, want, tolerance):
    for what, g, w, t in zip(("out", "dq", "dk", "dv"), got, want, tolerance):
        off = (g.detach().cpu().double() - w).abs()
        allowed = t + HALF[torch.bfloat16] * (w.abs() + t) * 1.01 + TINY
        assert bool((off <= allowed).all()), (what, float((off / allowed).max()))


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("shape", [(1, 40, 20, 2, 2, 32), (2, 33, 33, 2, 1, 64), (3, 7, 12, 8, 2, 96), (1, 130, 40, 3, 3, 128),
                                   (2, 64, 6, 4, 4, 24), (1, 1, 24, 4, 1, 128)], ids=lambda s: "x".join(map(str, s)))
def test_few_rows_and_keys(shape, causal):
    print(f"[bits] {shape} causal {causal}", flush=True)
    given = inputs(*shape, torch.bfloat16, seed=sum(shape))
    scale = shape[5] ** -0.5
    want = reference(*given, causal, None, scale, torch.bfloat16)[0]
    check(run(*given, causal=causal), want, tolerances(*given, causal, scale))


@pytest.mark.parametrize("shape", [(300, 1, 24, 8, 1, 128), (2, 1, 1500, 4, 1, 64), (1, 3, 2100, 2, 1, 96)],
                         ids=lambda s: "x".join(map(str, s)))
def test_tokens(shape):
    """Single queries of many sequences, and keys in parts of which the first few
    are there."""
    print(f"[bits] tokens {shape}", flush=True)
    q, k, v, dout = inputs(*shape, torch.bfloat16, seed=sum(shape))
    there = min(shape[2], 24)
    lengths = torch.full((shape[0],), there, dtype=torch.int32, device="cuda")
    k1, v1, scale = k[:, :there], v[:, :there], shape[5] ** -0.5
    want = reference(q, k1, v1, dout, False, None, scale, torch.bfloat16)[0]
    check((attention(q, k, v, key_lengths=lengths),), want, tolerances(q, k1, v1, dout, False, scale))
