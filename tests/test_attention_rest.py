"""What bfloat16's rounding of attention's out leaves over: the forward pass saves it,
and the backward pass takes it into delta = sum dout out.

Queries and keys have no element in common, so that scores are zero and each of n
keys has the probability 1 / n, exact up to binary32's roundings.  The values of a head
differ by a few of bfloat16's steps: out lies between them, and dp - delta is as small
as what its rounding takes away.  A delta of the rounded out is off by that whole
difference, a delta of out and what is saved besides by 2^-16 of sum |dout out|.
"""
import math

import pytest
import torch

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.attention import attention

U, H = 2.0 ** -24, 2.0 ** -8


def inputs(b, sq, sk, h, hk, d, device, seed=0):
    g = torch.Generator().manual_seed(seed)
    q, k = torch.randn(b, sq, h, d, generator=g), torch.randn(b, sk, hk, d, generator=g)
    q[..., d // 2:], k[..., :d // 2] = 0.0, 0.0
    base = 1.0 + torch.randint(0, 64, (b, 1, hk, d), generator=g) * 2.0 ** -7     # up to 1.5
    v = base + torch.randint(0, 3, (b, sk, hk, d), generator=g) * 2.0 ** -7
    v = v * (torch.randint(0, 2, (b, 1, hk, d), generator=g) * 2 - 1)
    dout = torch.randn(b, sq, h, d, generator=g)
    return [t.to(device).bfloat16() for t in (q, k, v, dout)]


def wanted(q, k, v, dout, rounded_out=False):
    """(out, dq, dk) in binary64 and their tolerances before the last rounding;
    `rounded_out`: with the mistake that delta is of out as it is returned."""
    q, k, v, dout = (t.cpu().double().transpose(1, 2) for t in (q, k, v, dout))
    (b, h, sq, d), (hk, n) = q.shape, k.shape[1:3]
    kk, vv = (t.repeat_interleave(h // hk, 1) for t in (k, v))
    scale = d ** -0.5
    out = vv.mean(2, keepdim=True).expand(b, h, sq, d)
    taken = out.bfloat16().double() if rounded_out else out
    dp, delta = dout @ vv.transpose(2, 3), (dout * taken).sum(3, keepdim=True)
    ds = (dp - delta) / n
    size = (dout.abs() * out.abs()).sum(3, keepdim=True)
    # delta: what is saved is rounded, and out's sum and chains; dp's chain; ds's rounding
    eds = (2.0 ** -16 * 1.01 + 4 * (d + n) * U) * size / n + 1.01 * H * ds.abs()
    dq, edq = scale * ds @ kk, scale * (eds + n * U * ds.abs()) @ kk.abs()
    dk, edk = (scale * t.transpose(2, 3) @ r for t, r in ((ds, q), (eds + h // hk * sq * U * ds.abs(), q.abs())))
    dk, edk = (t.reshape(b, hk, h // hk, n, d).sum(2) for t in (dk, edk))
    return [t.transpose(1, 2) for t in (out, dq, dk)], [t.transpose(1, 2) for t in (edq, edk)]


def check(got, want, tolerance):
    for what, g, w, t in zip(("dq", "dk"), got, want[1:], tolerance):
        off = (g.cpu().double() - w).abs()
        assert bool((off <= t + H * 1.01 * (w.abs() + t) + 2.0 ** -126).all()), (what, float((off / (t + H * w.abs())).max()))


# (batch, queries, keys, heads, kv_heads, dim, keys that there are): shared waves; workgroups
# of 128 rows; rows in parts; keys in parts; a token's
CASES = [(1, 200, 2, 4, 4, 64, 2), (2, 70, 12, 4, 2, 128, 12), (3, 33, 5, 2, 1, 96, 5), (16, 256, 3, 16, 16, 64, 3),
         (16, 130, 7, 32, 16, 128, 7), (1, 600, 12, 16, 1, 64, 12), (1, 40, 1200, 1, 1, 64, 9), (2, 2, 1500, 4, 1, 128, 11),
         (1, 3, 2000, 2, 2, 32, 2000)]
IDS = ["x".join(map(str, c)) for c in CASES]


def given(case, device):
    q, k, v, dout = inputs(*case[:6], device, seed=sum(case))
    n = case[6]
    return q, k, v, dout, k[:, :n], v[:, :n], None if n == case[2] else torch.full((case[0],), n, dtype=torch.int32, device=device)


@pytest.mark.parametrize("case", CASES[:5], ids=IDS[:5])
def test_a_rounded_delta_shows(case):
    q, _, _, dout, k, v, _ = given(case, "cpu")
    right, tolerance = wanted(q, k, v, dout)
    check([t.bfloat16() for t in right[1:]], right, tolerance)
    wrong = wanted(q, k, v, dout, rounded_out=True)[0]
    for i in (0, 1):
        with pytest.raises(AssertionError):
            check([t.bfloat16() if i == j else r.bfloat16() for j, (t, r) in enumerate(zip(wrong[1:], right[1:]))], right, tolerance)


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_gradients(case):
    print(f"[rest] gradients {case}", flush=True)
    q, k, v, dout, seen_k, seen_v, lengths = given(case, "cuda")
    leaves = [t.requires_grad_() for t in (q, k)]
    dq, dk = torch.autograd.grad(attention(q, k, v, key_lengths=lengths), leaves, dout)
    want, tolerance = wanted(q.detach(), seen_k.detach(), seen_v, dout)
    check((dq, dk[:, :case[6]]), want, tolerance)
    assert not dk[:, case[6]:].any()


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_what_is_saved(case):
    """out and what is saved besides are out to 16 bits."""
    print(f"[rest] saved {case}", flush=True)
    q, k, v, _, _, seen, lengths = given(case, "cuda")
    b, sq, sk, h, hk, d, n = case

    def heads(t):
        return ma.microadam_heads(t.data_ptr(), *t.stride()[:3])

    a = ma.microadam_attention(heads(q), heads(k), heads(v), None if lengths is None else lengths.data_ptr(), b, sq, sk, h, hk,
                               d, d ** -0.5, ma.MICROADAM_BF16, 0)
    saved = torch.full((ma.microadam_attention_saved(a),), 255, dtype=torch.uint8, device="cuda")
    workspace = torch.empty(max(256, ma.microadam_attention_workspace(a, False)), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    ma.microadam_attention_forward(a, heads(out), saved.data_ptr(), saved.numel(), workspace.data_ptr(), workspace.numel(),
                                   torch.cuda.current_stream().cuda_stream)
    count = b * h * sq
    lse = saved[:4 * count].view(torch.float32)
    assert float((lse.double() - math.log2(n)).abs().max()) <= 4 * U * max(1.0, math.log2(n))
    at = (4 * count + 255) // 256 * 256
    rest = saved[at:at + 2 * count * d].view(torch.bfloat16).view(b, h, sq, d).transpose(1, 2)
    want = seen.double().mean(1, keepdim=True).repeat_interleave(h // hk, 2).expand(b, sq, h, d)
    assert bool(((out.double() - want).abs() <= H * 1.01 * want.abs()).all()) and bool(rest.any())
    assert bool(((out.double() + rest.double() - want).abs() <= (2.0 ** -16 * 1.01 + (n + 4) * U) * want.abs()).all())
