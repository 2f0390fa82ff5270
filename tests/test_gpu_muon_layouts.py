"""Stacks whose matrices lie between each other's rows: a fused projection's
(rows, 3, cols) taken as three matrices.  The same values come out as from
contiguous stacks, bit for bit, since the kernels work on their own copy."""
import pytest
import torch

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.muon import Muon, muon_step, orthogonalize

pytestmark = pytest.mark.gpu


def fused(seed, rows=40, parts=3, cols=24, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, parts, cols, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lead", [(3,), (2, 2)], ids=str)
def test_interleaved_stacks(lead, dtype):
    print(f"[layouts] {lead} {dtype}", flush=True)
    n = lead[0] * (lead[1] if len(lead) > 1 else 1)

    def parted(t):   # (rows, n, cols) as a stack of n, or 2 x 2, matrices
        t = t.permute(1, 0, 2)
        return t.unflatten(0, lead) if len(lead) > 1 else t

    grad, param = fused(1, parts=n, dtype=dtype), fused(2, parts=n, dtype=dtype)
    whole = torch.full((40, n, 30), 7.0, dtype=dtype, device="cuda")
    out = parted(whole[:, :, 2:26])
    want = orthogonalize(parted(grad).contiguous())
    assert torch.equal(orthogonalize(parted(grad)), want)
    assert orthogonalize(parted(grad), out=out) is out and torch.equal(out, want)
    assert bool((whole[:, :, :2] == 7).all()) and bool((whole[:, :, 26:] == 7).all())
    p, v = parted(param.clone()), parted(torch.zeros_like(param))
    q, w = parted(param).contiguous(), torch.zeros_like(want)
    for _ in range(2):
        muon_step([p], [parted(grad)], [v], lr=0.1)
        muon_step([q], [parted(grad)], [w], lr=0.1)
    assert torch.equal(p, q) and torch.equal(v, w)


def test_the_optimizer_takes_them():
    print("[layouts] Muon", flush=True)
    a = torch.nn.Parameter(fused(3).permute(1, 0, 2))
    b = torch.nn.Parameter(a.detach().contiguous())
    assert not a.is_contiguous()
    grad = fused(4).permute(1, 0, 2)
    opts = [Muon([a], lr=0.1), Muon([b], lr=0.1)]
    for _ in range(2):
        for p, o in zip((a, b), opts):
            p.grad = grad.clone()
            o.step()
    assert torch.equal(a, b)


def test_stacks_that_overlap_are_refused():
    print("[layouts] refusals", flush=True)
    store = torch.zeros(4000, device="cuda")
    grad = fused(5, rows=8, parts=3, cols=16).permute(1, 0, 2).contiguous()
    for strides in ((15, 48, 1), (48, 48, 1), (0, 48, 1), (64, 49, 1)):
        out = store.as_strided((3, 8, 16), strides)
        with pytest.raises((ValueError, ma.MicroAdamError)):
            orthogonalize(grad, out=out)
        with pytest.raises((ValueError, ma.MicroAdamError)):
            muon_step([out], [grad], [torch.zeros_like(grad)], lr=0.1)
    assert bool((store == 0).all())
    # row i of one and row i + 1 of another side by side
    assert torch.equal(orthogonalize(grad, out=store.as_strided((3, 8, 16), (64, 48, 1))), orthogonalize(grad))
