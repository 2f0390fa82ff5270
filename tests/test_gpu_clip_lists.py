"""Gradient lists of several launches: thousands of small gradients, which the
caches hold however many chunks they take, and a whole model's, of more than 256 MiB
and both dtypes.  Tolerances as in test_gpu_clip.py."""
import math

import pytest
import torch

from paper_2405_15593_amd.clip import clip_grads, grad_norm, workspace_bytes
from test_gpu_clip import HALF, SLACK, bucket, check_norm

pytestmark = pytest.mark.gpu


def norm_of(grads):
    return math.sqrt(float(sum(g.double().square().sum() for g in grads)))


def check_scaled(after, before, factor):
    floor = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134}[after.dtype]
    for a, b in zip(after.reshape(-1).split(1 << 25), before.reshape(-1).split(1 << 25)):
        exact = b.double() * factor
        assert bool(((a.double() - exact).abs() <= exact.abs() * HALF[a.dtype] * SLACK + floor).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_thousands_of_small_gradients(dtype):
    """Two megabytes in 9000 gradients: the norm is not written to the workspace by
    a launch of its own, as it is for a list past the caches."""
    print(f"[clip] small ones {dtype}", flush=True)
    flat, grads = bucket([(i % 97 + 1,) for i in range(9000)], dtype, start=1)
    before, want = flat.clone(), norm_of([flat[1:-5]])
    store = torch.full((workspace_bytes() // 8,), -7.0, dtype=torch.float64, device="cuda")
    workspace = store.view(torch.uint8)
    limit = 0.37 * want
    check_norm(clip_grads(grads, limit, workspace=workspace), want)
    assert float(store[-1]) == -7.0
    check_scaled(flat[1:-5], before[1:-5], limit / (want + 1e-6))
    assert torch.equal(flat[:1], before[:1]) and torch.equal(flat[-5:], before[-5:])
    check_norm(grad_norm(grads, workspace=workspace), norm_of([flat[1:-5]]))


@pytest.mark.parametrize("limit", [0.37, 2.0], ids=["above", "below"])
def test_a_whole_model(limit):
    """700 gradients, 377 MB, matrices in bfloat16 and vectors in binary32 in turn."""
    print(f"[clip] whole model {limit}", flush=True)
    matrices, wide = bucket([(1021, 517 + i % 5) for i in range(350)], torch.bfloat16, seed=1, start=3)
    vectors, thin = bucket([(3001 + 7 * i,) for i in range(350)], torch.float32, seed=2, start=1)
    assert matrices.nbytes + vectors.nbytes > 256 << 20
    grads = [g for pair in zip(wide, thin) for g in pair]
    before = [matrices.clone(), vectors.clone()]
    want = norm_of([matrices[3:-5], vectors[1:-5]])
    check_norm(grad_norm(grads), want)
    check_norm(clip_grads(grads, limit * want), want)
    if limit > 1:
        assert torch.equal(matrices, before[0]) and torch.equal(vectors, before[1])
        return
    factor = limit * want / (want + 1e-6)
    for after, old, start in ((matrices, before[0], 3), (vectors, before[1], 1)):
        check_scaled(after[start:-5], old[start:-5], factor)
        assert torch.equal(after[:start], old[:start]) and torch.equal(after[-5:], old[-5:])
    again = [matrices.clone(), vectors.clone()]
    for t, old in zip((matrices, vectors), before):
        t.copy_(old)
    clip_grads(grads, limit * want)
    assert torch.equal(matrices, again[0]) and torch.equal(vectors, again[1])
