"""Queries that see no key take no part in the gradients, whatever q and dout hold
there: dk and dv have the same bits, out and dq zeros."""
import math

import pytest
import torch

from attention_reference import check, reference
from test_gpu_attention import TYPES, inputs, run

pytestmark = pytest.mark.gpu

# shared waves; workgroups of 128 keys, with values in LDS and without; rows in parts
SHAPES = [(1, 70, 50, 4, 2, 64), (2, 33, 1, 2, 2, 40), (1, 40, 39, 2, 1, 128), (16, 150, 100, 32, 32, 64), (8, 190, 150, 32, 32, 128),
          (8, 161, 130, 32, 32, 96), (1, 530, 270, 16, 1, 128), (1, 1081, 1050, 8, 1, 64), (3, 65, 32, 2, 1, 24)]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_keyless_queries(shape, types):
    print(f"[keyless] {shape} {types}", flush=True)
    b, sq, sk = shape[:3]
    q, k, v, dout = inputs(*shape, TYPES[types], seed=sum(shape))
    none = sq - sk
    q[:, :none], dout[:, :none] = 0.0, 0.0
    want = run(q, k, v, dout, causal=True)
    assert all(bool(t.isfinite().all()) for t in want)
    if b * shape[3] * sq * sk < 4e6:
        check(want, *reference(q, k, v, dout, True, None, shape[5] ** -0.5, TYPES[types]), TYPES[types])
    lengths = torch.full((b,), sk, dtype=torch.int32, device="cuda")
    lengths[b // 2:] = (sk + 1) // 2
    short = run(q, k, v, dout, causal=True, key_lengths=lengths)
    for bad in (math.nan, math.inf):
        q[:, :none], dout[:, :none] = bad, -bad
        for got, known in ((run(q, k, v, dout, causal=True), want),
                           (run(q, k, v, dout, causal=True, key_lengths=lengths), short)):
            assert all(torch.equal(g, w) for g, w in zip(got, known))
            assert not got[0][:, :none].any() and not got[1][:, :none].any()


@pytest.mark.parametrize("types", TYPES)
def test_sequences_without_keys(types):
    """All queries of a sequence of length 0."""
    print(f"[keyless] no keys {types}", flush=True)
    q, k, v, dout = inputs(3, 70, 80, 4, 2, 64, TYPES[types])
    lengths = torch.tensor([80, 0, 33], dtype=torch.int32, device="cuda")
    want = run(q, k, v, dout, key_lengths=lengths)
    q[1], dout[1] = math.nan, math.inf
    got = run(q, k, v, dout, key_lengths=lengths)
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    assert not any(t[1].any() for t in got)
