"""Attention over many keys, each of which counts (attention_needles.py): tiles and
parts that are lost, repeated or misread show."""
import pytest
import torch

from attention_needles import check_even, check_needles, even, limits, needles
from paper_2405_15593_amd.attention import attention
from test_gpu_attention import TYPES, inputs, some_lengths

pytestmark = pytest.mark.gpu

SHAPES = [
    # past the caches: a token's kernels of both types
    (1, 1, 132000, 8, 4, 128), (2, 2, 132000, 4, 4, 64), (3, 3, 180000, 2, 1, 128), (1, 16, 140000, 4, 2, 128),
    # within them, keys in parts and not
    (1, 1, 9001, 3, 3, 40), (2, 1, 32768, 8, 2, 128), (1, 9, 70001, 1, 1, 24), (3, 40, 9001, 2, 1, 96), (70, 1, 5003, 4, 4, 64),
    # prompts
    (1, 130, 9001, 2, 2, 64), (2, 300, 6001, 48, 48, 32), (1, 515, 3001, 64, 64, 128), (1, 520, 2077, 56, 56, 80),
]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_every_key_counts(shape, causal, types):
    print(f"[needles] {shape} causal {causal} {types}", flush=True)
    b, sq, sk, h, hk, d = shape
    some = [None] if sq > 100 else [None, some_lengths(b, sk), torch.full((b,), sk * 2 // 3, dtype=torch.int32, device="cuda")]
    q, k, v, place = even(*shape, TYPES[types], "cuda")
    for lengths in some:
        rows = slice(0, sq, 1 if sq < 50 else 37)
        n = limits(b, sq, sk, causal, lengths)
        out = attention(q, k, v, causal=causal, key_lengths=lengths)
        check_even(out[:, rows], place, n[:, rows])
    scale = d ** -0.5
    q, k, v, at, score = needles(*shape, TYPES[types], "cuda", scale)
    for lengths in some:
        n = limits(b, sq, sk, causal, lengths)
        out = attention(q, k, v, causal=causal, key_lengths=lengths)
        check_needles(out[:, rows], at, score, n[:, rows], hk, d)


@pytest.mark.parametrize("types,keys", [("bf16", 1100), ("f32", 600)])
def test_past_the_caches_and_within(types, keys):
    """Of one call over 256 MiB and of its halves, which find their keys in the
    caches' kernels, the bits are the same."""
    print(f"[needles] halves {types}", flush=True)
    q, k, v, _ = inputs(128, 1, keys, 8, 4, 128, TYPES[types])
    assert k.nbytes + v.nbytes > 256 << 20 > (k.nbytes + v.nbytes) // 2
    lengths = torch.randint(0, keys + 1, (128,), dtype=torch.int32, device="cuda")
    for n in (None, lengths):
        whole = attention(q, k, v, key_lengths=n)
        for part in (slice(0, 64), slice(64, 128)):
            half = attention(q[part], k[part], v[part], key_lengths=None if n is None else n[part])
            assert torch.equal(whole[part], half)
