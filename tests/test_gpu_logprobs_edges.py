"""Rows of logits where two of the header's rules meet."""
import math

import pytest
import torch

from paper_2405_15593_amd.logprobs import token_logprobs_and_grad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [100, 3000, 70001])
def test_a_bad_token_where_none_can_occur(vocab, dtype):
    """A row with no possible token and a token outside the vocabulary: the bad
    token decides, as for logp; an ignored row stays zeros."""
    print(f"[logprobs] bad token, empty row {vocab} {dtype}", flush=True)
    x = torch.zeros(6, vocab, dtype=dtype, device="cuda")
    x[:4] = -math.inf
    t = torch.tensor([vocab, -1, 5, -100, vocab, 7], device="cuda")
    one = torch.ones(6, device="cuda")
    for gh in (None, one):
        r = token_logprobs_and_grad(x, t, one, gh)
        for i in range(6):
            assert bool(r.grad[i].isnan().all()) == bool(r.grad[i].isnan().any()) == (i in (0, 1, 4)), i
            assert math.isnan(float(r.logp[i])) == (i in (0, 1, 4))
        assert bool((r.grad[2:4] == 0).all())
        assert bool((r.entropy[:4] == 0).all())
