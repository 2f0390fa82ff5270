"""Muon, MicroAdamW and token_logprobs together in the package's training loop."""
import pytest
import torch

from paper_2405_15593_amd.insitu import train

pytestmark = pytest.mark.gpu


def test_training_with_muon():
    """The loss falls as far as the loop's own test asks of MicroAdam alone;
    the state is one float32 momentum per matrix element and MicroAdam's for
    the rest."""
    print("[muon] in-situ training", flush=True)
    kw = dict(vocab=512, dim=128, layers=2, heads=4, seq=64, batch=16, lr=2e-3, log_every=25)
    r = train("muon", 150, **kw)
    first, last = r["losses"][0][1], r["final_loss"]
    print(f"[muon] loss {first:.3f} -> {last:.3f} (floor {r['loss_floor']:.3f}), "
          f"state {r['state_bytes_per_param']:.3f} B/param", flush=True)
    assert last < first - 0.8 and last > r["loss_floor"] - 0.2
    assert r["state_bytes_per_param"] < 4.5
    # the loss is cross entropy: the same first value as with the other loop's
    assert abs(first - train("microadam", 1, **kw)["losses"][0][1]) < 1e-4
    torch.cuda.synchronize()
