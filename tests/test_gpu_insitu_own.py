"""The training step's operators together, as the package's training loop runs
them: layer norm, attention, loss, clipping, optimizers."""
import pytest
import torch

from paper_2405_15593_amd.attention import attention
from paper_2405_15593_amd.clip import clip_grads, grad_norm
from paper_2405_15593_amd.insitu import MarkovTokens, TinyLM, train
from paper_2405_15593_amd.logprobs import token_logprobs
from paper_2405_15593_amd.norm import layer_norm

pytestmark = pytest.mark.gpu

SIZES = dict(vocab=211, dim=96, layers=2, heads=4, seq=50)


def model(own, dtype=torch.float32):
    torch.manual_seed(3)
    return TinyLM(*SIZES.values(), own=own).to("cuda", dtype)


def gradients(m, x, y, own):
    logits = m(x)
    logp = (token_logprobs(logits, y).logp if own
            else torch.log_softmax(logits, -1).gather(-1, y[..., None])[..., 0])
    loss = -logp.mean()
    return loss.detach(), dict(zip((n for n, _ in m.named_parameters()), torch.autograd.grad(loss, list(m.parameters()))))


def test_gradients_of_the_model():
    """Against the same model in binary64 with torch's operators.  Some twenty
    operators lie one behind the other in two layers, forward and backward, each
    off by at most 100 u of its result's norm (chains of up to 100 terms): 40 x
    100 u = 2^-12."""
    print("[own] gradients", flush=True)
    x, y = MarkovTokens(211, 50, 7, "cuda").next()
    loss, grads = gradients(model(True), x, y, True)
    want_loss, want = gradients(model(False, torch.float64), x, y, False)
    assert abs(float(loss) - float(want_loss)) < 2.0 ** -12 * float(want_loss)
    for name, g in grads.items():
        off = float((g.double() - want[name]).norm() / want[name].norm())
        assert off < 2.0 ** -12, (name, off)


@pytest.mark.parametrize("opt", ["microadam", "muon"])
def test_training_step(opt):
    """The loop runs, its norm is the gradients', and the first loss is the one
    of torch's operators."""
    print(f"[own] training {opt}", flush=True)
    kw = dict(vocab=256, dim=128, layers=2, heads=4, seq=64, batch=8, lr=1e-3, log_every=1)
    own = train(opt, 4, own=True, max_norm=0.1, **kw)
    plain = train(opt, 1, **kw)
    assert abs(own["losses"][0][1] - plain["losses"][0][1]) < 2.0 ** -12 * plain["losses"][0][1]
    assert len(own["losses"]) == 4 and all(torch.isfinite(torch.tensor(v)) for _, v in own["losses"])
    assert own["grad_norm"] > 0.1 and "grad_norm" not in plain


def test_clipped_gradients_reach_the_optimizer():
    print("[own] clipped", flush=True)
    m = model(True)
    x, y = MarkovTokens(211, 50, 7, "cuda").next()
    (-token_logprobs(m(x), y).logp.mean()).backward()
    grads = [p.grad for p in m.parameters()]
    before = float(grad_norm(grads))
    assert abs(float(clip_grads(grads, 0.25 * before)) - before) <= 2.0 ** -23 * before
    # each element is rounded once, and the limit lies 1e-6 / norm above the result
    assert abs(float(grad_norm(grads)) / (0.25 * before) - 1) < 2.0 ** -22 + 2e-6 / before


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_step_in_a_graph(dtype):
    """Layer norm, attention, loss, their gradients and clipping, captured
    together and replayed on new values."""
    print(f"[own] graph {dtype}", flush=True)
    b, s, h, d = 3, 70, 4, 32
    g = torch.Generator(device="cuda").manual_seed(1)

    def values():
        return [(torch.randn(shape, generator=g, device="cuda")).to(dtype)
                for shape in ((b, s, 3 * h * d), (3 * h * d,), (3 * h * d,))]

    targets = torch.randint(0, h * d, (b, s), generator=g, device="cuda")

    def step(leaves):
        q, k, v = layer_norm(*leaves).view(b, s, 3, h, d).unbind(2)
        logits = attention(q, k, v, causal=True).reshape(b, s, h * d)
        loss = -token_logprobs(logits, targets).logp.mean()
        grads = [t.clone() for t in torch.autograd.grad(loss, leaves)]
        return [loss.detach(), clip_grads(grads, 1e-2), *grads]

    leaves = [t.requires_grad_() for t in values()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(leaves)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step(leaves)
    for _ in range(4):
        new = values()
        with torch.no_grad():
            for t, n in zip(leaves, new):
                t.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        eager = step([t.requires_grad_() for t in new])
        assert float(eager[1]) > 1e-2
        for c, e in zip(captured[1:], eager[1:]):
            assert torch.equal(c, e)
