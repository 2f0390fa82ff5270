"""Argument checks of the attention entry points that need no GPU: every
refusal comes before any device work."""
import math
import os

import pytest
import torch

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.attention import attention

F32, BF16 = ma.MICROADAM_F32, ma.MICROADAM_BF16
INVALID, UNSUPPORTED, SIZE = (ma.MICROADAM_ERR_INVALID_ARG, ma.MICROADAM_ERR_UNSUPPORTED,
                              ma.MICROADAM_ERR_STATE_SIZE)
# addresses that no refusal follows, 16 mebibytes apart
Q, K, V, N, OUT, SAVED, DOUT, DQ, DK, DV, WS = ((i + 1) << 24 for i in range(11))
B, SQ, SK, H, HK, D = 2, 5, 7, 4, 2, 16


def heads(at, positions, count, **kw):
    h = dict(data=at, batch_stride=positions * count * D, pos_stride=count * D, head_stride=D)
    h.update(kw)
    return ma.microadam_heads(*h.values())


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ma.LIBRARY):
        from paper_2405_15593_amd import _build
        _build.build()
    return ma.load()


def given(**kw):
    a = dict(q=heads(Q, SQ, H), k=heads(K, SK, HK), v=heads(V, SK, HK), key_lengths=N, batch=B, queries=SQ, keys=SK,
             heads=H, kv_heads=HK, dim=D, scale=0.25, dtype=F32, causal=1)
    a.update(kw)
    return ma.microadam_attention(*a.values())


def forward(a, out=None, saved=SAVED, kept=1 << 24, ws=WS, size=1 << 24):
    ma.microadam_attention_forward(a, out or heads(OUT, SQ, H), saved, kept, ws, size)


def backward(a, out=None, saved=SAVED, kept=1 << 24, dout=None, dq=None, dk=None, dv=None, ws=WS, size=1 << 24):
    ma.microadam_attention_grad(a, out or heads(OUT, SQ, H), saved, kept, dout or heads(DOUT, SQ, H), dq or heads(DQ, SQ, H),
                                dk or heads(DK, SK, HK), dv or heads(DV, SK, HK), ws, size)


def refused(code, f, *args, **kw):
    with pytest.raises(ma.MicroAdamError) as e:
        f(*args, **kw)
    assert e.value.code == code, e.value


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), INVALID), (dict(causal=2), INVALID), (dict(causal=-1), INVALID), (dict(batch=-1), INVALID),
    (dict(queries=-1), INVALID), (dict(keys=-1), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID),
    (dict(kv_heads=3), INVALID), (dict(kv_heads=8), INVALID), (dict(dim=0), INVALID), (dict(dim=-8), INVALID),
    (dict(dim=12), UNSUPPORTED), (dict(dim=136), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=1e39), INVALID),
    (dict(scale=1e-46), INVALID), (dict(queries=(1 << 30) + 1), UNSUPPORTED), (dict(queries=1 << 30), UNSUPPORTED),
    (dict(keys=(1 << 30) + 1), UNSUPPORTED), (dict(batch=1 << 30, kv_heads=4), UNSUPPORTED)],
    ids=lambda v: str(v) if isinstance(v, dict) else "")
def test_sizes(kw, code):
    a = given(**kw)
    refused(code, forward, a)
    refused(code, backward, a)
    for grad in (False, True):
        refused(code, ma.microadam_attention_workspace, a, grad)


@pytest.mark.parametrize("name,positions,count,at", [("q", SQ, H, Q), ("k", SK, HK, K), ("v", SK, HK, V)])
@pytest.mark.parametrize("kw,code", [
    (dict(data=None), INVALID), (dict(data=Q + 2), INVALID), (dict(batch_stride=-1), INVALID),
    (dict(pos_stride=-16), INVALID), (dict(head_stride=-1), INVALID), (dict(pos_stride=(1 << 23) + 1), UNSUPPORTED),
    (dict(pos_stride=15), INVALID), (dict(pos_stride=0), INVALID), (dict(head_stride=(1 << 40) + 1), UNSUPPORTED)],
    ids=str)
def test_inputs(name, positions, count, at, kw, code):
    if kw.get("data"):
        kw = dict(data=at + 2)
    a = given(**{name: heads(at, positions, count, **kw)})
    refused(code, forward, a)
    refused(code, backward, a)


def test_inputs_with_shared_elements_are_allowed():
    """Where nothing is written, strides may be zero: up to the next refusal."""
    a = given(k=heads(K, SK, HK, batch_stride=0, head_stride=0))
    refused(INVALID, forward, a, saved=SAVED + 128)


@pytest.mark.parametrize("f,name,positions,count", [
    (forward, "out", SQ, H), (backward, "dq", SQ, H), (backward, "dk", SK, HK), (backward, "dv", SK, HK)])
@pytest.mark.parametrize("kw", [dict(data=None), dict(data=(1 << 28) + 1), dict(batch_stride=0), dict(pos_stride=15),
                                dict(head_stride=0), dict(head_stride=8), dict(batch_stride=40), dict(data=Q),
                                dict(data=K + 4), dict(data=V), dict(data=N)], ids=str)
def test_outputs(f, name, positions, count, kw):
    refused(INVALID, f, given(), **{name: heads(1 << 28, positions, count, **kw)})


def test_outputs_apart():
    a = given()
    refused(INVALID, forward, a, saved=OUT)
    refused(INVALID, forward, a, saved=Q + 512)
    refused(INVALID, forward, a, saved=SAVED + 4)
    refused(INVALID, backward, a, saved=None)
    refused(INVALID, backward, a, saved=SAVED + 4)
    refused(INVALID, backward, a, dq=heads(SAVED + 64, SQ, H))
    refused(INVALID, backward, a, dk=heads(DV + 4, SK, HK))
    refused(INVALID, backward, a, dq=heads(DOUT, SQ, H))
    refused(INVALID, backward, a, dq=heads(OUT, SQ, H))
    refused(INVALID, backward, a, dout=heads(None, SQ, H))
    refused(INVALID, forward, given(key_lengths=N + 2))


def test_workspace():
    need = ma.microadam_attention_workspace(given(), True)
    assert need == 256                                   # 2 x 4 x 5 sums, aligned
    refused(SIZE, backward, given(), size=need - 1)
    refused(INVALID, backward, given(), ws=None)
    refused(INVALID, backward, given(), ws=WS + 64)
    refused(INVALID, backward, given(), ws=Q)
    assert ma.microadam_attention_workspace(given(batch=0), True) == 0
    assert ma.microadam_attention_saved(given()) == 256
    kept = ma.microadam_attention_saved(given(dtype=BF16))
    assert kept == 256 + (B * H * SQ * D * 2 + 255) // 256 * 256
    for f in (forward, backward):
        refused(SIZE, f, given(), kept=255)
        refused(SIZE, f, given(dtype=BF16), kept=kept - 1)
    refused(INVALID, ma.microadam_attention_saved, given(causal=3))
    with pytest.raises(ma.MicroAdamError):
        ma._check(ma.load().microadam_attention_workspace(given(), 0, None), "microadam_attention_workspace")
    assert ma.load().microadam_attention_saved(given(), None) == INVALID
    assert ma.load().microadam_attention_forward(None, None, None, 0, None, 0, None) == INVALID
    assert ma.load().microadam_attention_forward(given(), None, None, 0, None, 0, None) == INVALID


def test_nothing_to_do():
    none = heads(None, SQ, H)
    for kw in (dict(batch=0), dict(queries=0)):
        forward(given(q=none, k=none, v=none, **kw), out=none, saved=None, kept=0, ws=None, size=0)
    backward(given(q=none, k=none, v=none, batch=0), none, None, 0, none, none, none, none, None, 0)


def test_workgroups():
    """A launch has fewer than 2^24 of them: the last size that passes, and the next."""
    for kw, most in ((dict(queries=1, keys=1), (1 << 23) - 1), (dict(queries=64, keys=1), (1 << 23) - 1),
                     (dict(queries=65, keys=1), (1 << 22) - 1), (dict(queries=1, keys=129), (1 << 22) - 1)):
        ma.microadam_attention_saved(given(batch=most, **kw))
        refused(UNSUPPORTED, ma.microadam_attention_saved, given(batch=most + 1, **kw))


def test_python():
    x = torch.ones(1, 2, 1, 8)
    with pytest.raises(ValueError):
        attention(x, x, x)
    with pytest.raises(TypeError):
        attention(x.half(), x.half(), x.half())
