"""Argument checks of the layer norm entry points that need no GPU: every
refusal comes before any device work."""
import math
import os

import pytest
import torch

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.norm import layer_norm

F32, BF16 = ma.MICROADAM_F32, ma.MICROADAM_BF16
INVALID, UNSUPPORTED, SIZE = (ma.MICROADAM_ERR_INVALID_ARG, ma.MICROADAM_ERR_UNSUPPORTED,
                              ma.MICROADAM_ERR_STATE_SIZE)
# addresses that no refusal follows, a mebibyte apart
X, W, B, Y, MEAN, RSTD, DY, DX, DW, DB, WS = ((i + 1) << 20 for i in range(11))


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ma.LIBRARY):
        from paper_2405_15593_amd import _build
        _build.build()
    return ma.load()


def rows(**kw):
    r = dict(x=X, weight=W, bias=B, rows=8, cols=16, ld=16, eps=1e-5, dtype=F32, weight_dtype=F32)
    r.update(kw)
    return ma.microadam_rows(*r.values())


def forward(r, y=Y, y_ld=16, mean=MEAN, rstd=RSTD):
    ma.microadam_layer_norm(r, y, y_ld, mean, rstd)


def backward(r, mean=MEAN, rstd=RSTD, dy=DY, dy_ld=16, dx=DX, dx_ld=16, dw=DW, db=DB, ws=WS, size=1 << 19):
    ma.microadam_layer_norm_grad(r, mean, rstd, dy, dy_ld, dx, dx_ld, dw, db, ws, size)


def refused(code, f, *args, **kw):
    with pytest.raises(ma.MicroAdamError) as e:
        f(*args, **kw)
    assert e.value.code == code, e.value


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), INVALID), (dict(x=X + 2), INVALID), (dict(weight=W + 2), INVALID), (dict(bias=B + 1), INVALID),
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(cols=-4), INVALID), (dict(ld=15), INVALID),
    (dict(dtype=2), INVALID), (dict(weight_dtype=-1), INVALID), (dict(eps=-1e-9), INVALID),
    (dict(eps=math.nan), INVALID), (dict(eps=1e39), INVALID), (dict(cols=(1 << 24) + 1, ld=1 << 25), UNSUPPORTED),
    (dict(rows=(1 << 31) + 1), UNSUPPORTED), (dict(ld=(1 << 40) + 1), UNSUPPORTED)], ids=str)
def test_rows(kw, code):
    refused(code, forward, rows(**kw))
    refused(code, backward, rows(**kw))


def test_reach():
    """A matrix ends within 2^60 elements: what lies where is known in 64 bits."""
    far = dict(rows=1 << 30, cols=16)
    for f in (forward, backward):
        refused(UNSUPPORTED, f, rows(ld=(1 << 30) + 1, **far))
    refused(UNSUPPORTED, forward, rows(**far), y_ld=1 << 40)
    refused(UNSUPPORTED, backward, rows(**far), dy_ld=1 << 31)
    refused(UNSUPPORTED, backward, rows(**far), dx_ld=1 << 31)
    refused(INVALID, forward, rows(ld=1 << 30, **far))     # (the reach is allowed: y lies in x)


@pytest.mark.parametrize("kw,code", [
    (dict(y=None), INVALID), (dict(y=Y + 2), INVALID), (dict(y_ld=15), INVALID), (dict(mean=None), INVALID),
    (dict(rstd=None), INVALID), (dict(mean=MEAN + 1), INVALID), (dict(y_ld=1 << 41), UNSUPPORTED),
    (dict(y=X), INVALID), (dict(y=X + 8 * 16 * 4 - 4), INVALID), (dict(y=W + 60), INVALID), (dict(mean=X + 4), INVALID),
    (dict(rstd=MEAN + 28), INVALID), (dict(mean=Y + 508), INVALID)], ids=str)
def test_forward(kw, code):
    refused(code, forward, rows(), **kw)


@pytest.mark.parametrize("kw,code", [
    (dict(mean=None), INVALID), (dict(rstd=None), INVALID), (dict(dy=None), INVALID), (dict(dy=DY + 2), INVALID),
    (dict(dy_ld=15), INVALID), (dict(dx_ld=15), INVALID), (dict(dx=DX + 2), INVALID), (dict(dw=DW + 2), INVALID),
    (dict(db=DB + 1), INVALID), (dict(ws=None), INVALID), (dict(ws=WS + 8), INVALID), (dict(size=0), SIZE),
    (dict(dx=X), INVALID), (dict(dx=DY), INVALID), (dict(dx=DY + 4 * 10000), INVALID), (dict(dw=W), INVALID),
    (dict(db=DW + 32), INVALID), (dict(ws=X), INVALID), (dict(dw=RSTD), INVALID)], ids=str)
def test_backward(kw, code):
    refused(code, backward, rows(rows=1000), **kw)


def test_workspace():
    need = ma.microadam_layer_norm_workspace(rows(rows=1000))
    assert need > 0 and need % 8 == 0
    refused(SIZE, backward, rows(rows=1000), size=need - 1)
    assert ma.microadam_layer_norm_workspace(rows()) == 0      # one workgroup
    assert ma.microadam_layer_norm_workspace(rows(x=None, rows=0)) == 0
    # one partial sum a workgroup, however many rows
    most = ma.microadam_layer_norm_workspace(rows(rows=1 << 31, cols=4096, ld=4096))
    assert 0 < most <= 2048 * 2 * 4096 * 4
    refused(INVALID, ma.microadam_layer_norm_workspace, rows(cols=0))
    with pytest.raises(ma.MicroAdamError):
        ma._check(ma.load().microadam_layer_norm_workspace(rows(), None), "microadam_layer_norm_workspace")
    assert ma.load().microadam_layer_norm(None, None, 0, None, None, None) == INVALID
    assert ma.load().microadam_layer_norm_grad(None, *[None] * 3, 0, None, 0, *[None] * 3, 0, None) == INVALID


def test_nothing_to_do():
    """Without rows nothing is read or written."""
    forward(rows(x=None, rows=0), y=None, mean=None, rstd=None)
    backward(rows(x=None, rows=0), mean=None, rstd=None, dy=None, dx=None, dw=None, db=None, ws=None, size=0)


def test_python():
    x = torch.ones(2, 4)
    for bad in (x, x.to(torch.float16), x.double()):
        with pytest.raises((ValueError, TypeError)):
            layer_norm(bad)


def test_the_tensor_side_is_not_built(monkeypatch, tmp_path):
    monkeypatch.setattr(ma, "_torch_side", None)
    monkeypatch.setattr(ma, "_PKG", str(tmp_path))
    with pytest.raises(RuntimeError, match="not built"):
        layer_norm(torch.ones(2, 3))
