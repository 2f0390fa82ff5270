"""Argument checks of the loss and matrix-update entry points that need no
GPU: every refusal comes before any device work."""
import ctypes
import math

import pytest
import torch

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.muon import Muon, workspace_bytes

F32, BF16 = ma.MICROADAM_F32, ma.MICROADAM_BF16
INVALID, UNSUPPORTED, SIZE = (ma.MICROADAM_ERR_INVALID_ARG, ma.MICROADAM_ERR_UNSUPPORTED,
                              ma.MICROADAM_ERR_STATE_SIZE)


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(ma.LIBRARY):
        from paper_2405_15593_amd import _build
        _build.build()
    return ma.load()


def matrices(*rows):
    return (ma.microadam_matrix * max(1, len(rows)))(*rows)


def good(**kw):
    m = dict(grad=4096, momentum=None, out=8192, rows=8, cols=16, grad_ld=16, momentum_ld=0, out_ld=16)
    m.update(kw)
    return matrices(tuple(m.values()))


def refused(code, f, *args):
    with pytest.raises(ma.MicroAdamError) as e:
        f(*args)
    assert e.value.code == code, e.value


def orth(cfg, mats, n=1, gd=F32, od=F32, ws=256, size=1 << 30):
    ma.microadam_orthogonalize(cfg, mats, n, gd, od, ws, size)


@pytest.mark.parametrize("kw", [dict(steps=0), dict(steps=17), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.inf),
                                dict(eps=math.nan), dict(precision=3), dict(precision=-1),
                                dict(coefficients=(1.0, math.nan, 0.0)), dict(coefficients=(math.inf, 0.0, 0.0))],
                         ids=str)
def test_schulz_config(kw):
    cfg = ma.make_schulz_config(**kw)
    refused(INVALID, orth, cfg, good())
    refused(INVALID, ma.microadam_matrix_workspace, cfg, good(), 1, F32)


def test_coefficient_lists():
    for bad in ((1.0, 2.0), ((1, 2, 3), (1, 2, 3)), ()):
        with pytest.raises(ValueError):
            ma.make_schulz_config(steps=5, coefficients=bad)
    cfg = ma.make_schulz_config(steps=2, coefficients=((1, 2, 3), (4, 5, 6)))
    assert [cfg.coefficients[i] for i in range(6)] == [1, 2, 3, 4, 5, 6]
    assert [ma.make_schulz_config(steps=2, coefficients=(1, 2, 3)).coefficients[i] for i in range(6)] == [1, 2, 3] * 2


@pytest.mark.parametrize("kw,code", [
    (dict(grad=None), INVALID), (dict(out=None), INVALID), (dict(grad=4098), INVALID), (dict(out=8193), INVALID),
    (dict(rows=0), INVALID), (dict(cols=-1), INVALID), (dict(grad_ld=15), INVALID), (dict(out_ld=0), INVALID),
    (dict(momentum=512), INVALID), (dict(rows=1 << 21), UNSUPPORTED), (dict(grad_ld=1 << 31), UNSUPPORTED),
    (dict(rows=1 << 20, cols=1 << 20, grad_ld=1 << 20, out_ld=1 << 20), UNSUPPORTED)], ids=str)
def test_matrix(kw, code):
    refused(code, orth, ma.make_schulz_config(), good(**kw))


def test_lists_types_and_workspace():
    cfg = ma.make_schulz_config()
    refused(INVALID, orth, cfg, good(), 0)
    refused(INVALID, orth, cfg, None, 1)
    refused(INVALID, orth, cfg, good(), 1, 2, F32)
    refused(INVALID, orth, cfg, good(), 1, F32, -1)
    refused(INVALID, orth, cfg, good(), 1, F32, F32, 0)
    refused(INVALID, orth, cfg, good(), 1, F32, F32, 128)
    least, useful = ma.microadam_matrix_workspace(cfg, good(), 1, F32)
    refused(SIZE, orth, cfg, good(), 1, F32, F32, 256, least - 1)
    # 8 x 16 works as 64 x 64: X transposed twice, A and B, two planes each
    assert least == useful == 96 * 256 * 8 + 4 * 64 * 64 * 2 * 2
    assert ma.microadam_matrix_workspace(cfg, good(), 1, BF16)[0] == 96 * 256 * 8 + 4 * 64 * 64 * 2
    # the second of two is the one that does not fit
    two = matrices((4096, None, 8192, 8, 16, 16, 0, 16), (4096, None, 8192, 600, 900, 900, 0, 900))
    refused(SIZE, orth, cfg, two, 2, F32, F32, 256, least)


def test_workspace_is_bounded():
    shapes = [(4096, 4096)] * 128
    least, useful = workspace_bytes(shapes)
    one = (2 * 4096 * 4096 + 2 * 4096 * 4096) * 2
    assert one < least < one + (1 << 20)
    assert (2 << 30) <= useful < (2 << 30) + (1 << 20)
    big = workspace_bytes([(32000, 32000)])
    assert big[0] == big[1]


def muon(cfg, mats, lr=0.1, dtypes=(F32, F32, F32), ws=256, size=1 << 30):
    ma.microadam_muon_step(cfg, mats, 1, *dtypes, lr, ws, size)


def muon_config(**kw):
    c = dict(schulz=ma.make_schulz_config(), momentum=0.9, weight_decay=0.0, nesterov=1, scale=0)
    c.update(kw)
    return ma.microadam_muon_config(*c.values())


@pytest.mark.parametrize("kw", [dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=math.nan),
                                dict(weight_decay=-1.0), dict(weight_decay=math.inf), dict(nesterov=2), dict(scale=3),
                                dict(schulz=ma.make_schulz_config(steps=0))], ids=lambda k: str(list(k.items())[0][:1]))
def test_muon_config(kw):
    refused(INVALID, muon, muon_config(**kw), good(momentum=512, momentum_ld=16))


def test_muon_arguments():
    cfg = muon_config()
    refused(INVALID, muon, cfg, good())                                   # no momentum
    refused(INVALID, muon, cfg, good(momentum=512, momentum_ld=3))
    refused(INVALID, muon, cfg, good(momentum=512, momentum_ld=16), math.nan)
    refused(INVALID, muon, cfg, good(momentum=512, momentum_ld=16), 0.1, (F32, 5, F32))
    refused(SIZE, muon, cfg, good(momentum=512, momentum_ld=16), 0.1, (F32, F32, F32), 256, 0)


@pytest.mark.parametrize("kw", [dict(lr=-1.0), dict(momentum=1.0), dict(weight_decay=-0.1), dict(eps=0.0),
                                dict(steps=0), dict(scale="rms"), dict(precision="f64"),
                                dict(momentum_dtype=torch.float16), dict(coefficients=(1, 2))], ids=str)
def test_muon_optimizer_settings(kw):
    with pytest.raises(ValueError):
        Muon([torch.nn.Parameter(torch.zeros(4, 4))], **kw)


def test_muon_takes_matrices_only():
    with pytest.raises(ValueError):
        Muon([torch.nn.Parameter(torch.zeros(4))])


def logits(**kw):
    c = dict(data=4096, targets=8192, rows=4, vocab=100, ld=100, ignore_index=-100, temperature=1.0, dtype=F32,
             reserved=0)
    c.update(kw)
    return ma.microadam_logits(*c.values())


LOGITS = [(dict(data=0), INVALID), (dict(targets=0), INVALID), (dict(data=4097), INVALID),
          (dict(targets=8196), INVALID), (dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(ld=99), INVALID),
          (dict(temperature=0.0), INVALID), (dict(temperature=math.nan), INVALID),
          (dict(temperature=1e-60), INVALID), (dict(temperature=1e60), INVALID), (dict(dtype=2), INVALID),
          (dict(reserved=1), INVALID), (dict(vocab=(1 << 24) + 1, ld=1 << 25), UNSUPPORTED),
          (dict(rows=(1 << 20) + 1), UNSUPPORTED), (dict(ld=1 << 41), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", LOGITS, ids=[str(k) for k, _ in LOGITS])
def test_logits(kw, code):
    refused(code, ma.microadam_token_logprobs, logits(**kw), 0, 256, 256, None, None)
    refused(code, ma.microadam_token_logprobs_grad, logits(**kw), 256, None, 256, 256, 65536, 1 << 26)


def test_logprob_arguments():
    f = ma.microadam_token_logprobs
    refused(INVALID, f, logits(), -1, 256, 256, 256, 256)
    refused(INVALID, f, logits(), 101, 256, 256, 256, 256)
    refused(UNSUPPORTED, f, logits(), 65, 256, 256, 256, 256)
    refused(INVALID, f, logits(), 5, 256, 256, None, 256)
    refused(INVALID, f, logits(), 5, 256, 256, 256, None)
    refused(INVALID, f, logits(), 5, 258, 256, 256, 256)
    refused(INVALID, f, logits(), 5, 256, 256, 256, 260)
    g = ma.microadam_token_logprobs_grad
    refused(INVALID, g, logits(), None, None, 256, 256, 65536, 100)
    refused(INVALID, g, logits(), 256, None, 256, 256, None, 100)
    refused(INVALID, g, logits(), 256, None, 256, 256, 65536, 99)
    refused(INVALID, g, logits(), 256, None, 256, 256, 65538, 100)
    refused(INVALID, g, logits(), 256, None, 256, 256, 4096, 104)     # in place, another stride
    f(logits(rows=0, data=0, targets=0), 3, None, None, None, None)   # nothing to do


@pytest.mark.parametrize("dtype,size", [(F32, 4), (BF16, 2)])
def test_gradient_that_overlaps_the_logits(dtype, size):
    """Rows of 100 at a stride of 256: a gradient that starts in a row, or ends
    in one, is refused; between the rows, behind them or in place is not (no
    target address: those come to the next refusal, by its own message)."""
    g = ma.microadam_token_logprobs_grad
    at = 1 << 20
    x = logits(data=at, ld=256, dtype=dtype)
    ends = 3 * 256 + 100  # of the four rows
    for off in (1, 99, 157, 255, 256, 355, 413, -1, -99, -157, -256, ends - 1, -(ends - 1)):
        with pytest.raises(ma.MicroAdamError, match="overlaps"):
            g(x, 256, None, 256, 256, at + off * size, 256)
    for off in (1, 100, ends - 1, -1, -(3 * 300 + 99)):  # another stride, ranges that meet
        with pytest.raises(ma.MicroAdamError, match="overlaps"):
            g(x, 256, None, 256, 256, at + off * size, 300)
    one = logits(data=at, rows=1, ld=100, dtype=dtype)
    for off in (1, 99, -1, -99):
        with pytest.raises(ma.MicroAdamError, match="overlaps"):
            g(one, 256, None, 256, 256, at + off * size, 100)
    # these pass the overlap check and are refused for logp's alignment
    for off, ld in ((100, 256), (156, 256), (356, 256), (-100, 256), (-156, 256), (ends, 300), (0, 256),
                    (-(3 * 300 + 100), 300)):
        with pytest.raises(ma.MicroAdamError, match="an argument is not aligned"):
            g(x, 256, None, 257, 256, at + off * size, ld)


@pytest.mark.parametrize("kw,code", [(dict(group_rows=3, group_stride=400), INVALID),
                                     (dict(group_rows=-2, group_stride=400), INVALID),
                                     (dict(group_rows=2, group_stride=-1), INVALID),
                                     (dict(group_rows=0, group_stride=400), INVALID),
                                     (dict(group_rows=2, group_stride=1 << 41), UNSUPPORTED)], ids=str)
def test_groups_of_rows(kw, code):
    refused(code, ma.microadam_token_logprobs, logits(**kw), 0, 256, 256, None, None)
    refused(code, ma.microadam_token_logprobs_grad, logits(**kw), 256, None, 256, 256, 65536, 1 << 26)


def test_a_gradient_among_groups():
    """Rows in groups: no gradient in place, nor where the groups reach."""
    g = ma.microadam_token_logprobs_grad
    at = 1 << 20
    x = logits(data=at, group_rows=2, group_stride=300)
    refused(INVALID, g, x, 256, None, 256, 256, at, 100)
    for off in (1, 250, 499, -1, -399):
        with pytest.raises(ma.MicroAdamError, match="overlaps"):
            g(x, 256, None, 256, 256, at + off * 4, 100)
    for off in (500, -400):
        with pytest.raises(ma.MicroAdamError, match="an argument is not aligned"):
            g(x, 256, None, 257, 256, at + off * 4, 100)


def test_a_matrix_twice():
    a = dict(grad=4096, momentum=None, out=8192, rows=8, cols=16, grad_ld=16, momentum_ld=0, out_ld=16)
    twice = matrices(tuple(a.values()), tuple(dict(a, grad=1 << 16).values()))
    refused(INVALID, orth, ma.make_schulz_config(), twice, 2)
    m = dict(a, momentum=1 << 17, momentum_ld=16)
    for other in (dict(m, momentum=1 << 18), dict(m, out=1 << 18)):
        refused(INVALID, ma.microadam_muon_step, muon_config(), matrices(tuple(m.values()), tuple(other.values())), 2,
                F32, F32, F32, 0.1, 256, 1 << 30)


def test_null_pointers():
    lib = ma.load()
    assert lib.microadam_orthogonalize(None, good(), 1, F32, F32, None, 0, None) == INVALID
    assert lib.microadam_muon_step(None, good(), 1, F32, F32, F32, 0.1, None, 0, None) == INVALID
    assert lib.microadam_matrix_workspace(ctypes.byref(ma.make_schulz_config()), good(), 1, F32, None, None) == INVALID
    assert lib.microadam_token_logprobs(None, 0, None, None, None, None, None) == INVALID
    assert lib.microadam_token_logprobs_grad(None, None, None, None, None, None, 0, None) == INVALID
