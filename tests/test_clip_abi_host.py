"""Argument checks of the gradient norm and clipping entry points that need no
GPU: every refusal comes before any device work."""
import ctypes
import math
import os

import pytest
import torch

import paper_2405_15593_amd as ma
from paper_2405_15593_amd.clip import clip_grad_norm, clip_grads, grad_norm, workspace_bytes

F32, BF16 = ma.MICROADAM_F32, ma.MICROADAM_BF16
INVALID, UNSUPPORTED, SIZE = (ma.MICROADAM_ERR_INVALID_ARG, ma.MICROADAM_ERR_UNSUPPORTED,
                              ma.MICROADAM_ERR_STATE_SIZE)
WS = 1 << 20      # addresses that no refusal follows


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ma.LIBRARY):
        from paper_2405_15593_amd import _build
        _build.build()
    return ma.load()


def arrays(*entries):
    n = max(1, len(entries))
    return ((ctypes.c_void_p * n)(*[e[0] for e in entries]), (ctypes.c_int64 * n)(*[e[1] for e in entries]),
            (ctypes.c_int32 * n)(*[e[2] for e in entries]))


def both(code, *entries, n=None, norm=64, ws=WS, size=None, given=None, limit=1.0, eps=1e-6, only_clip=False):
    given = given if given is not None else arrays(*entries)
    n = len(entries) if n is None else n
    size = workspace_bytes() if size is None else size
    calls = [lambda: ma.microadam_clip_grads(*given, n, limit, eps, norm, ws, size)]
    if not only_clip:
        calls.append(lambda: ma.microadam_grad_norm(*given, n, norm, ws, size))
    for call in calls:
        with pytest.raises(ma.MicroAdamError) as e:
            call()
        assert e.value.code == code, e.value


@pytest.mark.parametrize("entry,code", [
    ((None, 4, F32), INVALID), ((4096, -1, F32), INVALID), ((4096, 4, 2), INVALID), ((4096, 4, -1), INVALID),
    ((4098, 4, F32), INVALID), ((4097, 4, BF16), INVALID), ((4097, 0, BF16), INVALID),
    ((4096, (1 << 40) + 1, BF16), UNSUPPORTED)], ids=str)
def test_entries(entry, code):
    both(code, entry)
    both(code, (65536, 4, F32), entry)


def test_lists_and_pointers():
    both(INVALID, (4096, 4, F32), n=-1)
    for i in range(3):
        given = list(arrays((4096, 4, F32)))
        given[i] = None
        both(INVALID, n=1, given=given)
    both(INVALID, (4096, 4, F32), norm=None)
    both(INVALID, (4096, 4, F32), norm=66)
    both(INVALID, (4096, 4, F32), ws=None)
    both(INVALID, (4096, 4, F32), ws=WS + 4)
    both(SIZE, (4096, 4, F32), size=workspace_bytes() - 1)
    both(SIZE, size=0)


@pytest.mark.parametrize("kw", [dict(limit=-1.0), dict(limit=math.nan), dict(eps=-1e-9), dict(eps=math.nan),
                                dict(eps=math.inf)], ids=str)
def test_limits(kw):
    both(INVALID, (4096, 4, F32), only_clip=True, **kw)


@pytest.mark.parametrize("entries", [
    [(4096, 4, F32), (4096, 4, F32)], [(4096, 4, F32), (4108, 1, F32)], [(4108, 1, F32), (4096, 4, F32)],
    [(4096, 8, BF16), (4110, 1, BF16)], [(4096, 100, F32), (8192, 4, F32), (4400, 1, BF16)],
    [(WS + 8, 1, F32)], [(WS - 4, 2, F32)], [(60, 2, F32)], [(64, 1, BF16)]], ids=str)
def test_overlaps(entries):
    both(INVALID, *entries, only_clip=True)


def test_python():
    x = torch.ones(3)
    for f in (lambda g: grad_norm(g), lambda g: clip_grads(g, 1.0)):
        for bad in ([], [x]):
            with pytest.raises(ValueError):
                f(bad)
    p = torch.nn.Parameter(x)
    assert float(clip_grad_norm([p], 1.0)) == 0.0 and float(clip_grad_norm([], 1.0)) == 0.0
    assert workspace_bytes() % 8 == 0
    with pytest.raises(ma.MicroAdamError):
        ma._check(ma.load().microadam_clip_workspace(None), "microadam_clip_workspace")
