"""What may share memory in a list of matrices and what is refused: decided on
the host from addresses, shapes and strides, before any device work.  A list
that passes comes to the next refusal, that of the missing workspace."""
import ctypes

import pytest

import paper_2405_15593_amd as ma

F32, BF16 = ma.MICROADAM_F32, ma.MICROADAM_BF16
AT = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(ma.LIBRARY):
        from paper_2405_15593_amd import _build
        _build.build()
    return ma.load()


def matrix(grad, out, momentum=None, rows=8, cols=16, grad_ld=None, out_ld=None, momentum_ld=None):
    return (grad, momentum, out, rows, cols, grad_ld or cols, momentum_ld or cols if momentum else 0, out_ld or cols)


def answer(rows, grad=F32, momentum=None, out=F32):
    """The refusal's message; with `momentum` (a dtype) muon_step's."""
    mats = (ma.microadam_matrix * len(rows))(*rows)
    with pytest.raises(ma.MicroAdamError) as e:
        if momentum is None:
            ma.microadam_orthogonalize(ma.make_schulz_config(), mats, len(rows), grad, out, None, 1 << 30)
        else:
            cfg = ma.microadam_muon_config(ma.make_schulz_config(), 0.9, 0.0, 1, 0)
            ma.microadam_muon_step(cfg, mats, len(rows), grad, momentum, out, 0.1, None, 1 << 30)
    assert e.value.code == ma.MICROADAM_ERR_INVALID_ARG
    return str(e.value)


def refused(*a, **kw):
    return "overlap" in answer(*a, **kw)


def passes(*a, **kw):
    return "workspace is NULL" in answer(*a, **kw)


FAR = 1 << 30   # grads, out of the way


@pytest.mark.parametrize("out,size", [(F32, 4), (BF16, 2)])
def test_outputs_that_meet(out, size):
    """Two outputs of 8 x 16, rows 40 apart."""
    def pair(off, **kw):
        return [matrix(FAR, AT, out_ld=40), matrix(FAR, AT + off * size, **{"out_ld": 40, **kw})]

    reach = 7 * 40 + 16
    for off in (1, 15, 25, 39, 40, 55, reach - 1, -1, -15, -25, -40, -(reach - 1)):
        assert refused(pair(off), out=out), off
    for off in (16, 24, 56, 64, 16 + 6 * 40, reach, -16, -24, -56, -reach, 7 * 40 + 16, 8 * 40, 9 * 40):
        assert passes(pair(off), out=out), off
    # other strides: 80 apart lies in every second row's gap or on a row
    assert passes(pair(16, out_ld=80), out=out) and passes(pair(24 + 40, out_ld=80), out=out)
    assert refused(pair(15, out_ld=80), out=out) and refused(pair(40, out_ld=80), out=out)
    # 41 apart: row i starts at 20 + i of row i's 40, and meets the next row from i = 5 on
    assert passes(pair(20, out_ld=41, rows=5), out=out) and refused(pair(20, out_ld=41, rows=6), out=out)
    assert passes(pair(16, out_ld=41), out=out)
    # one long row against rows
    assert refused(pair(16, rows=1, cols=25, out_ld=25), out=out) and passes(pair(16, rows=1, cols=24, out_ld=24), out=out)
    # dense, side by side and one element into each other
    dense = [matrix(FAR, AT), matrix(FAR, AT + 128 * size)]
    assert passes(dense, out=out)
    assert refused([dense[0], matrix(FAR, AT + 127 * size)], out=out)


def test_many_outputs():
    """Columns of one buffer, a hundred matrices; one moved into its neighbour."""
    cols = [matrix(FAR, AT + i * 64, rows=50, out_ld=1600) for i in range(100)]
    assert passes(cols)
    for i in (0, 57, 99):
        bad = list(cols)
        bad[i] = matrix(FAR, cols[i][2] + (4 if i < 99 else -4), rows=50, out_ld=1600)
        assert refused(bad), i
        assert refused(bad[::-1]), i
    # a large one around small ones
    assert refused([matrix(FAR, AT, rows=1000, cols=1000)] + [matrix(FAR, AT - 8192 + i * 4096) for i in range(40)])


def test_an_output_and_the_grads():
    own = matrix(AT, AT)
    assert passes([own]) and passes([own, matrix(AT + 4096, AT + 4096)])       # each in its own grad's place
    assert passes([matrix(AT, AT + 64)])                                        # ... or partly: it has been read by then
    assert passes([matrix(AT, AT, out_ld=16)], grad=F32, out=BF16)
    # in another's: right or wrong by the batch that the workspace allows
    assert refused([matrix(AT, AT + 4096), matrix(AT + 4096, AT + 8192)])
    assert refused([matrix(AT, AT + 8192), matrix(AT + 4096, AT + 4)])
    assert refused([matrix(AT, AT), matrix(AT, AT + 4096)])                     # one grad twice, one output in it
    assert passes([matrix(AT, AT + 8192), matrix(AT, AT + 4096)])               # one grad twice
    # the grad's element size counts: 8 x 16 bfloat16 end at 256 bytes
    assert passes([matrix(AT, AT + 8192), matrix(AT + 4096, AT + 256)], grad=BF16)
    assert refused([matrix(AT, AT + 8192), matrix(AT + 4096, AT + 254)], grad=BF16, out=BF16)


@pytest.mark.parametrize("momentum,size", [(F32, 4), (BF16, 2)])
def test_momenta(momentum, size):
    kw = dict(momentum=momentum)
    fine = matrix(AT, AT + 4096, AT + 8192)
    assert passes([fine], **kw)
    assert refused([matrix(AT, AT + 4096, AT + 4096)], **kw)                    # the parameter itself
    assert refused([matrix(AT, AT + 4096, AT)], **kw)                           # its gradient
    assert refused([matrix(AT, AT + 4096, AT + 4096 - 128 * size + size * 2)], **kw)
    assert passes([matrix(AT, AT + 4096, AT + 4096 - 128 * size)], **kw)
    other = dict(grad=AT + 16384, out=AT + 20480, momentum=AT + 24576)
    assert passes([fine, matrix(**other)], **kw)
    for name, at in (("momentum", AT), ("momentum", AT + 4096), ("momentum", AT + 8192 + 64), ("out", AT),
                     ("out", AT + 4096 + 64), ("out", AT + 8192), ("grad", AT + 8192), ("grad", AT + 4096)):
        pair = [fine, matrix(**{**other, name: at})]
        assert refused(pair, **kw) and refused(pair[::-1], **kw), (name, at)
    # parameter, gradient and momentum as columns of one buffer
    one = [matrix(AT + i * 256, AT + i * 256 + 64, AT + i * 256 + 128, grad_ld=640, out_ld=640,
                  momentum_ld=640 if momentum == F32 else 1280) for i in range(10)]
    assert passes(one, **kw)


def test_against_every_element():
    """Small layouts, each against the sets of bytes that they take."""
    import random
    rng = random.Random(5)
    seen = [0, 0]

    def elements(at, rows, cols, ld):
        return {at + 4 * (r * ld + c) for r in range(rows) for c in range(cols)}

    for _ in range(3000):
        one = [rng.randint(1, 6), rng.randint(1, 9)]
        two = [rng.randint(1, 6), rng.randint(1, 9)]
        ld1, ld2 = one[1] + rng.randint(0, 12), two[1] + rng.randint(0, 12)
        if rng.random() < 0.4:
            ld2 = max(ld2, ld1)
            ld1 = max(ld1, ld2)
        off = 4 * rng.randint(-60, 60)
        meet = bool(elements(AT, *one, ld1) & elements(AT + off, *two, ld2))
        pair = [matrix(FAR, AT, rows=one[0], cols=one[1], out_ld=ld1),
                matrix(FAR, AT + off, rows=two[0], cols=two[1], out_ld=ld2)]
        assert refused(pair) == meet, (one, two, ld1, ld2, off)
        seen[meet] += 1
    assert min(seen) > 500


def test_size_comes_first():
    lib = ma.load()
    mats = (ma.microadam_matrix * 2)(matrix(FAR, AT), matrix(FAR, AT))
    rc = lib.microadam_orthogonalize(ctypes.byref(ma.make_schulz_config()), mats, 2, F32, F32, None, 0, None)
    assert rc == ma.MICROADAM_ERR_STATE_SIZE
