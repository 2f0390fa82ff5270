"""What the inputs of attention_needles.py notice, on the CPU: mistakes planted in a
plain attention in binary64, whose result is rounded to the dtype."""
import pytest
import torch

from attention_needles import check_even, check_needles, ends, even, even_wanted, limits, needles

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
KEYS, DIM, HEADS, KV = 132000, 128, 2, 1


def plain(q, k, v, scale, n, dtype, lost=(), values_of=None, twice=()):
    """One sequence and query; `lost` keys are left out, `twice` taken twice, and
    `values_of` (a, b): the values of the 32 keys from b on for those from a on."""
    k, v = k[0].double(), v[0].double()
    if values_of:
        v = v.clone()
        v[values_of[0]:values_of[0] + 32] = v[values_of[1]:values_of[1] + 32].clone()
    weight = torch.ones(k.shape[0], dtype=torch.float64)
    weight[int(n[0, 0]):] = 0.0
    weight[list(lost)] = 0.0
    weight[list(twice)] *= 2.0
    out = []
    for h in range(q.shape[2]):
        z = k[:, h // (q.shape[2] // k.shape[1])] @ q[0, 0, h].double() * scale
        p = weight * torch.exp(z - z.max())
        out.append(p @ v[:, h // (q.shape[2] // k.shape[1])] / p.sum())
    return torch.stack(out)[None, None].to(dtype)


FAULTS = {"first": dict(lost=range(32)), "last": dict(lost=range(KEYS - 32, KEYS)), "tile": dict(lost=range(32 * 1700, 32 * 1701)),
          "part": dict(lost=range(KEYS // 128, KEYS // 64)), "half": dict(lost=range(16500)), "again": dict(twice=range(64, 96))}


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("length", [KEYS, 66001, 33])
def test_even(types, length):
    dtype = TYPES[types]
    n = limits(1, 1, KEYS, False, torch.tensor([length]))
    q, k, v, place = even(1, 1, KEYS, HEADS, KV, DIM, dtype, "cpu")
    check_even(plain(q, k, v, 0.125, n, dtype), place, n)
    with pytest.raises(AssertionError):
        check_even(torch.zeros_like(q), place, n)
    for fault in FAULTS.values():
        if min(fault.get("lost", fault.get("twice"))) + 32 > length:
            continue
        if length == 33:      # one key is left
            continue
        with pytest.raises(AssertionError):
            check_even(plain(q, k, v, 0.125, n, dtype, **fault), place, n)


@pytest.mark.parametrize("types", TYPES)
def test_needles(types):
    dtype, scale = TYPES[types], DIM ** -0.5
    n = limits(1, 1, KEYS, False, None)
    q, k, v, at, score = needles(1, 1, KEYS, HEADS, KV, DIM, dtype, "cpu", scale)
    check_needles(plain(q, k, v, scale, n, dtype), at, score, n, KV, DIM)
    with pytest.raises(AssertionError):
        check_needles(torch.zeros_like(q), at, score, n, KV, DIM)
    for fault in (dict(lost=[KEYS - 1]), dict(lost=[0]), dict(lost=[31]), dict(values_of=(0, 32)), dict(values_of=(32, 0)),
                  dict(values_of=(KEYS - 64, KEYS - 32)), dict(values_of=(KEYS - 32, KEYS - 64))):
        with pytest.raises(AssertionError):
            check_needles(plain(q, k, v, scale, n, dtype, **fault), at, score, n, KV, DIM)


def test_ends():
    for keys in (1, 33, 700, 9001, KEYS):
        for dim in (8, 64, 128):
            at = ends(keys, dim)
            assert len(at) <= dim and len(set(at)) == len(at) and all(0 <= x < keys for x in at)
    assert {0, 31, 32, KEYS - 1, KEYS - 32, KEYS - 33} <= set(ends(KEYS, 128))


def test_even_is_a_share():
    n = limits(2, 3, 50, True, torch.tensor([50, 7]))
    assert n.tolist() == [[48, 49, 50], [7, 7, 7]]
    place = even(2, 3, 50, 4, 2, 8, torch.float32, "cpu")[3]
    want = even_wanted(place, n, 4, 8)
    assert torch.allclose(want.sum(3), torch.ones(2, 3, 4, dtype=torch.float64))
