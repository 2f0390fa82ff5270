"""Attention inputs in which every key counts, for calls over many keys, where a
worst-case tolerance of the scores' and chains' roundings would hide a lost tile.

`even`: q is zero, so that every key that a query sees has the probability 1 / n, and
the values are one-hot by the key's place: element e of an output is the share of the
seen keys whose place has e.  Sums of ones are exact in binary32 up to 2^24 and a p of
one is exact in bfloat16, so that outputs are off by two roundings of binary32 and their
own.  Places go by runs of keys, so that a lost, repeated or misread run of a hundredth
of a share shows.

`needles`: a few dozen keys, at the ends of tiles and of parts among others, share
all but a hundredth of the probability in equal parts, and each has its value in an
element of its own: a value taken from a neighbour, or a needle lost, changes its
element by its whole size.
"""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def limits(batch, queries, keys, causal, lengths):
    """How many of the first keys each sequence's queries see."""
    n = torch.full((batch,), keys) if lengths is None else lengths.cpu().long().clamp(0, keys)
    last = torch.arange(queries) + 1 + keys - queries if causal else torch.full((queries,), keys)
    return torch.minimum(n[:, None], last.clamp(min=0)[None])


def even(batch, queries, keys, heads, kv_heads, dim, dtype, device):
    """(q, k, v, the place of each key of each key head)."""
    g = torch.Generator().manual_seed(keys)
    q = torch.zeros(batch, queries, heads, dim, dtype=dtype, device=device)
    k = torch.randn(1, keys, kv_heads, dim, generator=g).to(device).to(dtype).expand(batch, -1, -1, -1).contiguous()
    # a head's runs begin elsewhere than another's
    place = torch.arange(keys)[:, None] * dim // keys + torch.arange(kv_heads)[None]
    place = (place % dim).to(device)
    v = torch.nn.functional.one_hot(place, dim).to(dtype)[None].expand(batch, -1, -1, -1).contiguous()
    return q, k, v, place.cpu()


def even_wanted(place, n, heads, dim):
    """The outputs in binary64."""
    group = heads // place.shape[1]
    out = torch.zeros(*n.shape, heads, dim, dtype=torch.float64)
    for b in range(n.shape[0]):
        for i in range(n.shape[1]):
            seen = int(n[b, i])
            if not seen:
                continue
            for h in range(heads):
                out[b, i, h] = torch.bincount(place[:seen, h // group], minlength=dim).double() / seen
    return out


def check_even(got, place, n):
    want = even_wanted(place, n, got.shape[2], got.shape[3])
    off = (got.cpu().double() - want).abs()
    # 1 / n and the product with it, and the rounding to the dtype
    allowed = want * (4 * U + HALF[got.dtype] * 1.01)
    assert bool((off <= allowed).all()), float((off - allowed).max())


def ends(keys, dim):
    """Up to `dim` keys: at the ends of tiles, of halves and quarters and so on, and in between."""
    some = [0, 1, 31, 32, 63, 64, 127, 128, keys - 1, keys - 2, keys - 31, keys - 32, keys - 33, keys - 64]
    for parts in (2, 3, 4, 8, 16, 64, 128, 256):
        some += [keys // parts // 32 * 32 + d for d in (-1, 0)] + [keys * (parts - 1) // parts]
    step = keys // dim * 3 // 2 + 1
    some += list(range(17, keys, step))
    return list(dict.fromkeys(x for x in some if 0 <= x < keys))[:dim]


def needles(batch, queries, keys, heads, kv_heads, dim, dtype, device, scale):
    """(q, k, v, the needles, their score)."""
    at = torch.tensor(ends(keys, dim))
    score = math.log(100.0 * keys / len(at))
    q = torch.zeros(batch, queries, heads, dim, dtype=dtype, device=device)
    k = torch.zeros(batch, keys, kv_heads, dim, dtype=dtype, device=device)
    v = torch.zeros(batch, keys, kv_heads, dim, dtype=dtype, device=device)
    q[..., 0] = 1.0
    k[:, at.to(device), :, 0] = score / scale
    score = float(k[0, at[0], 0, 0].double()) * scale      # as the dtype holds it
    for j in range(kv_heads):
        v[:, at.to(device), j, (torch.arange(len(at)) + j) % dim] = 1.0
    return q, k, v, at, score


def needles_wanted(at, score, n, heads, kv_heads, dim):
    out = torch.zeros(*n.shape, heads, dim, dtype=torch.float64)
    weight = math.exp(score)
    for b in range(n.shape[0]):
        for i in range(n.shape[1]):
            seen = at < n[b, i]
            if not int(n[b, i]):
                continue
            total = float(seen.sum()) * weight + float(n[b, i] - seen.sum())
            for h in range(heads):
                out[b, i, h, (torch.arange(len(at)) + h // (heads // kv_heads)) % dim] = seen.double() * weight / total
    return out


def check_needles(got, at, score, n, kv_heads, dim):
    want = needles_wanted(at, score, n, got.shape[2], kv_heads, dim)
    off = (got.cpu().double() - want).abs()
    # The score has one product, and is off by three roundings; the exponential by its
    # argument's, 3 U of its size in units of ln 2, and by one of its own, in the
    # needles' sum and in the total; the total's chain of ones, below 2^24 terms of
    # which the lanes, waves and parts add at most 2^13 each: 2^13 U.  p in bfloat16:
    # half a step where it is rounded.
    exponent = 2 * (3 * U * score + 3 * U * 1.45 * score + U)
    allowed = want * (exponent + 2.0 ** 13 * U + 2 * HALF[got.dtype] * 1.01) + 2.0 ** -126
    assert bool((off <= allowed).all()), float((off - allowed).max())
