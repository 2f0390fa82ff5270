"""What the operators of a training step around the loss are timed on.

Three operators, through the package's public functions:

* ``clip``: ``grad_norm``, the 2-norm over a list of gradients, and
  ``clip_grads``, which also scales them in place where it exceeds a limit;
* ``layer_norm``: forward, and backward with the weight's and bias's gradients;
* ``attention``: softmax attention with shared key/value heads, causal or not,
  with a number of keys per sequence; forward (one token after another, or a
  prompt), and forward with the gradients of queries, keys and values.

Where ``own`` is false each is computed in elementary torch operations in
binary32 (the long sum of squares in binary64).
"""
from __future__ import annotations

import math
import random

import torch

own = False

CLIP_EPS = 1e-6
NORM_EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------ cases
def _clip(name, kind, dim, inter, layers, vocab, dtype, mixed=False, scale=True):
    return {"name": name, "op": "clip", "kind": kind, "dim": dim, "inter": inter, "layers": layers, "vocab": vocab,
            "dtype": dtype, "mixed": mixed, "scale": scale}


def _norm(name, rows, cols, dtype, weight, pad=0, train=True):
    return {"name": name, "op": "layer_norm", "rows": rows, "cols": cols, "dtype": dtype, "weight": weight,
            "pad": pad, "train": train}


def _attn(name, batch, queries, keys, heads, kv_heads, dim, dtype, causal=True, lengths=False, packed=False,
          train=True):
    return {"name": name, "op": "attention", "batch": batch, "queries": queries, "keys": keys, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "causal": causal, "lengths": lengths,
            "packed": packed, "train": train}


def listed():
    return [
        # logging the norm: the gradients of the package's 4-layer, 256-wide
        # training loop, 53 tensors in one bucket
        _clip("norm_256x4_f32", "gelu", 256, 1024, 4, 1024, "f32", scale=False),
        # a model of odd widths, matrices in bfloat16 and vectors in binary32,
        # so that tensors start anywhere in their buckets
        _clip("clip_517x9_mixed", "gelu", 517, 1231, 9, 5003, "bf16", mixed=True),
        # 8 layers of the Llama-2-7B list with both embeddings: 1.9e9 elements
        _clip("clip_llama2_7b_8_bf16", "gated", 4096, 11008, 8, 32000, "bf16"),
        # one generated token
        _norm("ln_fwd_1x4096_bf16", 1, 4096, "bf16", "bf16", train=False),
        # the training loop's: batch 32 x 128 tokens
        _norm("ln_4096x256_f32", 4096, 256, "f32", "f32"),
        # odd sizes, rows at an odd stride, binary32 weights of bfloat16 activations
        _norm("ln_509x1031_bf16", 509, 1031, "bf16", "f32", pad=7),
        # fine-tuning: 8 sequences of 2048 tokens at once
        _norm("ln_16384x4096_bf16", 16384, 4096, "bf16", "bf16"),
        # generating: 8 sequences of up to 4096 tokens, four heads to a key head
        _attn("attn_decode_8x4096_bf16", 8, 1, 4096, 32, 8, 128, "bf16", causal=False, lengths=True, train=False),
        # a long prompt's next token alone, in binary32
        _attn("attn_decode_1x32768_f32", 1, 1, 32768, 32, 8, 128, "f32", causal=False, train=False),
        # the training loop's: q, k and v lie in one projection's output
        _attn("attn_32x128x64_f32", 32, 128, 128, 4, 4, 64, "f32", packed=True),
        # odd lengths, a padded batch with an empty sequence, shared heads
        _attn("attn_3x515x1031x80_bf16", 3, 515, 1031, 6, 2, 80, "bf16", causal=False, lengths=True),
        # fine-tuning: 2 sequences of 4096 tokens, 32 heads
        _attn("attn_2x4096x128_bf16", 2, 4096, 4096, 32, 32, 128, "bf16", packed=True),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(["clip", "layer_norm", "attention"])
    dtype = rng.choice(["bf16", "f32"])
    if op == "clip":
        while True:
            dim = _log_uniform(rng, 64, 4096)
            case = _clip("", rng.choice(["gelu", "gated"]), dim, int(dim * rng.uniform(2.0, 4.0)),
                         _log_uniform(rng, 1, 32), _log_uniform(rng, 256, 50257), dtype, rng.random() < 0.3,
                         rng.random() < 0.7)
            if work(case)["bytes"] <= 8e9:
                break
    elif op == "layer_norm":
        while True:
            rows, cols = _log_uniform(rng, 1, 65536), _log_uniform(rng, 64, 16384)
            if rows * cols * SIZE[dtype] <= 16384 * 4096 * 2:
                break
        case = _norm("", rows, cols, dtype, rng.choice([dtype, "f32"]), rng.choice([0, 0, 1, 24]),
                     rng.random() < 0.7)
    else:
        train = rng.random() < 0.6
        while True:
            group, kv = rng.choice([1, 1, 2, 4, 8]), _log_uniform(rng, 1, 32)
            keys = _log_uniform(rng, 1, 4096 if train else 65536)
            queries = (keys if rng.random() < 0.7 else _log_uniform(rng, 1, 4096)) if train else (
                1 if rng.random() < 0.6 else _log_uniform(rng, 1, 2048))
            case = _attn("", _log_uniform(rng, 1, 32), queries, keys, group * kv, kv,
                         rng.choice([32, 64, 64, 80, 96, 128, 128]), dtype, rng.random() < 0.6, rng.random() < 0.4,
                         group == 1 and queries == keys and rng.random() < 0.5, train)
            # the scores in binary32 at most 2 GiB, binary32 at a sixteenth of the largest case's products
            scores = case["batch"] * case["heads"] * queries * keys
            if scores <= 1 << 29 and work(case)["flops"] <= (1e12 if dtype == "bf16" else 6e10) and (
                    work(case)["bytes"] <= 4e9):
                break
    del case["name"]
    return case


# ----------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _lists(case):
    """(matrices, vectors): the shapes of a model's gradients."""
    d, f, n, v = case["dim"], case["inter"], case["layers"], case["vocab"]
    if case["kind"] == "gelu":
        layer = [(3 * d, d), (d, d), (f, d), (d, f)]
        small = [(d,)] * 4 + [(3 * d,), (d,), (f,), (d,)]
    else:
        layer = [(d, d)] * 4 + [(f, d)] * 2 + [(d, f)]
        small = [(d,)] * 2
    return [(v, d)] + layer * n + [(v, d)], small * n + [(d,)]


def _count(shapes):
    return sum(math.prod(s) for s in shapes)


def _bucket(shapes, dtype, g):
    """One flat buffer and the gradients as views of it, one behind the other:
    how data-parallel training keeps them."""
    flat = torch.randn(_count(shapes), generator=g, device="cuda").mul_(1e-3).to(dtype)
    views, at = [], 0
    for s in shapes:
        views.append(flat[at:at + math.prod(s)].view(s))
        at += math.prod(s)
    return flat, views


def _key_lengths(case, g):
    """Between no key and all of them: the first sequence is whole, the second
    empty, the others spread."""
    n = torch.randint(1, case["keys"] + 1, (case["batch"],), generator=g, device="cuda", dtype=torch.int32)
    n[0] = case["keys"]
    if case["batch"] > 1:
        n[1] = 0
    return n


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "clip":
        matrices, vectors = _lists(case)
        if case["mixed"]:
            parts = [_bucket(matrices, DTYPES[case["dtype"]], g), _bucket(vectors, torch.float32, g)]
        else:
            parts = [_bucket(matrices + vectors, DTYPES[case["dtype"]], g)]
        # the norm is about 1e-3 sqrt(elements): a limit below it
        limit = 0.37e-3 * math.sqrt(_count(matrices) + _count(vectors))
        return {"op": "clip", "buckets": [p[0] for p in parts], "grads": [v for p in parts for v in p[1]],
                "max_norm": limit, "scale": case["scale"]}
    if case["op"] == "layer_norm":
        rows, cols, dtype, wt = case["rows"], case["cols"], DTYPES[case["dtype"]], DTYPES[case["weight"]]
        # activations with a few strong channels and a row-dependent offset, as residual streams have them
        store = torch.randn(rows, cols + case["pad"], generator=g, device="cuda")
        store *= 0.5 + 4.0 * (torch.rand(cols + case["pad"], generator=g, device="cuda") > 0.98)
        store += torch.randn(rows, 1, generator=g, device="cuda") * 0.3
        x = store.to(dtype)[:, :cols]
        weight = (1.0 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(wt)
        bias = (0.1 * torch.randn(cols, generator=g, device="cuda")).to(wt)
        state = {"op": "layer_norm", "x": x, "weight": weight, "bias": bias, "train": case["train"]}
        if case["train"]:
            state["dy"] = (torch.randn(rows, cols, generator=g, device="cuda") * 1e-2).to(dtype)
            for k in ("x", "weight", "bias"):
                state[k].requires_grad_()
        return state
    b, sq, sk, h, hk, d, dtype = (case[k] for k in ("batch", "queries", "keys", "heads", "kv_heads", "dim", "dtype"))
    if case["packed"]:
        whole = torch.randn(b, sq, 3, h, d, generator=g, device="cuda").to(DTYPES[dtype])
        q, k, v = whole.unbind(2)
    else:
        q = torch.randn(b, sq, h, d, generator=g, device="cuda").to(DTYPES[dtype])
        k = torch.randn(b, sk, hk, d, generator=g, device="cuda").to(DTYPES[dtype])
        v = torch.randn(b, sk, hk, d, generator=g, device="cuda").to(DTYPES[dtype])
    state = {"op": "attention", "q": q, "k": k, "v": v, "causal": case["causal"], "train": case["train"],
             "lengths": _key_lengths(case, g) if case["lengths"] else None}
    if case["train"]:
        state["do"] = torch.randn(b, sq, h, d, generator=g, device="cuda").to(DTYPES[dtype])
        for n in ("q", "k", "v"):
            state[n] = state[n].detach().requires_grad_()
    return state


# ------------------------------------------------------------ plain forms
def _step_limit(state):
    """The limit of this pass, a hair below the last one's: a pass over
    gradients that a pass has clipped clips them again."""
    limit = state["max_norm"]
    state["max_norm"] = limit * (1.0 - 1e-5)
    return limit


def _plain_clip(state):
    total = sum((b.float().square().sum(dtype=torch.float64) for b in state["buckets"]),
                torch.zeros((), dtype=torch.float64, device="cuda"))
    norm = total.sqrt()
    if not state["scale"]:
        return {"norm": norm.float()}
    factor = (_step_limit(state) / (norm + CLIP_EPS)).clamp(max=1.0).float()
    [b.copy_(b.float() * factor) for b in state["buckets"]]
    return {"norm": norm.float(), "grads": state["buckets"]}


def _plain_layer_norm(state):
    x, w, b = state["x"].float(), state["weight"].float(), state["bias"].float()
    mean = x.mean(1, keepdim=True)
    centred = x - mean
    rstd = (centred.square().mean(1, keepdim=True) + NORM_EPS).rsqrt()
    xhat = centred * rstd
    out = {"y": (xhat * w + b).to(state["x"].dtype)}
    if state["train"]:
        dy = state["dy"].float()
        g = dy * w
        dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        out["dx"] = dx.to(state["x"].dtype)
        out["dweight"] = (dy * xhat).sum(0).to(state["weight"].dtype)
        out["dbias"] = dy.sum(0).to(state["bias"].dtype)
    return out


def _plain_attention(state):
    dtype = state["q"].dtype
    q, k, v = (state[n].float().transpose(1, 2) for n in ("q", "k", "v"))
    b, h, sq, d = q.shape
    hk, sk = k.shape[1:3]
    group, scale = h // hk, 1.0 / math.sqrt(d)
    q = q.reshape(b, hk, group * sq, d)            # heads that share keys, one behind the other
    k, v = k.contiguous(), v.contiguous()
    s = (q @ k.transpose(2, 3).contiguous()).mul_(scale)
    key = torch.arange(sk, device="cuda")
    if state["causal"]:
        last = torch.arange(sq, device="cuda").repeat(group) + (sk - sq)
        s.masked_fill_(key[None, :] > last[:, None], -math.inf)
    if state["lengths"] is not None:
        s.masked_fill_(key[None, :] >= state["lengths"][:, None, None, None], -math.inf)
    top = s.amax(3, keepdim=True)
    p = s.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(3, keepdim=True)
    p /= torch.where(total == 0, torch.ones_like(total), total)

    def back(t, heads):
        return t.reshape(b, heads, -1, d).transpose(1, 2).contiguous().to(dtype)

    out = {"out": back(p @ v, h)}
    if state["train"]:
        do = state["do"].float().transpose(1, 2).reshape(b, hk, group * sq, d)
        out["dv"] = back(p.transpose(2, 3).contiguous() @ do, hk)
        dp = do @ v.transpose(2, 3).contiguous()
        dp -= (p * dp).sum(3, keepdim=True)
        ds = dp.mul_(p).mul_(scale)
        out["dq"] = back(ds @ k, h)
        out["dk"] = back(ds.transpose(2, 3).contiguous() @ q, hk)
    return out


@torch.no_grad()
def _plain(state):
    return {"clip": _plain_clip, "layer_norm": _plain_layer_norm, "attention": _plain_attention}[state["op"]](state)


def run(state):
    if not own:
        return _plain(state)
    if state["op"] == "clip":
        from paper_2405_15593_amd.clip import clip_grads, grad_norm
        if not state["scale"]:
            return {"norm": grad_norm(state["grads"])}
        return {"norm": clip_grads(state["grads"], _step_limit(state), eps=CLIP_EPS), "grads": state["buckets"]}
    if state["op"] == "layer_norm":
        from paper_2405_15593_amd.norm import layer_norm
        y = layer_norm(state["x"], state["weight"], state["bias"], eps=NORM_EPS)
        if not state["train"]:
            return {"y": y}
        dx, dw, db = torch.autograd.grad(y, (state["x"], state["weight"], state["bias"]), state["dy"])
        return {"y": y, "dx": dx, "dweight": dw, "dbias": db}
    from paper_2405_15593_amd.attention import attention
    out = attention(state["q"], state["k"], state["v"], causal=state["causal"], key_lengths=state["lengths"])
    if not state["train"]:
        return {"out": out}
    dq, dk, dv = torch.autograd.grad(out, (state["q"], state["k"], state["v"]), state["do"])
    return {"out": out, "dq": dq, "dk": dk, "dv": dv}


# -------------------------------------------------------------- the floor
def work(case):
    if case["op"] == "clip":
        matrices, vectors = _lists(case)
        m, v = _count(matrices), _count(vectors)
        size = m * SIZE[case["dtype"]] + v * (4 if case["mixed"] else SIZE[case["dtype"]])
        # the factor is known only when all have been read: read, read again, written
        return {"bytes": size * (3 if case["scale"] else 1) + 4, "flops": (m + v) * (3 if case["scale"] else 2)}
    if case["op"] == "layer_norm":
        n, t = case["rows"] * case["cols"], SIZE[case["dtype"]]
        side = case["cols"] * SIZE[case["weight"]]
        if not case["train"]:
            return {"bytes": 2 * n * t + 2 * side, "flops": 8 * n}
        # forward: x in, y out; backward: x and dy in, dx out, two statistics a row
        return {"bytes": 5 * n * t + 5 * side + 16 * case["rows"], "flops": 22 * n}
    b, sq, sk, h, hk, d, t = (case[k] for k in ("batch", "queries", "keys", "heads", "kv_heads", "dim", "dtype"))
    pairs = sq * sk
    if case["causal"]:          # query i sees the keys up to i + sk - sq
        n, short = min(sq, sk), max(0, sk - sq)
        pairs = n * (n + 1) // 2 + n * short
    share = 0.5 if case["lengths"] and b > 1 else 1.0          # what the lengths leave, about
    products = 4 * b * h * d * pairs * share
    query, key = b * sq * h * d * SIZE[t], b * sk * hk * d * SIZE[t]
    if not case["train"]:
        return {"bytes": int(2 * query + 2 * key * share), "flops": int(products)}
    # backward: scores again, dp, dv, dq, dk
    return {"bytes": int(6 * query + 4 * key * share + 2 * key), "flops": int(3.5 * products)}


# ------------------------------------------------- definitions in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "clip":
        norm = math.sqrt(sum(float(torch.dot(part.double(), part.double())) for b in state["buckets"]
                             for part in b.split(1 << 26)))
        out = {"norm": torch.tensor(norm, dtype=torch.float64)}
        if case["scale"]:
            c = min(1.0, state["max_norm"] / (norm + CLIP_EPS))
            out["grads"] = [b.double() * c for b in state["buckets"]]
        return out
    with torch.no_grad():
        if case["op"] == "layer_norm":
            x, w = state["x"].double(), state["weight"].double()
            var, mean = torch.var_mean(x, 1, correction=0)
            sd = torch.sqrt(var + NORM_EPS)[:, None]
            xhat = (x - mean[:, None]) / sd
            out = {"y": torch.addcmul(state["bias"].double(), xhat, w)}
            if case["train"]:
                dy = state["dy"].double()
                g, n = dy * w, case["cols"]
                # the projection of g off the directions 1 and xhat
                out["dx"] = (g - (g @ torch.ones(n, 1, dtype=g.dtype, device="cuda")
                                  + xhat * (g * xhat).sum(1, keepdim=True)) / n) / sd
                out["dweight"] = torch.linalg.vecdot(dy, xhat, dim=0)
                out["dbias"] = torch.ones(case["rows"], dtype=g.dtype, device="cuda") @ dy
            return out
        return _exact_attention(case, state)


def _exact_attention(case, state):
    q, k, v = (state[n].detach().double() for n in ("q", "k", "v"))
    b, sq, h, d = q.shape
    sk, group = k.shape[1], h // k.shape[2]
    out = torch.zeros_like(q, memory_format=torch.contiguous_format)
    dq = torch.zeros_like(out)
    dk, dv = (torch.zeros(k.shape, dtype=k.dtype, device="cuda") for _ in range(2))
    lengths = [sk] * b if state["lengths"] is None else state["lengths"].tolist()
    for i in range(b):
        n = lengths[i]
        if n == 0:
            continue
        seen = torch.ones(sq, n, dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen = seen.tril(sk - sq)
        hidden, some = ~seen, seen.any(1, keepdim=True)
        for j in range(h):
            kj, vj = k[i, :n, j // group], v[i, :n, j // group]
            z = (q[i, :, j] @ kj.t().contiguous() / d ** 0.5).masked_fill_(hidden, -math.inf)
            p = torch.softmax(z, 1).masked_fill_(~some, 0.0)
            out[i, :, j] = p @ vj
            if case["train"]:
                do = state["do"][i, :, j].double()
                dv[i, :n, j // group] += p.t().contiguous() @ do
                pull = do @ vj.t().contiguous() - (do * out[i, :, j]).sum(1, keepdim=True)
                ds = p.mul_(pull) / d ** 0.5
                dq[i, :, j] = ds @ kj
                dk[i, :n, j // group] += ds.t().contiguous() @ q[i, :, j]
    return {"out": out, "dq": dq, "dk": dk, "dv": dv} if case["train"] else {"out": out}
