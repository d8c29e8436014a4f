"""Attention with its backward pass, group norm with an activation and its backward pass, and dropout, as cases
that can be timed and compared.

A case is one call on inputs, outputs and scratch that an adaptation step has in hand.
`listed()` gives the fixed cases, `draw(rng)` one more of the same ranges.  Where `own` is false the
operators are computed in their plain form, elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}
EPS = 1e-5                      # of the group norms


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------

def _attention(name, op, batch, heads, kv_heads, q_len, kv_len, head_dim, causal=False, ragged=False, layout="rows"):
    """`ragged`: a padded batch, whose lengths go from none to all of the rows.  `layout`: "rows" [batch, row, head, dim],
    "heads" [batch, head, row, dim], "packed" [batch, row, 3, head, dim] as one linear layer writes queries, keys and values."""
    return {"name": name, "op": op, "batch": batch, "heads": heads, "kv_heads": kv_heads, "q_len": q_len, "kv_len": kv_len,
            "head_dim": head_dim, "causal": causal, "ragged": ragged, "layout": layout}


def _group_norm(name, batch, positions, channels, groups, act, dtype, stats=True):
    return {"name": name, "op": "group_norm", "batch": batch, "positions": positions, "channels": channels,
            "groups": groups, "act": act, "dtype": dtype, "stats": stats}


def _group_norm_grad(name, batch, positions, channels, groups, act, dtype, grad_dtype):
    return {"name": name, "op": "group_norm_grad", "batch": batch, "positions": positions, "channels": channels,
            "groups": groups, "act": act, "dtype": dtype, "grad_dtype": grad_dtype}


def _dropout(name, n, dtype, p, residual):
    return {"name": name, "op": "dropout", "n": n, "dtype": dtype, "p": p, "residual": residual}


def listed():
    return [
        # one query a sequence over many keys that heads share (pooling by attention, a single token served): bytes of the keys and values
        _attention("attention one query", "attention", 8, 16, 4, 1, 8192, 128),
        # a ViT-B block at the benchmark's batch: 64 images of 197 tokens, straight from the qkv layer's output
        _attention("attention vit", "attention", 64, 12, 12, 197, 197, 64, layout="packed"),
        # Segformer-B5's first stage on one 1024x1024 image: a query per position, keys on the reduced grid
        _attention("attention segformer stage 1", "attention", 1, 1, 1, 65536, 1024, 64),
        # the backward pass of the ViT-B block, gradients straight to where the qkv layer's backward pass reads them
        _attention("attention grad vit", "attention_grad", 64, 12, 12, 197, 197, 64, layout="packed"),
        # a padded batch of images of different sizes, Segformer's third stage's heads, rows of a length that fills no tile
        _attention("attention grad padded batch", "attention_grad", 16, 5, 5, 1003, 1003, 64, ragged=True),
        # a long causal sequence with shared heads
        _attention("attention grad long causal", "attention_grad", 1, 8, 2, 8192, 8192, 128, causal=True, layout="heads"),
        # a Segformer head at a quarter of a 1024x1024 image's resolution: one image, 100 MB
        _group_norm("group norm segformer head", 1, 65536, 768, 32, "relu", "bf16"),
        # one small image in the last stage of a ResNet: latency
        _group_norm("group norm one small image", 1, 49, 2048, 32, "relu", "fp32"),
        # ResNet-50's first stage at the benchmark's batch (64 images of 56x56)
        _group_norm_grad("group norm grad resnet stage 1", 64, 3136, 256, 32, "relu", "bf16", "bf16"),
        # three images of an odd number of positions, ten channels a group, fp32 throughout
        _group_norm_grad("group norm grad odd", 3, 3001, 320, 32, "silu", "fp32", "fp32"),
        # after a ViT-B block's projection, with the skip connection
        _dropout("dropout vit", 64 * 197 * 768, "bf16", 0.1, True),
        # its gradient's form for one row of features of an odd length: latency
        _dropout("dropout one row", 2049, "fp32", 0.5, False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention_grad", "attention_grad", "group_norm", "group_norm_grad", "dropout"])
    if op in ("attention", "attention_grad"):
        d = rng.choice([64, 64, 128, 32, 80, 8 * rng.randint(1, 16)])
        kv_heads = _log_int(rng, 1, 12)
        heads = kv_heads * rng.choice([1, 1, 1, 2, 4])
        layout = rng.choice(["rows", "heads", "packed"])
        batch = _log_int(rng, 1, 64)
        # as many pairs of a query and a key as about half of the longest listed case computes
        pairs = (1 << 28) // (batch * heads) * 64 // max(d, 64)
        # (with one key the probability is 1 and the gradients of queries and keys are 0: nothing to compare)
        least = 1 if op == "attention" else 4
        kv_len = _log_int(rng, least, min(16384, max(2 * least, pairs)))
        q_len = kv_len if rng.random() < 0.5 else rng.choice([1, _log_int(rng, 1, 65536)])
        q_len = max(1, min(q_len, pairs // kv_len, (1 << 26) // (batch * heads * d)))
        kv_len = max(least, min(kv_len, (1 << 26) // (batch * kv_heads * d)))
        if layout == "packed":
            kv_heads, q_len = heads, max(least, min(q_len, kv_len))
            kv_len = q_len
        case = _attention("", op, batch, heads, kv_heads, q_len, kv_len, d, causal=rng.random() < 0.3,
                          ragged=rng.random() < 0.3, layout=layout)
    elif op in ("group_norm", "group_norm_grad"):
        groups = rng.choice([1, 8, 32, 32, 32, _log_int(rng, 1, 64)])
        channels = groups * max(1, _log_int(rng, 16, 2048) // groups)
        batch = _log_int(rng, 1, 64)
        # (of a group of one or two numbers hardly any gradient is left)
        positions = _log_int(rng, 8, max(8, min(65536, (1 << 25) // (channels * batch))))
        act, dtype = rng.choice(["none", "relu", "gelu", "silu"]), rng.choice(["bf16", "fp32"])
        if op == "group_norm":
            case = _group_norm("", batch, positions, channels, groups, act, dtype, stats=rng.random() < 0.7)
        else:
            case = _group_norm_grad("", batch, positions, channels, groups, act, dtype,
                                    rng.choice(["bf16", "fp32"]) if dtype == "bf16" else "fp32")
    else:
        case = _dropout("", _log_int(rng, 1, 20_000_000), rng.choice(["bf16", "fp32"]), rng.choice([0.05, 0.1, 0.5, rng.random()]),
                        rng.random() < 0.5)
    del case["name"]
    return case


def _lengths(case):
    """Rows of each sequence of a padded batch, queries and keys: from none to all."""
    b = case["batch"]
    part = [i / (b - 1) if b > 1 else 0.7 for i in range(b)]
    return [round(case["q_len"] * p) for p in part], [round(case["kv_len"] * p) for p in part]


def _pairs(case):
    """Pairs of a query and a key that it sees, of one head."""
    ql, kl = _lengths(case) if case["ragged"] else ([case["q_len"]] * case["batch"], [case["kv_len"]] * case["batch"])
    if not case["causal"]:
        return sum(q * k for q, k in zip(ql, kl))
    total = 0
    for q, k in zip(ql, kl):                      # query i sees the first i + 1 + k - q keys
        first, last = max(0, 1 + k - q), k
        total += (first + last) * (last - first + 1) // 2 if q else 0
    return total


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------

def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _views(case, dtype=torch.bfloat16, fill=None):
    """Queries, keys and values [batch, row, head, dim] as views of the case's layout, filled by fill(shape)."""
    b, h, hk, nq, nk, d = (case[k] for k in ("batch", "heads", "kv_heads", "q_len", "kv_len", "head_dim"))
    make = fill or (lambda *s: torch.empty(*s, dtype=dtype, device="cuda"))
    if case["layout"] == "packed":
        return make(b, nq, 3, h, d).unbind(2)
    if case["layout"] == "heads":
        return tuple(make(b, heads, n, d).transpose(1, 2) for heads, n in ((h, nq), (hk, nk), (hk, nk)))
    return tuple(make(b, n, heads, d) for heads, n in ((h, nq), (hk, nk), (hk, nk)))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _data(case, seed):
    """The tensors that the call reads, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    if op in ("attention", "attention_grad"):
        b, h, nq, d = (case[k] for k in ("batch", "heads", "q_len", "head_dim"))
        q, k, v = _views(case, fill=lambda *s: _randn(g, *s, dtype=torch.bfloat16))
        s = {"q": q, "k": k, "v": v, "q_lengths": None, "kv_lengths": None, "scale": d ** -0.5}
        if case["ragged"]:
            s["q_lengths"], s["kv_lengths"] = (_ints(v) for v in _lengths(case))
        if op == "attention_grad":
            o, lse = _forward(s, case, torch.float32)
            s["out"], s["lse"] = o.to(torch.bfloat16), lse
            s["dout"] = _randn(g, b, nq, h, d, scale=0.01, dtype=torch.bfloat16)
        return s
    if op in ("group_norm", "group_norm_grad"):
        b, p, c, dt = case["batch"], case["positions"], case["channels"], TYPES[case["dtype"]]
        # a convolution's outputs: their own spread and offset per channel
        x = (_randn(g, b, p, c) * (0.5 + torch.rand(c, generator=g, device="cuda")) + _randn(g, c, scale=0.5)).to(dt)
        s = {"x": x, "gamma": 1.0 + _randn(g, c, scale=0.2), "beta": _randn(g, c, scale=0.2)}
        if op == "group_norm_grad":
            s["dy"] = _randn(g, b, p, c, scale=0.01, dtype=TYPES[case["grad_dtype"]])
            f = x.view(b, p, case["groups"], -1).double()
            s["stats"] = torch.stack([f.mean((1, 3)), (f.var((1, 3), unbiased=False) + EPS).rsqrt()]).float()
        return s
    n, dt = case["n"], TYPES[case["dtype"]]
    return {"x": _randn(g, n, dtype=dt), "residual": _randn(g, n, dtype=dt) if case["residual"] else None,
            "seed": 0x9E3779B97F4A7C15 ^ seed, "offset": 12345 + (seed << 33)}


def prepare(case, seed):
    s = {"case": case, **_data(case, seed)}
    op = case["op"]
    if op == "attention":
        s["out"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(case["batch"], case["heads"], case["q_len"], device="cuda")
    elif op == "attention_grad":
        s["dq"], s["dk"], s["dv"] = _views(case)
    elif op == "group_norm":
        s["y"] = torch.empty_like(s["x"])
        s["stats"] = torch.empty(2, case["batch"], case["groups"], device="cuda") if case["stats"] else None
    elif op == "group_norm_grad":
        s["dx"] = torch.empty_like(s["dy"])
        s["dgamma"], s["dbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
    else:
        s["y"] = torch.empty_like(s["x"])
    if own:                                       # the handles and the scratch that a program makes once
        from paper_2503_20354_b200 import binding as B
        need = 0
        if op in ("attention", "attention_grad"):
            s["desc"] = B.attention_desc(case["batch"], case["heads"], case["q_len"], case["kv_len"], case["head_dim"],
                                         kv_heads=case["kv_heads"], causal=case["causal"], scale=s["scale"])
            need = (B.surgeon_attention_workspace if op == "attention" else B.surgeon_attention_grad_workspace)(s["desc"])
        elif op != "dropout":
            need = (B.surgeon_group_norm_workspace if op == "group_norm" else B.surgeon_group_norm_grad_workspace)(
                case["batch"], case["positions"], case["channels"], case["groups"])
        s["scratch"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _PLAIN[s["case"]["op"]](s)


def _run_own(s):
    from paper_2503_20354_b200 import binding as B
    case = s["case"]
    op = case["op"]
    if op == "attention":
        B.surgeon_attention(s["desc"], s["q"], s["k"], s["v"], q_lengths=s["q_lengths"], kv_lengths=s["kv_lengths"], out=s["out"],
                            lse=s["lse"], workspace=s["scratch"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "attention_grad":
        B.surgeon_attention_grad(s["desc"], s["q"], s["k"], s["v"], s["out"], s["dout"], s["lse"], q_lengths=s["q_lengths"],
                                 kv_lengths=s["kv_lengths"], dq=s["dq"], dk=s["dk"], dv=s["dv"], workspace=s["scratch"])
        return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    if op == "dropout":
        B.surgeon_dropout(s["x"], case["p"], s["seed"], s["offset"], residual=s["residual"], out=s["y"])
        return {"y": s["y"]}
    act = {"none": B.SURGEON_ACT_NONE, "relu": B.SURGEON_ACT_RELU, "gelu": B.SURGEON_ACT_GELU, "silu": B.SURGEON_ACT_SILU}[case["act"]]
    if op == "group_norm":
        B.surgeon_group_norm(s["x"], case["groups"], s["gamma"], s["beta"], EPS, act=act, out=s["y"], stats=s["stats"],
                             workspace=s["scratch"])
        return {"y": s["y"], "stats": s["stats"]}
    B.surgeon_group_norm_grad(s["x"], s["dy"], case["groups"], s["gamma"], s["beta"], s["stats"], act=act, dx=s["dx"],
                              dgamma=s["dgamma"], dbeta=s["dbeta"], workspace=s["scratch"])
    return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _heads_first(t, times, dtype):
    """[batch, head, row, dim] in `dtype`, every head `times` times in a row."""
    t = t.transpose(1, 2).to(dtype)
    return t.repeat_interleave(times, 1) if times > 1 else t


def _hidden(s, case):
    """Where a query does not see a key ([batch, 1, query, key] or less, true: hidden), or None."""
    q_len, kv_len = case["q_len"], case["kv_len"]
    i, j = torch.arange(q_len, device="cuda")[:, None], torch.arange(kv_len, device="cuda")[None]
    if case["ragged"]:
        ql, kl = s["q_lengths"].view(-1, 1, 1, 1), s["kv_lengths"].view(-1, 1, 1, 1)
        hidden = (i >= ql) | (j >= kl)
        return hidden | (j > i + (kl - ql)) if case["causal"] else hidden
    return (j > i + (kv_len - q_len))[None, None] if case["causal"] else None


def _scores(s, case, dtype):
    times = case["heads"] // case["kv_heads"]
    x = (_heads_first(s["q"], 1, dtype) @ _heads_first(s["k"], times, dtype).transpose(2, 3)) * s["scale"]
    hidden = _hidden(s, case)
    return x if hidden is None else x.masked_fill(hidden, -math.inf)


def _forward(s, case, dtype):
    """o [batch, query, head, dim] and lse [batch, head, query]."""
    x = _scores(s, case, dtype)
    top = x.amax(3, keepdim=True).clamp(min=-1e30)
    x = torch.exp(x - top)
    total = x.sum(3, keepdim=True)
    lse = (top + torch.log(total)).squeeze(3)
    o = (x @ _heads_first(s["v"], case["heads"] // case["kv_heads"], dtype)) / total.masked_fill(total == 0, 1.0)
    return o.transpose(1, 2).contiguous(), lse.masked_fill(total.squeeze(3) == 0, -math.inf)


def _plain_attention(s):
    o, lse = _forward(s, s["case"], torch.float32)
    return {"out": o.to(torch.bfloat16), "lse": lse}


def _backward(s, case, dtype):
    times = case["heads"] // case["kv_heads"]
    q, k, v = (_heads_first(s[n], 1 if n == "q" else times, dtype) for n in "qkv")
    o, do = (_heads_first(s[n], 1, dtype) for n in ("out", "dout"))
    lse = s["lse"].to(dtype)
    p = torch.exp(_scores(s, case, dtype) - lse.masked_fill(lse == -math.inf, 0.0)[..., None])
    dv = p.transpose(2, 3) @ do
    ds = (do @ v.transpose(2, 3) - (do * o).sum(3, keepdim=True)).mul_(p).mul_(s["scale"])
    del p
    dq, dk = ds @ k, ds.transpose(2, 3) @ q
    b, nk, hk, d = s["k"].shape
    shared = lambda t: t.view(b, hk, times, nk, d).sum(2).transpose(1, 2)
    return {"dq": dq.transpose(1, 2), "dk": shared(dk), "dv": shared(dv)}


def _plain_attention_grad(s):
    grads = _backward(s, s["case"], torch.float32)
    for name, t in grads.items():
        s[name].copy_(t)
    return {name: s[name] for name in grads}


def _plain_act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * 2.0 ** -0.5))
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _plain_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 2.0 ** -0.5)) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig))


def _plain_group_norm(s):
    case = s["case"]
    x = s["x"].float().view(case["batch"], case["positions"], case["groups"], -1)
    mean = x.mean((1, 3), keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean((1, 3), keepdim=True) + EPS)
    z = (c * rstd).view_as(s["x"]) * s["gamma"] + s["beta"]
    stats = torch.stack([mean.view(case["batch"], -1), rstd.view(case["batch"], -1)]) if case["stats"] else None
    return {"y": _plain_act(z, case["act"]).to(s["x"].dtype), "stats": stats}


def _plain_group_norm_grad(s):
    case = s["case"]
    x = s["x"].float().view(case["batch"], case["positions"], case["groups"], -1)
    mean, rstd = (t[:, None, :, None] for t in s["stats"])
    xh = ((x - mean) * rstd).view_as(s["x"])
    dz = s["dy"].float()
    if case["act"] != "none":
        dz = dz * _plain_slope(xh * s["gamma"] + s["beta"], case["act"])
    g, h = (dz * s["gamma"]).view_as(x), xh.view_as(x)
    dx = rstd * (g - g.mean((1, 3), keepdim=True) - h * (g * h).mean((1, 3), keepdim=True))
    return {"dx": dx.view_as(dz).to(s["dy"].dtype), "dgamma": (dz * xh).sum((0, 1)), "dbeta": dz.sum((0, 1))}


def _plain_bits(n, seed, offset):
    """16 random bits for each of n elements: Philox 4x32 with ten rounds, eight elements to a counter."""
    low = 0xFFFFFFFF
    i = torch.arange(-(-n // 8), device="cuda")
    offset &= (1 << 64) - 1
    a, b = i & low, i >> 32
    c, d = torch.full_like(i, offset & low), torch.full_like(i, offset >> 32)
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        x, y = a * 0xD2511F53, c * 0xCD9E8D57    # (the upper halves are right although the products wrap)
        a, b, c, d = (y >> 32 & low) ^ b ^ k0, y & low, (x >> 32 & low) ^ d ^ k1, x & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    words = torch.stack([a, b, c, d], 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:n]


def _plain_dropout(s):
    case = s["case"]
    dropped = int(math.floor(case["p"] * 65536 + 0.5))
    keep = _plain_bits(case["n"], s["seed"], s["offset"]) >= dropped
    y = torch.where(keep, s["x"].float() * (65536.0 / max(65536 - dropped, 1)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(s["x"].dtype)}


_PLAIN = {"attention": _plain_attention, "attention_grad": _plain_attention_grad, "group_norm": _plain_group_norm,
          "group_norm_grad": _plain_group_norm_grad, "dropout": _plain_dropout}


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without, and what it returns in 64 bits
# ---------------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op in ("attention", "attention_grad"):
        b, h, hk, nq, nk, d = (case[k] for k in ("batch", "heads", "kv_heads", "q_len", "kv_len", "head_dim"))
        q_in, kv_in = (sum(v) for v in _lengths(case)) if case["ragged"] else (b * nq, b * nk)
        q, kv, flops = h * d * 2, 2 * hk * d * 2, _pairs(case) * h * d
        if op == "attention":
            return {"bytes": q_in * q + kv_in * kv + b * nq * (q + 4 * h), "flops": 4 * flops}
        return {"bytes": q_in * (3 * q + 4 * h) + kv_in * kv + b * (nq * q + nk * kv), "flops": 10 * flops}
    if op == "dropout":
        return {"bytes": case["n"] * (3 if case["residual"] else 2) * SIZE[case["dtype"]], "flops": 2 * case["n"]}
    c = case["channels"]
    n, stats = case["batch"] * case["positions"] * c, 8 * case["batch"] * case["groups"]
    if op == "group_norm":
        return {"bytes": 2 * n * SIZE[case["dtype"]] + 8 * c + (stats if case["stats"] else 0), "flops": 8 * n}
    return {"bytes": n * (SIZE[case["dtype"]] + 2 * SIZE[case["grad_dtype"]]) + 16 * c + stats, "flops": 14 * n}


def _visible(case, q_rows, kv_rows):
    """1 where a query sees a key, of one sequence."""
    m = torch.zeros(case["q_len"], case["kv_len"], dtype=torch.float64, device="cuda")
    m[:q_rows, :kv_rows] = 1.0
    if case["causal"] and q_rows:
        m[:q_rows] = torch.tril(m[:q_rows], diagonal=kv_rows - q_rows)
    return m


def _exact_attention(case, d):
    """One sequence and one head of the keys at a time: out and lse, or the three gradients."""
    grad = case["op"] == "attention_grad"
    b, h, hk, nq = case["batch"], case["heads"], case["kv_heads"], case["q_len"]
    times = h // hk
    zeros = lambda t: torch.zeros(t.shape, dtype=torch.float64, device="cuda")
    out, lse = zeros(d["q"]), torch.full((b, h, nq), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = (zeros(d[n]) for n in "qkv")
    rows = _lengths(case) if case["ragged"] else ([nq] * b, [case["kv_len"]] * b)
    masks = {}
    for i in range(b):
        key = (rows[0][i], rows[1][i])
        if key not in masks:
            masks = {key: _visible(case, *key)}
        m = masks[key]
        seen = m.any(1)
        for j in range(h):
            q, k, v = d["q"][i, :, j].double(), d["k"][i, :, j // times].double(), d["v"][i, :, j // times].double()
            x = torch.mm(q, k.t()).mul_(_scale(case))
            if not grad:
                x.masked_fill_(m == 0, -math.inf)
                l = torch.logsumexp(x, 1)
                lse[i, j] = l
                out[i, :, j] = torch.mm(torch.exp(x - torch.where(seen, l, 0.0)[:, None]), v)
                continue
            l = d["lse"][i, j].double()
            p = torch.exp(x - torch.where(seen, l, 0.0)[:, None]).mul_(m)
            do = d["dout"][i, :, j].double()
            delta = torch.einsum("nd,nd->n", do, d["out"][i, :, j].double())
            dv[i, :, j // times] += torch.mm(p.t(), do)
            p.mul_(torch.mm(do, v.t()).sub_(delta[:, None])).mul_(_scale(case))
            dq[i, :, j] = torch.mm(p, k)
            dk[i, :, j // times] += torch.mm(p.t(), q)
    return {"dq": dq, "dk": dk, "dv": dv} if grad else {"out": out, "lse": lse}


def _scale(case):
    return 1.0 / math.sqrt(case["head_dim"])


def _exact_bits(n, seed, offset):
    """The generator's definition on the host, in unsigned numbers."""
    m = np.uint64(0xFFFFFFFF)
    i = np.arange(-(-n // 8), dtype=np.uint64)
    offset = offset % (1 << 64)
    x = [i & m, i >> np.uint64(32), np.full_like(i, offset % (1 << 32)), np.full_like(i, offset // (1 << 32))]
    key = [seed % (1 << 32), seed // (1 << 32) % (1 << 32)]
    for r in range(10):
        k0, k1 = (np.uint64((key[0] + r * 0x9E3779B9) % (1 << 32)), np.uint64((key[1] + r * 0xBB67AE85) % (1 << 32)))
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(q >> np.uint64(32)) ^ x[1] ^ k0, q & m, (p >> np.uint64(32)) ^ x[3] ^ k1, p & m]
    words = np.stack(x, 1).astype(np.uint32)
    return words.view(np.uint16).reshape(-1)[:n]   # (the lower half of a word first)


def exact(case, seed):
    d = _data(case, seed)
    op = case["op"]
    if op in ("attention", "attention_grad"):
        return _exact_attention(case, d)
    if op == "dropout":
        t = math.floor(case["p"] * 65536 + 0.5)
        keep = torch.from_numpy((_exact_bits(case["n"], d["seed"], d["offset"]) >= t).astype(np.float64)).cuda()
        y = d["x"].double() * keep * (65536.0 / max(65536 - t, 1))
        return {"y": y if d["residual"] is None else y + d["residual"].double()}
    b, p, c, n = case["batch"], case["positions"], case["channels"], case["groups"]
    x, gamma, beta = d["x"].double().view(b, p, n, c // n), d["gamma"].double().view(n, -1), d["beta"].double().view(n, -1)
    if op == "group_norm":
        var, mean = torch.var_mean(x, (1, 3), correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
    else:
        mean, rstd = d["stats"].double()
    xh = torch.einsum("bpnc,bn->bpnc", x - mean[:, None, :, None], rstd)
    z = torch.addcmul(beta, xh, gamma)
    act = case["act"]
    if op == "group_norm":
        y = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, torch.zeros_like(z)), "silu": lambda: z * torch.sigmoid(z),
             "gelu": lambda: 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))}[act]()
        return {"y": y.view(b, p, c), "stats": torch.stack([mean, rstd]) if case["stats"] else None}
    dz = d["dy"].double().view_as(z)
    if act == "relu":
        dz = torch.where(z > 0, dz, torch.zeros_like(dz))
    elif act == "gelu":
        dz = dz * (0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
    elif act == "silu":
        dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
    g = dz * gamma
    m = p * (c // n)
    c1, c2 = torch.einsum("bpnc->bn", g) / m, torch.einsum("bpnc,bpnc->bn", g, xh) / m
    dx = torch.einsum("bpnc,bn->bpnc", g - c1[:, None, :, None] - xh * c2[:, None, :, None], rstd)
    return {"dx": dx.reshape(b, p, c), "dgamma": torch.einsum("bpnc,bpnc->nc", dz, xh).reshape(-1),
            "dbeta": torch.einsum("bpnc->nc", dz).reshape(-1)}
