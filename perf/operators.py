"""The layers around the compressed store, as cases that can be timed and compared: layer norm and
its backward pass, the linear layer with its epilogue and its backward pass, and the global norm
and clipping of a list of gradients.

A case is one call on inputs, outputs and scratch that an adaptation step has in hand.
`listed()` gives the fixed cases, `draw(rng)` one more of the same ranges.  Where `own` is false the
operators are computed in their plain form, elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}
EPS = 1e-6                      # of the layer norms (ViT's and Segformer's)
CLIP_EPS = 1e-6                 # added to the norm before the division


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------

def _norm(name, rows, channels, dtype, affine=True, stats=True):
    return {"name": name, "op": "norm", "rows": rows, "channels": channels, "dtype": dtype, "affine": affine,
            "stats": stats}


def _norm_grad(name, rows, channels, dtype, grad_dtype, residual=True):
    return {"name": name, "op": "norm_grad", "rows": rows, "channels": channels, "dtype": dtype,
            "grad_dtype": grad_dtype, "residual": residual}


def _clip(name, sizes, dtype, relative, align):
    return {"name": name, "op": "clip", "sizes": sizes, "dtype": dtype, "relative": relative, "align": align}


def _linear(name, rows, c_in, c_out, act, bias=True, residual=False, keep=False, out="bf16"):
    return {"name": name, "op": "linear", "rows": rows, "c_in": c_in, "c_out": c_out, "act": act, "bias": bias,
            "residual": residual, "keep": keep, "out": out}


def _linear_grad(name, rows, c_in, c_out, act):
    return {"name": name, "op": "linear_grad", "rows": rows, "c_in": c_in, "c_out": c_out, "act": act}


def listed():
    return [
        # the class token of one image before the classifier: latency alone
        _norm("norm one token", 1, 768, "bf16", stats=False),
        # a ViT-B block's norm at the benchmark's batch (64 images of 197 tokens), statistics kept for the backward pass
        _norm("norm vit", 12608, 768, "bf16"),
        # fp32 features of an odd width (rows start at no 16-byte boundary)
        _norm("norm odd and wide", 1009, 5003, "fp32"),
        # the backward pass of the ViT-B norm: bf16 activations, fp32 gradients as the weight gradients take them,
        # the gradient of the skip connection added on the way
        _norm_grad("norm grad vit", 12608, 768, "bf16", "fp32"),
        # Segformer-B5's first stage on one 1024x1024 image: many short rows, gradients in bf16
        _norm_grad("norm grad segformer stage 1", 65536, 64, "bf16", "bf16"),
        # the norm layers' parameters alone, adapted as in "SURGEON (BN)": ResNet-50's 106 short tensors
        _clip("clip norm layers", "resnet50_bn", "fp32", 0.5, 128),
        # every weight and bias of ViT-B: 86 million fp32 gradients
        _clip("clip vit", "vit", "fp32", 0.3, 128),
        # the classifier on one image: a single row, fp32 logits
        _linear("linear classifier of one image", 1, 2048, 1000, "none", out="fp32"),
        # Segformer's MLP in its second stage, the pre-activation kept for the backward pass
        _linear("linear segformer stage 2 mlp", 16384, 128, 512, "gelu", keep=True),
        # a wide layer with its skip connection: the matrix product is the whole of it
        _linear("linear wide with residual", 16384, 2048, 2048, "none", residual=True),
        # the input gradient of ViT-B's qkv layer
        _linear_grad("linear grad vit qkv", 12608, 768, 2304, "none"),
        # Segformer's third-stage MLP on an image that fills no whole tile
        _linear_grad("linear grad segformer stage 3 mlp", 4037, 320, 1280, "gelu"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A channel count: often a multiple of 64 or 8, else any number."""
    c = _log_int(rng, lo, hi)
    step = rng.choice([64, 64, 8, 1])
    return max(step, c // step * step)


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "clip", "linear", "linear_grad"])
    if op in ("norm", "norm_grad"):
        channels = _width(rng, 8, 8192)
        rows = _log_int(rng, 1, max(1, min(65536, (1 << 24) // channels)))
        dtype = rng.choice(["bf16", "fp32"])
        if op == "norm":
            case = _norm("", rows, channels, dtype, affine=rng.random() < 0.8, stats=rng.random() < 0.7)
        else:
            case = _norm_grad("", rows, channels, dtype, rng.choice(["bf16", "fp32"]) if dtype == "bf16" else "fp32",
                              residual=rng.random() < 0.5)
    elif op == "clip":
        sizes, total = [], 0
        for _ in range(_log_int(rng, 1, 200)):
            n = _log_int(rng, 1, 4_000_000)
            if total + n <= 80_000_000:
                sizes.append(n)
                total += n
        case = _clip("", " ".join(str(n) for n in sizes), rng.choice(["fp32", "fp32", "bf16"]),
                     rng.choice([0.01, 0.5, 0.9, 2.0]), rng.choice([1, 128]))
    else:
        c_in, c_out = _width(rng, 16, 4096), _width(rng, 16, 4096)
        rows = _log_int(rng, 1, max(1, min(65536, int(6e10 / (2.0 * c_in * c_out)))))
        act = rng.choice(["none", "relu", "gelu"])
        if op == "linear":
            case = _linear("", rows, c_in, c_out, act, bias=rng.random() < 0.8, residual=rng.random() < 0.5,
                           keep=act != "none" and rng.random() < 0.5, out=rng.choice(["bf16", "bf16", "fp32"]))
        else:
            case = _linear_grad("", rows, c_in, c_out, act)
    del case["name"]
    return case


def _sizes(case):
    """Element counts of a list of gradients."""
    if case["sizes"] == "resnet50_bn":
        widths = [64]
        for s, blocks in enumerate((3, 4, 6, 3)):
            w = 64 << s
            for b in range(blocks):
                widths += [w, w, 4 * w] + ([4 * w] if b == 0 else [])
        return [w for w in widths for _ in range(2)]
    if case["sizes"] == "vit":
        d = 768
        block = [d, d, 3 * d * d, 3 * d, d * d, d, d, d, 4 * d * d, 4 * d, 4 * d * d, d]
        return [d, 197 * d, d * 3 * 16 * 16, d] + 12 * block + [d, d, 1000 * d, 1000]
    return [int(n) for n in case["sizes"].split()]


def _places(case):
    """Where each gradient starts in the flat buffer, and the buffer's length (`align`: elements)."""
    at, places = 0, []
    for n in _sizes(case):
        places.append(at)
        at += -(-n // case["align"]) * case["align"]
    return places, at


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _data(case, seed):
    """The tensors that the call reads, from the seed alone."""
    g = _gen(seed)
    if case["op"] in ("norm", "norm_grad"):
        t, c, dt = case["rows"], case["channels"], TYPES[case["dtype"]]
        # a residual stream: its own spread and offset per channel
        x = (_randn(g, t, c) * (0.5 + torch.rand(c, generator=g, device="cuda")) + _randn(g, c, scale=0.3)).to(dt)
        d = {"x": x, "gamma": 1.0 + _randn(g, c, scale=0.2), "beta": _randn(g, c, scale=0.2)}
        if case["op"] == "norm_grad":
            gt = TYPES[case["grad_dtype"]]
            d["dy"] = _randn(g, t, c, scale=0.01, dtype=gt)
            d["skip"] = _randn(g, t, c, scale=0.01, dtype=gt) if case["residual"] else None
            f = x.double()
            mean = f.mean(1)
            d["stats"] = torch.stack([mean, (f.var(1, unbiased=False) + EPS).rsqrt()]).float()
        elif not case["affine"]:
            d["gamma"] = d["beta"] = None
        return d
    if case["op"] == "clip":
        places, length = _places(case)
        flat = torch.zeros(length, dtype=TYPES[case["dtype"]], device="cuda")
        grads = [flat[a:a + n] for a, n in zip(places, _sizes(case))]
        total = 0.0
        for v in grads:
            sigma = 10.0 ** (-4.0 + 2.0 * torch.rand(1, generator=g, device="cuda").item())
            v.copy_(_randn(g, v.numel(), scale=sigma))
            total += sigma * sigma * v.numel()
        return {"grads": grads, "max_norm": case["relative"] * math.sqrt(total)}
    t, ci, co = case["rows"], case["c_in"], case["c_out"]
    w = _randn(g, co, ci, scale=ci ** -0.5, dtype=torch.bfloat16)
    if case["op"] == "linear":
        return {"w": w, "x": _randn(g, t, ci, dtype=torch.bfloat16),
                "bias": _randn(g, co, scale=0.2) if case["bias"] else None,
                "residual": _randn(g, t, co, dtype=TYPES[case["out"]]) if case["residual"] else None}
    return {"w": w, "dy": _randn(g, t, co, scale=0.01, dtype=torch.bfloat16),
            "pre": _randn(g, t, co, dtype=torch.bfloat16) if case["act"] != "none" else None}


def prepare(case, seed):
    s = {"case": case, **_data(case, seed)}
    op = case["op"]
    if op == "norm":
        s["y"] = torch.empty_like(s["x"])
        s["stats"] = torch.empty(2, case["rows"], device="cuda") if case["stats"] else None
    elif op == "norm_grad":
        s["dx"] = torch.empty_like(s["dy"])
        s["dgamma"], s["dbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
    elif op == "clip":
        places, length = _places(case)
        s["flat"] = torch.zeros(length, dtype=TYPES[case["dtype"]], device="cuda")
        s["outs"] = [s["flat"][a:a + n] for a, n in zip(places, _sizes(case))]
        s["norm"] = torch.empty(1, dtype=torch.float64, device="cuda")
        s["gi"] = torch.empty(len(s["outs"]), dtype=torch.float64, device="cuda")
    elif op == "linear":
        s["y"] = torch.empty(case["rows"], case["c_out"], dtype=TYPES[case["out"]], device="cuda")
        s["pre"] = torch.empty(case["rows"], case["c_out"], dtype=torch.bfloat16, device="cuda") if case["keep"] else None
    else:
        s["dx"] = torch.empty(case["rows"], case["c_in"], dtype=torch.bfloat16, device="cuda")
        s["dz"] = torch.empty(case["rows"], case["c_out"], device="cuda")
        s["dbias"] = torch.empty(case["c_out"], device="cuda")
    if own:                                       # the handles and the scratch that a program makes once
        from paper_2503_20354_b200 import binding as B
        need = 0
        if op == "norm_grad":
            need = B.surgeon_layer_norm_grad_workspace(case["rows"], case["channels"])
        elif op == "clip":
            s["list"] = B.GradientList(s["grads"], s["outs"])
            need = B.surgeon_gradient_norm_workspace(s["list"])
        elif op == "linear":
            s["desc"] = B.linear_desc(case["rows"], case["c_in"], case["c_out"])
            need = B.surgeon_linear_workspace(s["desc"])
        elif op == "linear_grad":
            s["desc"] = B.linear_desc(case["rows"], case["c_in"], case["c_out"])
            need = B.surgeon_linear_grad_workspace(s["desc"])
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
    if op == "norm":
        B.surgeon_layer_norm(s["x"], s["gamma"], s["beta"], EPS, out=s["y"], stats=s["stats"])
        return {"y": s["y"], "stats": s["stats"]}
    if op == "norm_grad":
        B.surgeon_layer_norm_grad(s["x"], s["dy"], s["gamma"], s["stats"], residual_grad=s["skip"], dx=s["dx"],
                                  dgamma=s["dgamma"], dbeta=s["dbeta"], workspace=s["scratch"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if op == "clip":
        B.surgeon_clip_gradients(s["list"], s["max_norm"], norm=s["norm"], gi=s["gi"], workspace=s["scratch"])
        return {"grads": s["flat"], "norm": s["norm"], "gi": s["gi"]}
    act = {"none": B.SURGEON_ACT_NONE, "relu": B.SURGEON_ACT_RELU, "gelu": B.SURGEON_ACT_GELU}[case["act"]]
    if op == "linear":
        B.surgeon_linear(s["desc"], s["x"], s["w"], bias=s["bias"], act=act, residual=s["residual"], out=s["y"],
                         pre=s["pre"], workspace=s["scratch"])
        return {"y": s["y"], "pre": s["pre"]}
    B.surgeon_linear_grad(s["desc"], s["dy"], s["w"], pre=s["pre"], act=act, dx=s["dx"], dz=s["dz"],
                          dbias=s["dbias"], workspace=s["scratch"])
    return {"dx": s["dx"], "dz": s["dz"], "dbias": s["dbias"]}


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    y = c * rstd
    if s["gamma"] is not None:
        y = y * s["gamma"] + s["beta"]
    return {"y": y.to(s["x"].dtype), "stats": torch.cat([mean, rstd], 1).t().contiguous() if s["stats"] is not None else None}


def _plain_norm_grad(s):
    mean, rstd = s["stats"][0][:, None], s["stats"][1][:, None]
    xh, dy = (s["x"].float() - mean) * rstd, s["dy"].float()
    g = dy * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if s["skip"] is not None:
        dx = dx + s["skip"].float()
    return {"dx": dx.to(s["dy"].dtype), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def _plain_clip(s):
    squares = torch.stack([v.double().square().sum() for v in s["grads"]])
    norm = squares.sum().sqrt().reshape(1)
    coef = torch.clamp(s["max_norm"] / (norm + CLIP_EPS), max=1.0).float()
    lengths = torch.tensor([v.numel() for v in s["grads"]], dtype=torch.float64)
    torch._foreach_copy_(s["outs"], [(v.float() * coef).to(v.dtype) for v in s["grads"]])
    return {"grads": s["flat"], "norm": norm, "gi": (squares / lengths.to(squares.device, non_blocking=True)).sqrt()}


def _plain_act(z, act):
    return z if act == "none" else torch.clamp(z, min=0.0) if act == "relu" else 0.5 * z * (1.0 + torch.erf(z * 2.0 ** -0.5))


def _plain_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    return 0.5 * (1.0 + torch.erf(z * 2.0 ** -0.5)) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5


def _plain_linear(s):
    z = s["x"].float() @ s["w"].float().t()
    if s["bias"] is not None:
        z = z + s["bias"]
    y = _plain_act(z, s["case"]["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(s["y"].dtype), "pre": z.to(torch.bfloat16) if s["pre"] is not None else None}


def _plain_linear_grad(s):
    dz = s["dy"].float()
    if s["pre"] is not None:
        dz = dz * _plain_slope(s["pre"].float(), s["case"]["act"])
    return {"dx": (dz @ s["w"].float()).to(torch.bfloat16), "dz": dz, "dbias": dz.sum(0)}


_PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "clip": _plain_clip, "linear": _plain_linear,
          "linear_grad": _plain_linear_grad}


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without, and what it returns in 64 bits
# ---------------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "norm":
        n, c = case["rows"] * case["channels"], case["channels"]
        return {"bytes": 2 * n * SIZE[case["dtype"]] + (8 * c if case["affine"] else 0) +
                (8 * case["rows"] if case["stats"] else 0), "flops": 8 * n}
    if op == "norm_grad":
        n, c = case["rows"] * case["channels"], case["channels"]
        return {"bytes": n * (SIZE[case["dtype"]] + (3 if case["residual"] else 2) * SIZE[case["grad_dtype"]]) +
                12 * c + 8 * case["rows"], "flops": 14 * n}
    if op == "clip":
        n = sum(_sizes(case))
        return {"bytes": 2 * n * SIZE[case["dtype"]] + 8 * (len(_sizes(case)) + 1), "flops": 3 * n}
    t, ci, co = case["rows"], case["c_in"], case["c_out"]
    flops = 2.0 * t * ci * co
    if op == "linear":
        return {"bytes": 2 * (t * ci + ci * co) + (4 * co if case["bias"] else 0) + 2 * t * co * case["keep"] +
                (2 if case["residual"] else 1) * t * co * SIZE[case["out"]], "flops": flops + 4 * t * co}
    return {"bytes": 2 * (t * ci + ci * co) + (8 if case["act"] != "none" else 6) * t * co + 4 * co,
            "flops": flops + 4 * t * co}


def exact(case, seed):
    d = {k: ([t.double() for t in v] if isinstance(v, list) else v.double() if isinstance(v, torch.Tensor) else v)
         for k, v in _data(case, seed).items()}
    op = case["op"]
    if op == "norm":
        var, mean = torch.var_mean(d["x"], 1, correction=0)
        sd = torch.sqrt(var + EPS)
        y = (d["x"] - mean[:, None]) / sd[:, None]
        if case["affine"]:
            y = torch.addcmul(d["beta"], y, d["gamma"])
        return {"y": y, "stats": torch.stack([mean, 1.0 / sd]) if case["stats"] else None}
    if op == "norm_grad":
        mean, rstd = d["stats"]
        xh = torch.einsum("tc,t->tc", d["x"] - mean[:, None], rstd)
        g = torch.einsum("tc,c->tc", d["dy"], d["gamma"])
        along = torch.einsum("tc,tc->t", g, xh) / case["channels"]
        dx = torch.einsum("tc,t->tc", g - g.sum(1, keepdim=True) / case["channels"] - xh * along[:, None], rstd)
        return {"dx": dx if d["skip"] is None else dx + d["skip"], "dgamma": torch.einsum("tc,tc->c", d["dy"], xh),
                "dbeta": torch.einsum("tc->c", d["dy"])}
    if op == "clip":
        total = [torch.dot(v, v) for v in d["grads"]]
        norm = torch.sqrt(sum(total))
        coef = min(1.0, d["max_norm"] / (norm.item() + CLIP_EPS))
        places, length = _places(case)
        flat = torch.zeros(length, dtype=torch.float64, device="cuda")
        for a, v in zip(places, d["grads"]):
            flat[a:a + v.numel()] = v * coef
        return {"grads": flat, "norm": norm.reshape(1),
                "gi": torch.stack([torch.sqrt(q / v.numel()) for q, v in zip(total, d["grads"])])}
    if op == "linear":
        z = torch.einsum("ti,oi->to", d["x"], d["w"])
        z = z if d["bias"] is None else z + d["bias"][None]
        y = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, torch.zeros_like(z)),
             "gelu": lambda: 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))}[case["act"]]()
        return {"y": y if d["residual"] is None else y + d["residual"], "pre": z if case["keep"] else None}
    dz = d["dy"]
    if case["act"] == "relu":
        dz = torch.where(d["pre"] > 0, dz, torch.zeros_like(dz))
    elif case["act"] == "gelu":
        p = d["pre"]
        dz = dz * (0.5 * torch.special.erfc(-p / math.sqrt(2.0)) + p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi))
    return {"dx": torch.einsum("to,oi->ti", dz, d["w"]), "dz": dz, "dbias": torch.einsum("to->o", dz)}
