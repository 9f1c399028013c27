"""Cases for the operators around a block-sparse MLP: the product with bias, activation and residual in its epilogue, the
gradient of those epilogues, and the norms before and after a block with its gate and residual, forward and backward.

Every case is a dict of plain values.  `op` says which operator:
  linear     Y = act(W X + bias) + residual, W a pruned rows x cols matrix in b x b blocks; `pre`: W X + bias is kept too
  act_grad   dZ = dY act'(Z) and its column sums; `gated`: dG, dU and H = act(G) U from dH instead
  norm       h' = h + scale * gate * post(y), x = norm(h'); `post`: y goes through a norm of its own first
  norm_grad  the gradient of `norm` with respect to h, y, the gate and the weights
Token-major activations throughout; `serve`: the program repeats the call on kept buffers, as a decoding loop does.
"""
import math

import numpy as np
import torch

own = False

# (hidden, inter, b) of the repository's layers: the 1B-, 8B- and 405B-class MLPs and the GPT2-XL block
SHAPE = {"1b": (2048, 8192, 64), "8b": (4096, 14336, 128), "405b": (16384, 53248, 128), "gpt2xl": (1600, 6400, 64)}
W_STD = 0.02
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "none": None}


def _linear(rows, cols, b, sparsity, tokens, act, bias, residual, out, pre=False, serve=False):
    return {"op": "linear", "rows": rows, "cols": cols, "b": b, "sparsity": sparsity, "tokens": tokens, "act": act,
            "bias": bias, "residual": residual, "out": out, "pre": pre, "serve": serve}


def _act_grad(width, tokens, act, gated, bias, dy):
    return {"op": "act_grad", "width": width, "tokens": tokens, "act": act, "gated": gated, "bias": bias, "dy": dy}


def _norm(op, width, tokens, kind, h, y, params, post=False, gate="none", scale=1.0, serve=False):
    c = {"op": op, "width": width, "tokens": tokens, "kind": kind, "h": h, "y": y, "params": params, "post": post,
         "gate": gate, "scale": scale}
    return dict(c, serve=serve) if op == "norm" else c


def listed():
    gpt, one, eight, big = SHAPE["gpt2xl"], SHAPE["1b"], SHAPE["8b"], SHAPE["405b"]
    named = [
        # one decoded token through the first projection of a GELU block with biases: the smallest product
        ("linear_gpt2xl_up_t1", _linear(gpt[1], gpt[0], 64, 0.80, 1, "gelu", True, "none", "bf16", serve=True)),
        # a short prompt, or a chunk of one, through that block's second projection and onto the residual stream
        ("linear_gpt2xl_down_t333", _linear(gpt[0], gpt[1], 64, 0.80, 333, "none", True, "bf16", "bf16")),
        # a prompt through a small model's down projection, added to a residual stream kept in 32 bits
        ("linear_1b_down_t2048", _linear(one[0], one[1], 64, 0.90, 2048, "none", False, "f32", "f32")),
        # forward pass of a training step: the widest projection, what its gradient needs kept beside the result
        ("linear_8b_up_t4096", _linear(eight[1], eight[0], 128, 0.95, 4096, "silu", True, "none", "bf16", pre=True)),
        # a few sequences of a fine-tuning step: through the GELU, with the gradient of the bias
        ("act_grad_gpt2xl_t333", _act_grad(gpt[1], 333, "gelu", False, True, "bf16")),
        # a training step of the widest gated layer: both gradients, and the intermediate made again
        ("act_grad_8b_gated_t4096", _act_grad(eight[1], 4096, "silu", True, False, "f32")),
        # one decoded token: the residual add and the norm before the next block
        ("norm_8b_t1", _norm("norm", eight[0], 1, "rms", "bf16", "f32", "bf16", serve=True)),
        # a short prompt through a block with layer norms and biases
        ("norm_gpt2xl_t333", _norm("norm", gpt[0], 333, "layer", "bf16", "bf16", "f32")),
        # a prompt through a block normalised on both sides, with a learned gate, the stream kept in 32 bits
        ("norm_1b_sandwich_t2048", _norm("norm", one[0], 2048, "rms", "f32", "bf16", "bf16", True, "vector", 0.5)),
        # a fine-tuning step on a few sequences
        ("norm_grad_gpt2xl_t333", _norm("norm_grad", gpt[0], 333, "layer", "bf16", "bf16", "f32")),
        # a training step of a small model, normalised on both sides with a learned gate
        ("norm_grad_1b_sandwich_t2048", _norm("norm_grad", one[0], 2048, "rms", "f32", "bf16", "bf16", True, "vector", 0.5)),
        # a training step of the widest model, the gate computed per token
        ("norm_grad_405b_gated_t2048", _norm("norm_grad", big[0], 2048, "rms", "bf16", "bf16", "bf16", True, "tokens")),
    ]
    return [dict(c, name=n) for n, c in named]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "act_grad", "norm", "norm_grad"])
    tokens = _log_int(rng, 1, 4096)
    if op == "linear":
        b = rng.choice([16, 32, 64, 64, 128, 128])
        rows, cols = (b * max(4, _log_int(rng, 1024, 14336) // b) for _ in range(2))
        while rows * cols > 14336 * 4096:
            rows, cols = (max(1024, v // 2 // b * b) for v in (rows, cols))
        act = rng.choice(["none", "silu", "gelu", "relu"])
        out = rng.choice(["f32", "bf16"])
        return _linear(rows, cols, b, rng.choice([0.70, 0.80, 0.90, 0.95]) if b >= 32 else rng.choice([0.90, 0.95]),
                       tokens if rows * cols * tokens <= 1024 * 8192 * 4096 else min(tokens, 1024), act, rng.random() < 0.7,
                       rng.choice(["none", "bf16", "f32"]), out, act != "none" and rng.random() < 0.4, tokens <= 16)
    width = 16 * _log_int(rng, 32, 1024)
    if op == "act_grad":
        act = rng.choice(["silu", "gelu", "relu"])
        return _act_grad(width, tokens, act, rng.random() < 0.5, rng.random() < 0.5, rng.choice(["f32", "bf16"]))
    y = rng.choice(["bf16", "bf16", "f32", "none"])
    post = y != "none" and rng.random() < 0.5
    gate = rng.choice(["none", "vector", "tokens"]) if y != "none" else "none"
    return _norm(op, width, tokens if width * tokens <= 2048 * 16384 else 2048, rng.choice(["rms", "layer"]),
                 rng.choice(["f32", "bf16"]), y, rng.choice(["f32", "bf16"]), post, gate,
                 rng.choice([1.0, 0.5, 0.22]) if y != "none" else 1.0, tokens <= 16)


# ---- inputs --------------------------------------------------------------------------------------------------------

def _gauss(gen, shape, std, dtype, mean=0.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std).add_(mean).to(dtype)


def _kept(n, sparsity):
    return n - (int(round(sparsity * 10000)) * n + 9999) // 10000


def _block_mask(case, seed):
    """A seeded permutation of the blocks keeps the share that the sparsity leaves."""
    shape = (case["rows"] // case["b"], case["cols"] // case["b"])
    mask = np.zeros(shape[0] * shape[1], dtype=np.uint8)
    mask[np.random.default_rng(seed).permutation(mask.size)[:_kept(mask.size, case["sparsity"])]] = 1
    return torch.from_numpy(mask.reshape(shape)).cuda()


def _linear_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols, b, t = case["rows"], case["cols"], case["b"], case["tokens"]
    mask = _block_mask(case, seed)
    w = _gauss(gen, (rows, cols), W_STD, torch.bfloat16)
    w = w.view(rows // b, b, cols // b, b).mul_(mask[:, None, :, None]).view(rows, cols)
    x = _gauss(gen, (t, cols), 1.0, torch.bfloat16)
    bias = _gauss(gen, (rows,), 0.1, torch.float32) if case["bias"] else None
    r = TYPES[case["residual"]]
    return {"w": w, "x": x, "bias": bias, "residual": None if r is None else _gauss(gen, (t, rows), 1.0, r)}, mask


def _act_grad_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    shape = (case["tokens"], case["width"])
    return {"z": _gauss(gen, shape, 1.0, torch.bfloat16),
            "u": _gauss(gen, shape, 1.0, torch.bfloat16) if case["gated"] else None,
            "dy": _gauss(gen, shape, 0.1, TYPES[case["dy"]])}


def _norm_inputs(case, seed):
    """A residual stream with a few strong features, as trained ones have."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, e, p = case["tokens"], case["width"], TYPES[case["params"]]
    strong = torch.where(torch.rand((e,), generator=gen, device="cuda") < 0.01, 8.0, 1.0)
    st = {"h": (_gauss(gen, (t, e), 1.0, torch.float32, 0.1) * strong).to(TYPES[case["h"]])}
    y = TYPES[case["y"]]
    st["y"] = None if y is None else _gauss(gen, (t, e), 0.7, y, 0.05)
    layer = case["kind"] == "layer"
    st["weight"] = _gauss(gen, (e,), 0.2, p, 1.0)
    st["bias"] = _gauss(gen, (e,), 0.1, p) if layer else None
    st["post_weight"] = _gauss(gen, (e,), 0.2, p, 1.0) if case["post"] else None
    st["post_bias"] = _gauss(gen, (e,), 0.1, p) if case["post"] and layer else None
    st["gate"] = {"none": None, "vector": (e,), "tokens": (t, e)}[case["gate"]]
    if st["gate"] is not None:
        st["gate"] = _gauss(gen, st["gate"], 0.3, p, 0.5)
    if case["op"] == "norm_grad":
        st["dx"] = _gauss(gen, (t, e), 0.1, torch.bfloat16)
        st["dh"] = _gauss(gen, (t, e), 0.1, st["h"].dtype)
    return st


def prepare(case, seed):
    if case["op"] == "linear":
        st, mask = _linear_inputs(case, seed)
    else:
        st, mask = (_act_grad_inputs if case["op"] == "act_grad" else _norm_inputs)(case, seed), None
    st["case"] = case
    if case["op"] == "norm_grad":  # the forward pass' statistics, which a training program keeps
        st["stats"] = _stats(st["h"].float(), None if not case["post"] else st["y"].float(), case["kind"])
    if own:
        from paper_2507_03117_amd import api

        if case["op"] == "linear":
            st["packed"] = api.bsr_pack(st["w"], case["b"], mask=mask)
        if case.get("serve"):
            shape = (case["tokens"], case["rows"] if case["op"] == "linear" else case["width"])
            if case["op"] == "linear":
                y = torch.empty(shape, dtype=TYPES[case["out"]], device="cuda")
                z = torch.empty(shape, dtype=torch.bfloat16, device="cuda") if case["pre"] else None
                st["kept"] = {"y": y, "z": z} if case["pre"] else {"y": y}
                st["call"] = api.prepare_bsr_linear(st["packed"], st["x"], y, bias=st["bias"], act=_act(case),
                                                    residual=st["residual"], pre=z)
            else:
                h = st["h"] if st["y"] is None else torch.empty_like(st["h"])
                x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
                stats = torch.empty((case["tokens"], 4), dtype=torch.float32, device="cuda")
                st["kept"] = {"h": h, "x": x, "stats": stats}
                st["call"] = api.prepare_norm_residual(st["h"], st["y"], h, x, stats=stats, **_norm_args(st))
    return st


def _act(case):
    return None if case["act"] == "none" else case["act"]


def _norm_args(st):
    c = st["case"]
    return {"kind": c["kind"], "weight": st["weight"], "bias": st["bias"], "post": c["post"], "post_weight": st["post_weight"],
            "post_bias": st["post_bias"], "gate": st["gate"], "scale": c["scale"], "eps": EPS}


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(st):
    if own:
        return _run_own(st)
    return {"linear": _plain_linear, "act_grad": _plain_act_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad}[st["case"]["op"]](st)


def _run_own(st):
    from paper_2507_03117_amd import api

    c = st["case"]
    if "call" in st:
        st["call"]()
        return st["kept"]
    if c["op"] == "linear":
        z = torch.empty((c["tokens"], c["rows"]), dtype=torch.bfloat16, device="cuda") if c["pre"] else None
        y = api.bsr_linear(st["packed"], st["x"], bias=st["bias"], act=_act(c), residual=st["residual"],
                           out_dtype=TYPES[c["out"]], pre=z)
        return {"y": y, "z": z} if c["pre"] else {"y": y}
    if c["op"] == "act_grad":
        if c["gated"]:
            g = api.gated_act_backward(st["z"], st["u"], st["dy"], act=c["act"], bias_grad=c["bias"])
            return {"dg": g.dG, "du": g.dU, "h": g.H, **({"dbg": g.dbias_g, "dbu": g.dbias_u} if c["bias"] else {})}
        g = api.act_backward(st["z"], st["dy"], act=c["act"], bias_grad=c["bias"])
        return {"dz": g.dZ, **({"db": g.dbias} if c["bias"] else {})}
    if c["op"] == "norm":
        h, x, stats = api.norm_residual(st["h"], st["y"], with_stats=True, **_norm_args(st))
        return {"h": h, "x": x, "stats": stats}
    g = api.norm_residual_backward(st["h"], st["y"], st["stats"], st["dx"], st["dh"], **_norm_args(st))
    out = {"dh": g.dh, "dy": g.dy, "dgate": g.dgate, "dweight": g.dweight, "dbias": g.dbias,
           "dpost_weight": g.dpost_weight, "dpost_bias": g.dpost_bias}
    return {k: v for k, v in out.items() if v is not None}


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _plain_act(name, z):
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return torch.clamp_min(z, 0) if name == "relu" else z


def _plain_slope(name, z):
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return (z > 0).to(z.dtype)


def _plain_linear(st):
    c = st["case"]
    z = st["x"].float() @ st["w"].float().t()
    if st["bias"] is not None:
        z = z + st["bias"].float()
    y = _plain_act(c["act"], z)
    if st["residual"] is not None:
        y = y + st["residual"].float()
    y = y.to(TYPES[c["out"]])
    return {"y": y, "z": z.to(torch.bfloat16)} if c["pre"] else {"y": y}


def _plain_act_grad(st):
    c = st["case"]
    z, dy = st["z"].float(), st["dy"].float()
    low = torch.bfloat16
    if not c["gated"]:
        dz = dy * _plain_slope(c["act"], z)
        return {"dz": dz.to(low), **({"db": dz.sum(0)} if c["bias"] else {})}
    u, a = st["u"].float(), _plain_act(c["act"], z)
    dg, du = dy * u * _plain_slope(c["act"], z), dy * a
    return {"dg": dg.to(low), "du": du.to(low), "h": (a * u).to(low),
            **({"dbg": dg.sum(0), "dbu": du.sum(0)} if c["bias"] else {})}


def _moments(v, kind):
    """Mean (0 for "rms") and reciprocal deviation of every row."""
    mean = v.mean(1) if kind == "layer" else torch.zeros_like(v[:, 0])
    return mean, ((v - mean[:, None]).square().mean(1) + EPS).rsqrt()


def _stats(h, y, kind):
    """[tokens, 4]: mean and reciprocal deviation of h, then of y (zeros where y has no norm)."""
    s = list(_moments(h, kind))
    s += [torch.zeros_like(s[0])] * 2 if y is None else list(_moments(y, kind))
    return torch.stack(s, 1)


def _affine(n, weight, bias):
    n = n if weight is None else n * weight.float()
    return n if bias is None else n + bias.float()


def _plain_norm(st):
    c = st["case"]
    h, y = st["h"].float(), None
    if st["y"] is not None:
        y = p = st["y"].float()
        if c["post"]:
            mean, r = _moments(y, c["kind"])
            p = _affine((y - mean[:, None]) * r[:, None], st["post_weight"], st["post_bias"])
        if st["gate"] is not None:
            p = p * st["gate"].float()
        h = h + c["scale"] * p
    stats = _stats(h, y if c["post"] else None, c["kind"])
    x = _affine((h - stats[:, :1]) * stats[:, 1:2], st["weight"], st["bias"])
    return {"h": h.to(st["h"].dtype), "x": x.to(torch.bfloat16), "stats": stats}


def _through_norm(dn, n, r, kind):
    """Gradient of the values that a norm was taken of, from that of the normalised ones `n`."""
    d = dn - n * (dn * n).mean(1, keepdim=True)
    return r * (d - dn.mean(1, keepdim=True) if kind == "layer" else d)


def _plain_norm_grad(st):
    c, s = st["case"], st["stats"]
    dx = st["dx"].float()
    n = (st["h"].float() - s[:, :1]) * s[:, 1:2]
    dh = st["dh"].float() + _through_norm(dx * st["weight"].float(), n, s[:, 1:2], c["kind"])
    out = {"dh": dh.to(st["h"].dtype), "dweight": (dx * n).sum(0)}
    if st["bias"] is not None:
        out["dbias"] = dx.sum(0)
    if st["y"] is None:
        return out
    y = p = st["y"].float()
    if c["post"]:
        m = (y - s[:, 2:3]) * s[:, 3:4]
        p = _affine(m, st["post_weight"], st["post_bias"])
    dp = c["scale"] * dh
    if st["gate"] is not None:
        dgate = dp * p
        out["dgate"] = dgate.sum(0) if c["gate"] == "vector" else dgate.to(st["gate"].dtype)
        dp = dp * st["gate"].float()
    dy = dp
    if c["post"]:
        out["dpost_weight"] = (dp * m).sum(0)
        if st["post_bias"] is not None:
            out["dpost_bias"] = dp.sum(0)
        dy = _through_norm(dp * st["post_weight"].float(), m, s[:, 3:4], c["kind"])
    out["dy"] = dy.to(torch.bfloat16)
    return out


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _sigma(v):
    return torch.sigmoid(v)


def _normal(v):
    """Distribution function and density of the standard normal distribution."""
    return 0.5 * torch.erfc(-v / math.sqrt(2.0)), torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)


def _activation(name, v):
    """(act(v), act'(v))."""
    if name == "silu":
        s = _sigma(v)
        return v * s, s + v * s * (1 - s)
    if name == "gelu":
        cdf, pdf = _normal(v)
        return v * cdf, cdf + v * pdf
    if name == "relu":
        on = (v > 0).double()
        return v * on, on
    return v, torch.ones_like(v)


def exact(case, seed):
    if case["op"] == "linear":
        s, _ = _linear_inputs(case, seed)
        v = torch.matmul(s["w"].double(), s["x"].double().t().contiguous()).t()
        v = v + s["bias"].double() if case["bias"] else v
        y = _activation(case["act"], v)[0]
        y = y if s["residual"] is None else s["residual"].double() + y
        return {"y": y, "z": v} if case["pre"] else {"y": y}
    if case["op"] == "act_grad":
        s = _act_grad_inputs(case, seed)
        dy = s["dy"].double()
        a, slope = _activation(case["act"], s["z"].double())
        if not case["gated"]:
            return {"dz": dy * slope, **({"db": (dy * slope).sum(0)} if case["bias"] else {})}
        u = s["u"].double()
        sums = {"dbg": (dy * u * slope).sum(0), "dbu": (dy * a).sum(0)} if case["bias"] else {}
        return {"dg": dy * u * slope, "du": dy * a, "h": a * u, **sums}
    # the norm's gradient by differentiation of its definition, not by the formula
    s = _norm_inputs(case, seed)
    v = {k: t.double().requires_grad_(case["op"] == "norm_grad") for k, t in s.items() if t is not None}

    def normed(t, w, b):
        if case["kind"] == "layer":
            t = t - t.mean(1, keepdim=True)
        r = (t.pow(2).mean(1, keepdim=True) + EPS).pow(-0.5)
        t = t * r if w is None else t * r * v[w]
        return (t if b is None or b not in v else t + v[b]), r

    def mean_of(t):
        return t.mean(1, keepdim=True) if case["kind"] == "layer" else torch.zeros_like(t[:, :1])

    branch, left = None, [torch.zeros((case["tokens"], 1), dtype=torch.float64, device="cuda")] * 2
    if "y" in v:
        branch = v["y"]
        if case["post"]:
            branch, r = normed(v["y"], "post_weight", "post_bias")
            left = [mean_of(v["y"]), r]
        branch = branch * v["gate"] if "gate" in v else branch
    if case["op"] == "norm":
        h = v["h"] if branch is None else v["h"] + case["scale"] * branch
        x, r = normed(h, "weight", "bias")
        return {"h": h, "x": x, "stats": torch.cat([mean_of(h), r] + left, 1)}
    # (the gradients' inputs hold the updated stream: the branch adds what its gradient passes on)
    x, _ = normed(v["h"], "weight", "bias")
    want = [k for k in ("weight", "bias") if k in v]
    first = torch.autograd.grad(x, [v["h"]] + [v[k] for k in want], v["dx"].detach())
    dh = v["dh"].detach() + first[0]
    out = {"dh": dh, **{"d" + k: g for k, g in zip(want, first[1:])}}
    if branch is not None:
        names = ["y"] + [k for k in ("gate", "post_weight", "post_bias") if k in v]
        grads = torch.autograd.grad(branch, [v[k] for k in names], case["scale"] * dh)
        out.update({"d" + k: g for k, g in zip(names, grads)})
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "none": 0}
    t = case["tokens"]
    if case["op"] == "linear":
        b, rows, cols = case["b"], case["rows"], case["cols"]
        kept = _kept((rows // b) * (cols // b), case["sparsity"])
        acts = t * (2 * cols + rows * (size[case["out"]] + size[case["residual"]] + (2 if case["pre"] else 0)))
        return {"bytes": kept * (2 * b * b + 4) + acts + (4 * rows if case["bias"] else 0), "flops": 2.0 * b * b * kept * t}
    n = t * case["width"]
    if case["op"] == "act_grad":
        sums = case["width"] * 4 * (1 + case["gated"]) if case["bias"] else 0
        return {"bytes": n * ((10 if case["gated"] else 4) + size[case["dy"]]) + sums, "flops": n * (24.0 if case["gated"] else 16.0)}
    h, y, p = size[case["h"]], size[case["y"]], size[case["params"]]
    gate = p if case["gate"] == "tokens" else 0
    vectors = case["width"] * (1 + case["post"]) * (1 + (case["kind"] == "layer")) + (case["width"] if case["gate"] == "vector" else 0)
    if case["op"] == "norm":
        moved = h + y + gate + (h if y else 0) + 2
        return {"bytes": n * moved + vectors * p + 16 * t, "flops": n * (16.0 if case["post"] else 8.0)}
    moved = 3 * h + 2 + y + (2 if y else 0) + 2 * gate
    return {"bytes": n * moved + vectors * (p + 4) + 16 * t, "flops": n * (30.0 if case["post"] else 16.0)}
