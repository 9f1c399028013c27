"""Cases for the operators on 8-bit floating point with a scale per group: products of block-sparse weights, the gated half of a
feed-forward block, and the backward pass that reads activations kept in that form.

A scaled 8-bit tensor is codes (E4M3 or E5M2) [tokens, features] and scales [groups, tokens], a power of two for each token and
group of 64 or 128 features, held as its biased exponent; a weight has one such scale for each stored block.  The scale is the
smallest power of two, at least 2^-100, by which the group's largest magnitude becomes a value of the format.

Every case is a dict of plain values.  `op` says which operator:
  keep      an activation into that form
  linear    Y = act(W X + bias) + residual, W and X in 8 bits; `out` is the type of Y, `pre`: W X + bias is kept, in 8 bits
  gated     H = act(G) U, G = Wg X, U = Wu X; H in 8 bits (or bf16), `pre`: G and U are kept, in 8 bits
  wgrad     the gradient of the stored blocks, dY X^T, from dY in bf16 and X in 8 bits
  act_grad  dZ = dY act'(Z) and its column sums from Z in 8 bits; `gated`: dG, dU and H = act(G) U
`serve`: the program repeats the call on kept buffers, as a decoding loop does.
"""
import math

import numpy as np
import torch

own = False

# (hidden, inter, b) of the repository's layers: the 1B-, 8B- and 405B-class MLPs and the GPT2-XL block
SHAPE = {"1b": (2048, 8192, 64), "8b": (4096, 14336, 128), "405b": (16384, 53248, 128), "gpt2xl": (1600, 6400, 64)}
W_STD = 0.02
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "none": None}
EIGHT = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
# the largest value of a format is 1.75 * 2^TOP, its smallest normal one 2^LOW, its mantissa has BITS bits
TOP, LOW, BITS = {"e4m3": 8, "e5m2": 15}, {"e4m3": -6, "e5m2": -14}, {"e4m3": 3, "e5m2": 2}
LEAST = -100  # smallest exponent of a scale


def _keep(width, tokens, x, group, fmt, serve=False):
    return {"op": "keep", "width": width, "tokens": tokens, "x": x, "group": group, "fmt": fmt, "serve": serve}


def _linear(rows, cols, b, sparsity, tokens, group, wfmt, xfmt, act, bias, residual, out, pre=False, serve=False):
    return {"op": "linear", "rows": rows, "cols": cols, "b": b, "sparsity": sparsity, "tokens": tokens, "group": group,
            "wfmt": wfmt, "xfmt": xfmt, "act": act, "bias": bias, "residual": residual, "out": out, "pre": pre, "serve": serve}


def _gated(rows, cols, b, sparsity, tokens, group, act, out, pre, serve=False):
    return {"op": "gated", "rows": rows, "cols": cols, "b": b, "sparsity": sparsity, "tokens": tokens, "group": group,
            "wfmt": "e4m3", "xfmt": "e4m3", "act": act, "out": out, "pre": pre, "serve": serve}


def _wgrad(rows, cols, b, sparsity, tokens, group, xfmt):
    return {"op": "wgrad", "rows": rows, "cols": cols, "b": b, "sparsity": sparsity, "tokens": tokens, "group": group, "xfmt": xfmt}


def _act_grad(width, tokens, group, fmt, act, gated, bias, dy):
    return {"op": "act_grad", "width": width, "tokens": tokens, "group": group, "fmt": fmt, "act": act, "gated": gated,
            "bias": bias, "dy": dy}


def listed():
    gpt, one, eight, big = SHAPE["gpt2xl"], SHAPE["1b"], SHAPE["8b"], SHAPE["405b"]
    named = [
        # one decoded token's activation before a product: the smallest call
        ("keep_1b_t1", _keep(one[0], 1, "bf16", 64, "e4m3", serve=True)),
        # a training step's intermediate, kept for the way back
        ("keep_8b_t4096", _keep(eight[1], 4096, "bf16", 128, "e4m3")),
        # one decoded token through a wide projection
        ("linear_8b_up_t1", _linear(eight[1], eight[0], 128, 0.95, 1, 128, "e4m3", "e4m3", "none", False, "none", "bf16", serve=True)),
        # a short prompt, or a chunk of one, through a block's second projection with bias and onto the residual stream
        ("linear_gpt2xl_down_t333", _linear(gpt[0], gpt[1], 64, 0.80, 333, 64, "e4m3", "e4m3", "none", True, "bf16", "bf16")),
        # a prompt through a small model's down projection, added to a residual stream kept in 32 bits
        ("linear_1b_down_t2048", _linear(one[0], one[1], 64, 0.90, 2048, 64, "e4m3", "e4m3", "none", False, "f32", "f32")),
        # backward pass of the widest model: gradients in E5M2 through the transposed down projection
        ("linear_405b_back_t2048", _linear(big[1], big[0], 128, 0.95, 2048, 128, "e4m3", "e5m2", "none", False, "none", "bf16")),
        # a few decoded tokens through the gated half of a small model
        ("gated_1b_t5", _gated(one[1], one[0], 64, 0.90, 5, 64, "silu", "e4m3", False, serve=True)),
        # forward pass of a training step of the gated half, G and U kept
        ("gated_8b_t4096", _gated(eight[1], eight[0], 128, 0.95, 4096, 128, "silu", "e4m3", True)),
        # a few sequences of a fine-tuning step: gradient of the first projection's blocks
        ("wgrad_gpt2xl_t333", _wgrad(gpt[1], gpt[0], 64, 0.80, 333, 64, "e4m3")),
        # a training step: gradient of a wide projection's blocks
        ("wgrad_8b_t4096", _wgrad(eight[1], eight[0], 128, 0.95, 4096, 128, "e4m3")),
        # a fine-tuning step: through the GELU, with the gradient of the bias
        ("act_grad_gpt2xl_t333", _act_grad(gpt[1], 333, 64, "e4m3", "gelu", False, True, "bf16")),
        # a training step of the gated half: both gradients, and the intermediate made again
        ("act_grad_8b_gated_t4096", _act_grad(eight[1], 4096, 128, "e4m3", "silu", True, False, "bf16")),
    ]
    return [dict(c, name=n) for n, c in named]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["keep", "linear", "linear", "gated", "wgrad", "act_grad"])
    tokens = _log_int(rng, 1, 4096)
    fmt = rng.choice(["e4m3", "e4m3", "e5m2"])
    act = rng.choice(["silu", "gelu", "relu"])
    if op in ("keep", "act_grad"):
        width, group = 8 * _log_int(rng, 64, 1792), rng.choice([64, 128])
        if op == "keep":
            return _keep(width, tokens, rng.choice(["bf16", "f32"]), group, fmt, tokens <= 16)
        return _act_grad(width, tokens, group, fmt, act, rng.random() < 0.5, rng.random() < 0.5, rng.choice(["f32", "bf16"]))
    b = rng.choice([64, 128])
    group = 128 if b == 128 else rng.choice([64, 128])
    rows, cols = (b * max(4, _log_int(rng, 1024, 14336) // b) for _ in range(2))
    while rows * cols > 14336 * 4096:
        rows, cols = (max(1024, v // 2 // b * b) for v in (rows, cols))
    sparsity = rng.choice([0.70, 0.80, 0.90, 0.95])
    if op == "wgrad":
        return _wgrad(rows, cols, b, sparsity, tokens, group, fmt)
    if op == "gated":
        return _gated(rows, cols, b, sparsity, tokens, group, act, rng.choice(["e4m3", "e4m3", "bf16"]), rng.random() < 0.5, tokens <= 16)
    act = rng.choice(["none", act])
    return _linear(rows, cols, b, sparsity, tokens, group, rng.choice(["e4m3", "e5m2"]), fmt, act, rng.random() < 0.6,
                   rng.choice(["none", "bf16", "f32"]), rng.choice(["f32", "bf16", "e4m3"]), act != "none" and rng.random() < 0.5,
                   tokens <= 16)


# ---- inputs --------------------------------------------------------------------------------------------------------

def _gauss(gen, shape, std, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _kept(n, sparsity):
    return n - (int(round(sparsity * 10000)) * n + 9999) // 10000


def _block_mask(case, seed):
    """A seeded permutation of the blocks keeps the share that the sparsity leaves."""
    shape = (case["rows"] // case["b"], case["cols"] // case["b"])
    mask = np.zeros(shape[0] * shape[1], dtype=np.uint8)
    mask[np.random.default_rng(seed).permutation(mask.size)[:_kept(mask.size, case["sparsity"])]] = 1
    return torch.from_numpy(mask.reshape(shape)).cuda()


def _exponents(most, fmt):
    """Exponent of the scale of a group whose largest magnitude is `most`: 32-bit integers."""
    fraction, exponent = torch.frexp(most)
    e = torch.clamp_min(exponent - 1 - TOP[fmt] + (fraction > 0.875).to(torch.int32), LEAST)
    return torch.where(most > 0, e, LEAST)


def _power(e):
    """2^e for -126 <= e <= 127, from its bits: torch.ldexp is an ulp off for some exponents on the GPU."""
    return ((e + 127) << 23).view(torch.float32)


def _padded(tokens):
    return (tokens + 15) // 16 * 16


def _quantised(v, group, fmt):
    """fp32 [tokens, features] -> codes, scales [groups, tokens padded to 16]."""
    t, k = v.shape
    n = (k + group - 1) // group
    w = torch.nn.functional.pad(v, (0, n * group - k)).view(t, n, group)
    e = _exponents(w.abs().amax(2), fmt)
    codes = (w * _power(-e)[:, :, None]).view(t, n * group)[:, :k].to(EIGHT[fmt])
    scales = torch.zeros((n, _padded(t)), dtype=torch.uint8, device=v.device)
    scales[:, :t] = (e + 127).to(torch.uint8).t()
    return codes, scales


def _values(codes, scales, group):
    """fp32 values of a scaled 8-bit tensor."""
    t, k = codes.shape
    f = _power(scales[:, :t].to(torch.int32) - 127).t()
    return codes.float() * f.repeat_interleave(group, 1)[:, :k]


def _activation_inputs(gen, shape, std):
    """Activations with a few strong features, as trained networks have them, and tokens of different size."""
    strong = torch.where(torch.rand((shape[1],), generator=gen, device="cuda") < 0.01, 8.0, 1.0)
    size = torch.exp2(_gauss(gen, (shape[0], 1), 1.0))
    return _gauss(gen, shape, std) * strong * size


def _weight(gen, case, seed):
    """Stored blocks of a pruned weight: bf16 values, their codes and scales, and where they lie."""
    b, mask = case["b"], _block_mask(case, seed)
    where = mask.nonzero()
    blocks = _gauss(gen, (where.shape[0], b, b), W_STD, torch.bfloat16)
    v = blocks.float()
    e = _exponents(v.abs().amax((1, 2)), case["wfmt"])
    codes = (v * _power(-e)[:, None, None]).to(EIGHT[case["wfmt"]])
    return {"mask": mask, "where": where, "blocks": blocks, "codes": codes, "scales": (e + 127).to(torch.uint8)}


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, op = case["tokens"], case["op"]
    st = {"case": case}
    if op == "keep":
        st["x"] = _activation_inputs(gen, (t, case["width"]), 1.0).to(TYPES[case["x"]])
        return st
    if op == "act_grad":
        shape = (t, case["width"])
        st["z"] = _quantised(_gauss(gen, shape, 1.0), case["group"], case["fmt"])
        st["u"] = _quantised(_gauss(gen, shape, 1.0), case["group"], case["fmt"]) if case["gated"] else None
        st["dy"] = _gauss(gen, shape, 0.1, TYPES[case["dy"]])
        return st
    st["x"] = _quantised(_activation_inputs(gen, (t, case["cols"]), 1.0), case["group"], case["xfmt"])
    if op == "wgrad":
        st["mask"] = _block_mask(case, seed)
        st["where"] = st["mask"].nonzero()
        st["dy"] = _gauss(gen, (t, case["rows"]), 0.1, torch.bfloat16)
        return st
    st["w"] = _weight(gen, case, seed)
    if op == "gated":
        st["wu"] = _weight(gen, case, seed + (1 << 30))
        return st
    st["bias"] = _gauss(gen, (case["rows"],), 0.1) if case["bias"] else None
    r = TYPES[case["residual"]]
    st["residual"] = None if r is None else _gauss(gen, (t, case["rows"]), 1.0, r)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    for k in ("w", "wu"):
        if k in st and not own:
            del st[k]["blocks"]
    if own:
        _prepare_own(st)
    return st


# ---- the framework's calls -------------------------------------------------------------------------------------------

def _scaled(api, pair, group, fmt):
    codes, scales = pair
    return api.Scaled8(codes.view(torch.uint8), scales, group, fmt)


def _packed(api, case, blocks, where, mask):
    b = case["b"]
    dense = torch.zeros((case["rows"], case["cols"]), dtype=torch.bfloat16, device="cuda")
    if blocks is not None:
        dense.view(case["rows"] // b, b, case["cols"] // b, b).transpose(1, 2)[where[:, 0], where[:, 1]] = blocks
    return api.bsr_pack(dense, b, mask=mask)


def _act(case):
    return None if case["act"] == "none" else case["act"]


def _prepare_own(st):
    from paper_2507_03117_amd import api

    c, op = st["case"], st["case"]["op"]
    if op == "keep":
        if c["serve"]:
            st["kept"] = api.empty_scaled8(c["tokens"], c["width"], group=c["group"], fmt=c["fmt"], device="cuda")
            st["call"] = api.prepare_quantize_scaled8(st["x"], st["kept"])
        return
    if op == "act_grad":
        st["z8"] = _scaled(api, st["z"], c["group"], c["fmt"])
        st["u8"] = _scaled(api, st["u"], c["group"], c["fmt"]) if c["gated"] else None
        return
    st["x8"] = _scaled(api, st["x"], c["group"], c["xfmt"])
    if op == "wgrad":
        st["packed"] = _packed(api, c, None, None, st["mask"])
        return
    for k in ("w", "wu"):
        if k in st:
            w = st[k]
            st[k + "8"] = api.bsr_quantize_scaled8(_packed(api, c, w["blocks"], w["where"], w["mask"]), fmt=c["wfmt"])
            del w["blocks"]
    if c["serve"]:
        t, rows = c["tokens"], c["rows"]

        def eight():
            return api.empty_scaled8(t, rows, group=c["b"], fmt="e4m3", device="cuda")

        out = eight() if c["out"] == "e4m3" else torch.empty((t, rows), dtype=TYPES[c["out"]], device="cuda")
        if op == "gated":
            keep = (eight(), eight()) if c["pre"] else None
            st["call"] = api.prepare_bsr_gated_scaled8(st["w8"], st["wu8"], st["x8"], out, act=c["act"], keep=keep)
            st["kept"] = api.Gated8(out, *(keep or (None, None)))
        else:
            pre = eight() if c["pre"] else None
            st["call"] = api.prepare_bsr_linear_scaled8(st["w8"], st["x8"], out, bias=st["bias"], act=_act(c),
                                                        residual=st["residual"], pre=pre)
            st["kept"] = (out, pre)


def _told(v, tokens):
    """A tensor as it is; of a scaled 8-bit one the codes' values and the scales'."""
    if isinstance(v, torch.Tensor):
        return {"v": v}
    return {"codes": v.codes.view(EIGHT[v.fmt]), "scales": v.scales.view(torch.float8_e8m0fnu)[:, :tokens]}


def _run_own(st):
    from paper_2507_03117_amd import api

    c, op = st["case"], st["case"]["op"]
    t = c["tokens"]
    if "call" in st:
        st["call"]()
    if op == "keep":
        q = st["kept"] if "call" in st else api.quantize_scaled8(st["x"], group=c["group"], fmt=c["fmt"])
        return {"codes": q.codes.view(EIGHT[c["fmt"]]), "scales": q.scales[:, :t]}
    if op == "linear":
        if "call" in st:
            y, z = st["kept"]
        else:
            z = api.empty_scaled8(t, c["rows"], group=c["b"], fmt="e4m3", device="cuda") if c["pre"] else None
            how = {"out_fmt": "e4m3"} if c["out"] == "e4m3" else {"out_dtype": TYPES[c["out"]]}
            y = api.bsr_linear_scaled8(st["w8"], st["x8"], bias=st["bias"], act=_act(c), residual=st["residual"], pre=z, **how)
        return {"y": _told(y, t), **({"z": _told(z, t)} if c["pre"] else {})}
    if op == "gated":
        g = st["kept"] if "call" in st else api.bsr_gated_scaled8(
            st["w8"], st["wu8"], st["x8"], act=c["act"], keep=c["pre"], out_fmt="e4m3" if c["out"] == "e4m3" else None)
        return {"h": _told(g.H, t), **({"g": _told(g.G, t), "u": _told(g.U, t)} if c["pre"] else {})}
    if op == "wgrad":
        return {"dw": api.bsr_sddmm_scaled8(st["packed"], st["dy"], st["x8"])}
    if c["gated"]:
        g = api.gated_act_backward_scaled8(st["z8"], st["u8"], st["dy"], act=c["act"], bias_grad=c["bias"])
        return {"dg": g.dG, "du": g.dU, "h": g.H, **({"dbg": g.dbias_g, "dbu": g.dbias_u} if c["bias"] else {})}
    g = api.act_backward_scaled8(st["z8"], st["dy"], act=c["act"], bias_grad=c["bias"])
    return {"dz": g.dZ, **({"db": g.dbias} if c["bias"] else {})}


def run(st):
    return _run_own(st) if own else PLAIN[st["case"]["op"]](st)


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


def _plain_out(v, kind, b):
    if kind in EIGHT:
        codes, scales = _quantised(v, b, kind)
        return {"codes": codes, "scales": scales.view(torch.float8_e8m0fnu)[:, :v.shape[0]]}
    return {"v": v.to(TYPES[kind])}


def _plain_keep(st):
    c = st["case"]
    codes, scales = _quantised(st["x"].float(), c["group"], c["fmt"])
    return {"codes": codes, "scales": scales[:, :c["tokens"]]}


def _dense(case, w):
    """The pruned weight in 32 bits, zeros where no block is stored."""
    b, nr, nc = case["b"], case["rows"] // case["b"], case["cols"] // case["b"]
    d = torch.zeros((nr, nc, b, b), device="cuda")
    d[w["where"][:, 0], w["where"][:, 1]] = w["codes"].float() * _power(w["scales"].to(torch.int32) - 127)[:, None, None]
    return d.transpose(1, 2).reshape(case["rows"], case["cols"])


def _plain_linear(st):
    c = st["case"]
    z = _values(*st["x"], c["group"]) @ _dense(c, st["w"]).t()
    if st["bias"] is not None:
        z = z + st["bias"]
    y = _plain_act(c["act"], z)
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return {"y": _plain_out(y, c["out"], c["b"]), **({"z": _plain_out(z, "e4m3", c["b"])} if c["pre"] else {})}


def _plain_gated(st):
    c = st["case"]
    x = _values(*st["x"], c["group"])
    g, u = x @ _dense(c, st["w"]).t(), x @ _dense(c, st["wu"]).t()
    out = {"h": _plain_out(_plain_act(c["act"], g) * u, c["out"], c["b"])}
    if c["pre"]:
        out.update(g=_plain_out(g, "e4m3", c["b"]), u=_plain_out(u, "e4m3", c["b"]))
    return out


def _plain_wgrad(st):
    c = st["case"]
    b = c["b"]
    full = st["dy"].float().t() @ _values(*st["x"], c["group"])
    blocks = full.view(c["rows"] // b, b, c["cols"] // b, b).transpose(1, 2)
    return {"dw": blocks[st["where"][:, 0], st["where"][:, 1]]}


def _plain_act_grad(st):
    c, low = st["case"], torch.bfloat16
    z, dy = _values(*st["z"], c["group"]), st["dy"].float()
    if not c["gated"]:
        dz = dy * _plain_slope(c["act"], z)
        return {"dz": dz.to(low), **({"db": dz.sum(0)} if c["bias"] else {})}
    u, a = _values(*st["u"], c["group"]), _plain_act(c["act"], z)
    dg, du = dy * u * _plain_slope(c["act"], z), dy * a
    return {"dg": dg.to(low), "du": du.to(low), "h": (a * u).to(low),
            **({"dbg": dg.sum(0), "dbu": du.sum(0)} if c["bias"] else {})}


PLAIN = {"keep": _plain_keep, "linear": _plain_linear, "gated": _plain_gated, "wgrad": _plain_wgrad, "act_grad": _plain_act_grad}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _rounded(v, fmt):
    """The format's value nearest to each of `v`, ties to the even mantissa."""
    size = v.abs().clamp_min(2.0 ** LOW[fmt])
    step = torch.exp2(torch.floor(torch.log2(size)) - BITS[fmt])
    return torch.round(v / step) * step


def _eight(v, group, fmt):
    """{codes, scales} of the definition: the smallest power of two that brings the group under the format's largest value."""
    t, k = v.shape
    n = -(-k // group)
    w = torch.zeros((t, n * group), dtype=torch.float64, device=v.device)
    w[:, :k] = v
    w = w.view(t, n, group)
    most = w.abs().amax(2) / (1.75 * 2.0 ** TOP[fmt])
    scale = torch.exp2(torch.ceil(torch.log2(most.clamp_min(2.0 ** LEAST))))
    codes = _rounded(w / scale[:, :, None], fmt).view(t, n * group)[:, :k]
    return {"codes": codes, "scales": scale.t()}


def _meant(pair, group):
    """What a scaled 8-bit tensor stands for."""
    codes, scales = pair
    t, k = codes.shape
    f = torch.exp2(scales[:, :t].double() - 127.0).t().contiguous()
    return codes.to(torch.float64) * f[:, torch.arange(k, device=codes.device) // group]


def _weight_meant(case, w):
    """[rows, cols], block by block into its place."""
    b = case["b"]
    d = torch.zeros((case["rows"], case["cols"]), dtype=torch.float64, device="cuda")
    places = d.view(case["rows"] // b, b, case["cols"] // b, b).permute(0, 2, 1, 3)
    places[w["where"][:, 0], w["where"][:, 1]] = w["codes"].to(torch.float64) * torch.exp2(w["scales"].double() - 127.0).view(-1, 1, 1)
    return d


def _activation(name, v):
    """(act(v), act'(v))."""
    if name == "silu":
        s = torch.sigmoid(v)
        return v * s, s + v * s * (1 - s)
    if name == "gelu":
        cdf, pdf = 0.5 * torch.erfc(-v / math.sqrt(2.0)), torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
        return v * cdf, cdf + v * pdf
    if name == "relu":
        on = (v > 0).double()
        return v * on, on
    return v, torch.ones_like(v)


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "keep":
        return {"codes": _eight(s["x"].double(), case["group"], case["fmt"])["codes"], "scales": None}
    if op == "act_grad":
        a, slope = _activation(case["act"], _meant(s["z"], case["group"]))
        dy = s["dy"].double()
        if not case["gated"]:
            return {"dz": dy * slope, **({"db": (dy * slope).sum(0)} if case["bias"] else {})}
        u = _meant(s["u"], case["group"])
        sums = {"dbg": (dy * u * slope).sum(0), "dbu": (dy * a).sum(0)} if case["bias"] else {}
        return {"dg": dy * u * slope, "du": dy * a, "h": a * u, **sums}
    x = _meant(s["x"], case["group"])
    if op == "wgrad":
        b = case["b"]
        full = torch.matmul(s["dy"].double().t().contiguous(), x).view(case["rows"] // b, b, case["cols"] // b, b)
        return {"dw": full.permute(0, 2, 1, 3)[s["where"][:, 0], s["where"][:, 1]]}

    def told(v, kind):
        return _eight(v, case["b"], kind) if kind in EIGHT else {"v": v}

    z = torch.matmul(_weight_meant(case, s["w"]), x.t().contiguous()).t()
    if op == "gated":
        u = torch.matmul(_weight_meant(case, s["wu"]), x.t().contiguous()).t()
        out = {"h": told(_activation(case["act"], z)[0] * u, case["out"])}
        return {**out, "g": told(z, "e4m3"), "u": told(u, "e4m3")} if case["pre"] else out
    z = z if s["bias"] is None else z + s["bias"].double()
    y = _activation(case["act"], z)[0]
    y = y if s["residual"] is None else y + s["residual"].double()
    return {"y": told(y, case["out"]), **({"z": told(z, "e4m3")} if case["pre"] else {})}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "none": 0}
    t, op = case["tokens"], case["op"]

    def eight(width, group):
        return t * (width + -(-width // group))

    if op == "keep":
        n = t * case["width"]
        return {"bytes": n * size[case["x"]] + eight(case["width"], case["group"]), "flops": 4.0 * n}
    if op == "act_grad":
        n = t * case["width"]
        read = eight(case["width"], case["group"]) * (2 if case["gated"] else 1) + n * size[case["dy"]]
        sums = case["width"] * 4 * (1 + case["gated"]) if case["bias"] else 0
        return {"bytes": read + n * (6 if case["gated"] else 2) + sums, "flops": n * (24.0 if case["gated"] else 16.0)}
    b, rows, cols = case["b"], case["rows"], case["cols"]
    kept = _kept((rows // b) * (cols // b), case["sparsity"])
    x = eight(cols, case["group"])
    if op == "wgrad":
        return {"bytes": t * rows * 2 + x + kept * (4 * b * b + 4), "flops": 2.0 * b * b * kept * t}
    out = eight(rows, b) if case["out"] == "e4m3" else t * rows * size[case["out"]]
    pre = eight(rows, b) if case["pre"] else 0
    if op == "gated":
        return {"bytes": 2 * kept * (b * b + 5) + x + out + 2 * pre, "flops": 4.0 * b * b * kept * t}
    vectors = t * rows * size[case["residual"]] + (4 * rows if case["bias"] else 0)
    return {"bytes": kept * (b * b + 5) + x + out + pre + vectors, "flops": 2.0 * b * b * kept * t}
