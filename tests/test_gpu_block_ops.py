"""The operators around the MLP - blast_bsr_linear, blast_act_backward, blast_norm_residual and its backward - element by
element against their definitions in 64 bits.

Tolerances, derived before any run.  u = 2^-24 is the rounding of one fp32 operation, and a bf16 result is rounded once:
2^-8 of its value, half the spacing of eight significant bits (1 % is added for the rounding of values that already carry the fp32 error).
  A sum of n fp32 terms: at most n u times the sum of the absolute terms; products of bf16 values are exact.
  SiLU, GELU and their slopes: exp2 and reciprocal in hardware and the fitted tail are each within 4 u of their value, the
  exponent's own rounding adds |z| u exp(-|z|) z, below 2 u: 16 u of |z| + 1 covers a value and its slope.
  A norm: centring and scaling err by a few u of the row's largest value times the reciprocal deviation; the row sums are
  trees of at most 64 levels and serial steps, so 64 u of that covers the normalised values."""
import math

import numpy as np
import pytest
import torch

from paper_2507_03117_amd import api, synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def close(got, want, slack, what=""):
    """|got - want| <= slack, plus one rounding where `got` is bf16; everywhere."""
    assert tuple(got.shape) == tuple(want.shape), (what, got.shape, want.shape)
    g, w = got.detach().double().cpu(), want.double().cpu()
    allowed = torch.as_tensor(slack, dtype=torch.float64).cpu() + (2.0 ** -8 * 1.01 * w.abs() if got.dtype == torch.bfloat16 else 0)
    off = (g - w).abs()
    bad = ~(off <= allowed)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: " \
                          f"{g[bad][0].item()!r} for {w[bad][0].item()!r}, allowed {allowed.expand_as(w)[bad][0].item():.3g}"


def rand(seed, shape, dtype=torch.float32, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype)


def wide(t, extra=0, shift=0, tail=0):
    """`t` on the GPU inside a larger buffer: rows `extra` elements apart, the first `shift` elements in."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + extra) + shift + tail,), float("nan"), dtype=t.dtype, device=DEV)
    v = torch.as_strided(buf, (rows, cols), (cols + extra, 1), shift)
    v.copy_(t)
    return v


# ---- the definitions, in 64 bits on the CPU ------------------------------------------------------------------------------

def act64(name, z):
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    return z.clamp_min(0) if name == "relu" else z


def slope64(name, z):
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return (z > 0).double() if name == "relu" else torch.ones_like(z)


def norm64(v, kind, eps, w, b):
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    r = 1 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + eps)
    n = (v - mean) * r
    out = n if w is None else n * w.double()
    return (out if b is None else out + b.double()), n, mean, r


# ---- product with an epilogue ----------------------------------------------------------------------------------------------

def matrix(seed, rows, cols, b, density, empty=True):
    """(packed, dense 64-bit, number of stored blocks of every row): one block row without blocks, one full."""
    rng = np.random.default_rng(seed)
    mask = (rng.random((rows // b, cols // b)) < density).astype(np.uint8)
    mask[-1] = 1
    if empty and rows // b > 1:
        mask[0] = 0
    w = rand(seed, (rows, cols), torch.bfloat16, 0.1)
    packed = api.bsr_pack(w.to(DEV), b, mask=torch.from_numpy(mask).to(DEV))
    keep = torch.from_numpy(np.kron(mask, np.ones((b, b)))).double()
    return packed, w.double() * keep


def check_linear(packed, dense, x, bias, act, residual, out, pre, layout=api.TOKEN_MAJOR, what="", at={}):
    """x, residual: CPU tensors [T, ...]; at: device operands to use instead."""
    turn = (lambda t: t) if layout == api.TOKEN_MAJOR else (lambda t: t.t().contiguous())
    xd = at.get("x", None)
    xd = turn(x).to(DEV) if xd is None else xd
    rd = at.get("residual", None)
    rd = None if residual is None else turn(residual).to(DEV) if rd is None else rd
    shape = turn(torch.empty(x.shape[0], dense.shape[0])).shape
    z = at.get("pre", torch.full(shape, float("nan"), dtype=torch.bfloat16, device=DEV)) if pre else None
    y = at.get("out", torch.full(shape, float("nan"), dtype=TYPES[out], device=DEV))
    got = api.bsr_linear(packed, xd, bias=None if bias is None else bias.to(DEV), act=act, residual=rd, pre=z, layout=layout,
                         out=y)
    assert got is y
    torch.cuda.synchronize()
    x64 = x.double()
    z64 = x64 @ dense.t() + (0 if bias is None else bias.double())
    terms = int(((dense != 0).sum(1).max()).item()) + 2
    size = x64.abs() @ dense.abs().t() + (0 if bias is None else bias.double().abs())
    slack = terms * U * size
    y64 = act64(act, z64) + (0 if residual is None else residual.double())
    more = 16 * U * (z64.abs() + 1) + U * y64.abs() + (0 if residual is None else U * residual.double().abs())
    back = turn(y) if layout == api.FEATURE_MAJOR else y
    close(back, y64, 1.13 * slack + more, what + " y")
    if pre:
        close(turn(z) if layout == api.FEATURE_MAJOR else z, z64, slack, what + " z")


@pytest.mark.parametrize("b", [16, 32, 64, 128])
@pytest.mark.parametrize("T", [1, 2, 5, 16, 17, 33, 64, 100, 257])
def test_linear_blocks_and_tokens(b, T):
    """Every block size over the token counts at which another kernel runs, with all of the epilogue."""
    packed, dense = matrix(b * 1000 + T, 6 * b if b < 128 else 512, 5 * b, b, 0.5)
    rows, cols = dense.shape
    x = rand(T, (T, cols), torch.bfloat16)
    bias, r = rand(T + 1, (rows,), std=0.5), rand(T + 2, (T, rows), torch.bfloat16)
    check_linear(packed, dense, x, bias, "gelu", r, "bf16", True, what=f"b={b} T={T}")
    check_linear(packed, dense, x, bias, None, r.float(), "f32", False, what=f"b={b} T={T} plain")


@pytest.mark.parametrize("act", [None, "silu", "gelu", "relu"])
@pytest.mark.parametrize("bias,residual,pre,out", [(False, None, False, "f32"), (True, None, False, "bf16"),
                                                   (True, "f32", False, "bf16"), (False, "bf16", True, "f32"),
                                                   (True, "f32", True, "f32"), (False, None, True, "bf16")])
@pytest.mark.parametrize("T", [3, 200])
def test_linear_epilogue_parts(act, bias, residual, pre, out, T):
    """Each part of the epilogue with and without the others."""
    for b in (16, 64, 128):
        packed, dense = matrix(7 + b, 3 * b + b * (b < 64), 4 * b, b, 0.6)
        rows, cols = dense.shape
        check_linear(packed, dense, rand(1, (T, cols), torch.bfloat16), rand(2, (rows,)) if bias else None, act,
                     None if residual is None else rand(3, (T, rows), TYPES[residual]), out, pre, what=f"b={b}")


@pytest.mark.parametrize("b,rows,cols,T,density", [(64, 2048, 2048, 700, 0.3), (64, 6400, 1600, 333, 0.2), (64, 1600, 6400, 333, 0.2),
                                                   (128, 4096, 2048, 1000, 0.1), (128, 14336, 1024, 515, 0.3),
                                                   (32, 2048, 4096, 515, 0.1), (16, 1024, 2048, 515, 0.1),
                                                   (64, 64, 1024, 4097, 0.9), (128, 16384, 2048, 1, 0.2)])
def test_linear_layer_sizes(b, rows, cols, T, density):
    """Sizes at which the product takes its large tiles, splits a row's blocks over waves, or takes one token.  The rows and
    tokens of a sample are checked."""
    packed, dense = matrix(rows + cols, rows, cols, b, density)
    x = rand(T, (T, cols), torch.bfloat16).to(DEV)
    bias, r = rand(5, (rows,)).to(DEV), rand(6, (T, rows), torch.bfloat16).to(DEV)
    z = torch.full((T, rows), float("nan"), dtype=torch.bfloat16, device=DEV)
    y = api.bsr_linear(packed, x, bias=bias, act="silu", residual=r, pre=z, out_dtype=torch.bfloat16)
    d = dense.to(DEV)
    z64 = torch.matmul(x.double(), d.t().contiguous()) + bias.double()
    slack = (cols + 2) * U * (torch.matmul(x.double().abs(), d.abs().t().contiguous()) + bias.double().abs())
    # (fp32 sums of up to `cols` terms whose rounding errors are independent: 32 deviations of a walk, and never the whole bound)
    slack = slack * min(1.0, 32 / math.sqrt(cols))
    close(z, z64, slack, "z")
    y64 = z64 * torch.sigmoid(z64) + r.double()
    close(y, y64, 1.13 * slack + 16 * U * (z64.abs() + 1) + U * (r.double().abs() + y64.abs()), "y")


@pytest.mark.parametrize("b", [16, 32, 64, 128])
@pytest.mark.parametrize("T", [4, 70])
def test_linear_layouts_pitches_and_places(b, T):
    """Feature-major operands; rows with odd pitches and addresses that allow no wide access; the residual added in place."""
    packed, dense = matrix(b, 4 * b, 3 * b, b, 0.5)
    rows, cols = dense.shape
    x, bias, r = rand(1, (T, cols), torch.bfloat16), rand(2, (rows,)), rand(3, (T, rows))
    check_linear(packed, dense, x, bias, "silu", r, "f32", True, layout=api.FEATURE_MAJOR, what="feature-major")
    check_linear(packed, dense, x, bias, "silu", r.bfloat16(), "bf16", True, layout=api.FEATURE_MAJOR, what="feature-major bf16")
    odd = {"residual": wide(r, 3, 1), "pre": wide(torch.zeros(T, rows, dtype=torch.bfloat16), 5, 3),
           "out": wide(torch.zeros(T, rows), 7, 1)}
    check_linear(packed, dense, x, bias, "gelu", r, "f32", True, what="odd pitches", at=odd)
    odd = {"x": wide(x, 1, 1), "residual": wide(r, 2, 2), "out": wide(torch.zeros(T, rows, dtype=torch.bfloat16), 1, 1)}
    check_linear(packed, dense, x, bias, "relu", r, "bf16", False, what="odd x", at=odd)
    odd = {"residual": wide(r, 8, 4), "out": wide(torch.zeros(T, rows, dtype=torch.bfloat16), 8, 8),
           "pre": wide(torch.zeros(T, rows, dtype=torch.bfloat16), 3, 0)}
    check_linear(packed, dense, x, bias, None, r, "bf16", True, what="one odd pitch", at=odd)
    for dtype in (torch.float32, torch.bfloat16):
        stream = r.to(dtype).to(DEV)
        check_linear(packed, dense, x, bias, None, r.to(dtype), "f32" if dtype == torch.float32 else "bf16", False,
                     what="in place", at={"residual": stream, "out": stream})


@pytest.mark.parametrize("b,rows,cols,T", [(128, 8192, 512, 1030), (128, 1024, 512, 700), (64, 8192, 512, 1030), (64, 2048, 512, 1030), (32, 2048, 512, 515),
                                           (16, 512, 512, 515)])
@pytest.mark.parametrize("odd", ["none", "y", "r", "z", "all"])
def test_linear_large_tiles_with_odd_pitches(b, rows, cols, T, odd):
    """The kernels of many tokens store and read two rows at a time where every operand allows it, and only there; a last tile
    that the tokens end in; the residual in place."""
    packed, dense = matrix(rows + b, rows, cols, b, 0.3)
    d = dense.to(DEV)
    x, bias = rand(T, (T, cols), torch.bfloat16).to(DEV), rand(5, (rows,)).to(DEV)
    z64 = torch.matmul(x.double(), d.t().contiguous()) + bias.double()
    slack = (cols + 2) * U * (torch.matmul(x.double().abs(), d.abs().t().contiguous()) + bias.double().abs())
    for r_type, y_type in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)):
        r = rand(6, (T, rows), r_type)
        place = lambda t, n: wide(t, 3, 1) if odd in (n, "all") else t.to(DEV)  # noqa: E731
        rd, y, z = place(r, "r"), place(torch.zeros(T, rows, dtype=y_type), "y"), place(torch.zeros(T, rows, dtype=torch.bfloat16), "z")
        api.bsr_linear(packed, x, bias=bias, act="relu", residual=rd, pre=z, out=y)
        close(z, z64, slack, "z")
        y64 = z64.clamp_min(0) + r.to(DEV).double()
        close(y, y64, slack + U * (r.to(DEV).double().abs() + y64.abs()), "y")
        same = place(r, "r")
        api.bsr_linear(packed, x, bias=bias, residual=same, out=same)
        y64 = z64 + r.to(DEV).double()
        close(same, y64, slack + U * (r.to(DEV).double().abs() + y64.abs()), "in place")


@pytest.mark.parametrize("b", [32, 64, 128])
def test_linear_activations_beyond_32_bit_offsets(b):
    """More tokens than 32-bit offsets into X reach: token ranges of their own, whose residual, Z and Y move along."""
    packed, dense = matrix(b, 256, 256, b, 0.7)
    T, pitch = 600, 4 << 20
    buf = torch.empty((T - 1) * pitch + 256, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (T, 256), (pitch, 1))
    host = rand(1, (T, 256), torch.bfloat16)
    x.copy_(host)
    check_linear(packed, dense, host, rand(2, (256,)), "silu", rand(3, (T, 256)), "bf16", True, what="long", at={"x": x})


def test_linear_without_blocks_tokens_or_epilogue():
    """No stored block: act(bias) + residual.  No token: nothing.  No epilogue: the bits of bsr_spmm in bf16."""
    for b in (16, 64, 128):
        w = torch.zeros((2 * b, b), dtype=torch.bfloat16, device=DEV)
        packed = api.bsr_pack(w, b, mask=torch.zeros((2, 1), dtype=torch.uint8, device=DEV))
        bias, r = rand(1, (2 * b,)), rand(2, (70, 2 * b))
        for T in (1, 70):
            check_linear(packed, torch.zeros(2 * b, b, dtype=torch.float64), rand(3, (T, b), torch.bfloat16), bias, "gelu", r[:T],
                         "f32", True, what=f"empty b={b}")
        assert api.bsr_linear(packed, torch.zeros((0, b), dtype=torch.bfloat16, device=DEV), bias=bias.to(DEV)).shape == (0, 2 * b)
        packed, dense = matrix(b, 4 * b, 4 * b, b, 0.5)
        for T in (1, 40, 300):
            x = rand(T, (T, 4 * b), torch.bfloat16).to(DEV)
            close(api.bsr_linear(packed, x), api.bsr_spmm(packed, x).double(), (dense != 0).sum(1).max().item() * U * (x.double().cpu().abs() @ dense.abs().t()))


def test_linear_offsets_beyond_32_bits():
    """The residual, Z and Y of a few tokens whose rows lie more than 2^31 elements apart in one buffer."""
    packed, dense = matrix(3, 128, 128, 64, 1.0, empty=False)
    pitch = (1 << 30) + 8
    buf = torch.empty(3 * pitch, dtype=torch.bfloat16, device=DEV)
    x, r = rand(1, (3, 128), torch.bfloat16), rand(2, (3, 128), torch.bfloat16)
    places = [torch.as_strided(buf, (3, 128), (pitch, 1), at) for at in (0, 1024, 2048)]
    places[0].copy_(r)
    check_linear(packed, dense, x, None, "silu", r, "bf16", True, what="far",
                 at={"residual": places[0], "pre": places[1], "out": places[2]})


def test_row_operators_beyond_32_bit_offsets():
    """Rows more than 2^31 elements apart in one buffer."""
    pitch = (1 << 30) + 8
    buf = torch.empty(3 * pitch, dtype=torch.bfloat16, device=DEV)
    place = lambda at, t: torch.as_strided(buf, t.shape, (pitch, 1), at).copy_(t)  # noqa: E731
    z, u, dy = (rand(k, (3, 72), torch.bfloat16) for k in range(3))
    far = [place(128 * k, t) for k, t in enumerate((z, u, dy))]
    api._act_backward(*far, "silu", far[0], far[1], far[2], None, None)
    check_act(z, u, dy, "silu", False, {"dz": far[0], "du": far[1], "h": far[2]}, "far")
    s = norm_inputs(5, 3, 72, "layer", "bf16", "bf16", "f32", True, "tokens")
    s["args"]["gate"] = s["args"]["gate"].bfloat16()
    at = {"h": place(1024, s["h"]), "y": place(1152, s["y"]), "h_out": place(1280, s["h"]), "out": place(1408, s["h"])}
    check_forward(s, "far", **at)
    at = {"h": place(1024, s["h"]), "y": place(1152, s["y"]), "dx": place(1280, s["dx"]), "dh": place(1408, s["dh"]), "to": place(1536, s["h"])}
    check_backward(s, "far", **at)


# ---- gradient of an activation -----------------------------------------------------------------------------------------------

def check_act(z, u, dy, act, bias_grad, got, what=""):
    z64 = None if z is None else z.double().cpu()
    d = dy.double().cpu()
    slope = torch.ones_like(d) if z is None else slope64(act, z64)
    a = d if z is None else act64(act, z64)
    size = torch.ones_like(d) if z is None else z64.abs() + 1
    dz = d * slope if u is None else d * u.double().cpu() * slope
    scale = d.abs() if u is None else (d * u.double().cpu()).abs()
    close(got["dz"], dz, 24 * U * scale * size, what + " dz")
    T = d.shape[0]
    if u is not None:
        close(got["du"], d * a, 24 * U * d.abs() * size, what + " du")
        if got.get("h") is not None:
            close(got["h"], a * u.double().cpu(), 24 * U * u.double().cpu().abs() * size, what + " h")
    if bias_grad:
        close(got["db"], dz.sum(0), U * ((T + 24) * (scale * size).sum(0)), what + " db")
        if u is not None:
            close(got["dbu"], (d * a).sum(0), U * ((T + 24) * (d.abs() * size).sum(0)), what + " dbu")


def run_act(z, u, dy, act, bias_grad, with_h=True):
    if u is None:
        g = api.act_backward(z, dy, act=act, bias_grad=bias_grad)
        return {"dz": g.dZ, "db": g.dbias}
    g = api.gated_act_backward(z, u, dy, act=act, bias_grad=bias_grad, with_h=with_h)
    return {"dz": g.dG, "du": g.dU, "h": g.H, "db": g.dbias_g, "dbu": g.dbias_u}


@pytest.mark.parametrize("T,N", [(1, 1), (1, 8), (2, 3), (7, 16), (8, 256), (9, 264), (33, 250), (64, 1600), (333, 6400), (1000, 40),
                                 (4100, 24), (3, 20000)])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("gated", [False, True])
def test_act_backward_sizes(T, N, act, gated):
    for k, (dtype, bias_grad) in enumerate(((torch.float32, True), (torch.bfloat16, False), (torch.bfloat16, True))):
        z = rand(T + N, (T, N), torch.bfloat16, 2.0).to(DEV)
        u = rand(T + N + 1, (T, N), torch.bfloat16).to(DEV) if gated else None
        dy = rand(T + N + 2, (T, N), dtype).to(DEV)
        check_act(z, u, dy, act, bias_grad, run_act(z, u, dy, act, bias_grad, with_h=k != 1), f"{T}x{N} {dtype}")


@pytest.mark.parametrize("T", [63, 64, 65, 255, 256, 257, 511, 512, 513, 1024])
@pytest.mark.parametrize("N", [8, 31, 32, 40, 512, 520, 1000])
def test_act_backward_sums_at_the_seams(T, N):
    """Row counts at which the columns' sums change hands, widths that end inside a workgroup's columns."""
    z, u = rand(T, (T, N), torch.bfloat16, 2.0).to(DEV), rand(N, (T, N), torch.bfloat16).to(DEV)
    dy = rand(T + N, (T, N)).to(DEV)
    for gate in (None, u):
        check_act(z, gate, dy, "silu", True, run_act(z, gate, dy, "silu", True), f"{T}x{N}")


def test_act_backward_over_the_range_of_bf16():
    """Every finite bf16 value of the pre-activation: slopes at zeros of both signs, in the tails and beyond them."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    z = bits.view(torch.bfloat16)
    z = torch.where(torch.isfinite(z), z, torch.zeros_like(z)).view(64, 1024).to(DEV)
    dy = rand(1, (64, 1024)).to(DEV)
    for act in ("silu", "gelu", "relu"):
        got = api.act_backward(z, dy, act=act).dZ.double().cpu()
        z64, d = z.double().cpu(), dy.double().cpu()
        # far out the slope is 0 or 1 to within 24 u, not to within |z| u
        size = torch.minimum(z64.abs() + 1, torch.full_like(z64, 128.0))
        assert bool(((got - d * slope64(act, z64)).abs() <= 24 * U * size * d.abs() + 2.0 ** -8 * 1.01 * (d * slope64(act, z64)).abs() + 1e-40).all())


def test_act_backward_of_a_bias_alone():
    """No activation: the gradient passes, and its sum over the tokens is the bias'."""
    for T, N in ((1, 5), (300, 1600)):
        dy = rand(T, (T, N)).to(DEV)
        check_act(None, None, dy, None, True, run_act(None, None, dy, None, True), "bias")


@pytest.mark.parametrize("gated", [False, True])
def test_act_backward_pitches_and_places(gated):
    """Rows apart by odd and by wide pitches, odd addresses, results over the operands they come from."""
    T, N = 37, 72
    for extra, shift in ((0, 0), (8, 8), (3, 1), (5, 0), (0, 4)):
        z, u, dy = (wide(rand(k, (T, N), torch.bfloat16), extra, shift) for k in range(3))
        check_act(z, u if gated else None, dy, "silu", True, run_act(z, u if gated else None, dy, "silu", True), f"{extra} {shift}")
    z, u, dy = (rand(k, (T, N), torch.bfloat16).to(DEV) for k in range(3))
    if gated:
        kept = z.clone(), u.clone(), dy.clone()
        api._act_backward(z, u, dy, "gelu", z, u, dy, None, None)
        check_act(kept[0], kept[1], kept[2], "gelu", False, {"dz": z, "du": u, "h": dy}, "in place")
    else:
        kept = z.clone()
        api.act_backward(z, dy, act="gelu", out=z)
        check_act(kept, None, dy, "gelu", False, {"dz": z}, "in place")


def test_act_backward_over_no_rows_and_repeatability():
    z = torch.zeros((0, 48), dtype=torch.bfloat16, device=DEV)
    g = api.gated_act_backward(z, z, z, bias_grad=True)
    assert g.dG.shape == (0, 48) and not g.dbias_g.any() and not g.dbias_u.any()
    z, dy = rand(1, (5000, 320), torch.bfloat16).to(DEV), rand(2, (5000, 320)).to(DEV)
    first = api.act_backward(z, dy, act="silu", bias_grad=True).dbias
    for _ in range(3):
        assert torch.equal(first, api.act_backward(z, dy, act="silu", bias_grad=True).dbias)


# ---- norms with gate and residual ------------------------------------------------------------------------------------------

def norm_inputs(seed, T, E, kind, h="f32", y="bf16", params="f32", post=False, gate=None, scale=1.0, mean=0.3):
    p = TYPES[params]
    layer = kind == "layer"
    return {"h": rand(seed, (T, E), TYPES[h], 1.5, mean), "y": None if y is None else rand(seed + 1, (T, E), TYPES[y], 0.7, 0.1),
            "dx": rand(seed + 2, (T, E), torch.bfloat16), "dh": rand(seed + 3, (T, E), TYPES[h]),
            "args": {"kind": kind, "weight": rand(seed + 4, (E,), p, 0.3, 1.0), "bias": rand(seed + 5, (E,), p) if layer else None,
                     "post": post, "post_weight": rand(seed + 6, (E,), p, 0.3, 1.0) if post else None,
                     "post_bias": rand(seed + 7, (E,), p) if post and layer else None,
                     "gate": None if gate is None else rand(seed + 8, (E,) if gate == "vector" else (T, E), p, 0.5, 0.4),
                     "scale": scale, "eps": 1e-5}}


def on_gpu(args):
    return {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in args.items()}


def forward64(s, h=None, y=None):
    a = s["args"]
    h = s["h"].double() if h is None else h
    st = [torch.zeros_like(h[:, :1])] * 2
    p = None
    if s["y"] is not None:
        y = s["y"].double() if y is None else y
        p = y
        if a["post"]:
            p, _, mean, r = norm64(y, a["kind"], a["eps"], a["post_weight"], a["post_bias"])
            st = [mean, r]
        if a["gate"] is not None:
            p = p * a["gate"].double()
        h = h + a["scale"] * p
    x, n, mean, r = norm64(h, a["kind"], a["eps"], a["weight"], a["bias"])
    return h, x, torch.cat([mean, r] + st, 1), n


def check_forward(s, what="", **places):
    a, hd = on_gpu(s["args"]), places.get("h", s["h"].to(DEV))
    yd = None if s["y"] is None else places.get("y", s["y"].to(DEV))
    h, x, stats = api.norm_residual(hd, yd, with_stats=True, h_out=places.get("h_out"), out=places.get("out"), **a)
    torch.cuda.synchronize()
    h64, x64, st64, n64 = forward64(s)
    top = lambda t: t.abs().max(1, keepdim=True).values  # noqa: E731
    r, r_y = st64[:, 1:2], st64[:, 3:4]
    # the branch: 64 u of its normalised values' row, or one product; the stream adds one rounding of each
    slack_h = torch.zeros_like(h64)
    if s["y"] is not None:
        w = torch.ones(1) if a["post_weight"] is None else s["args"]["post_weight"]
        g = torch.ones(1) if a["gate"] is None else s["args"]["gate"]
        branch = (h64 - s["h"].double()).abs()
        n_y = top(s["y"].double()) * r_y + 1 if a["post"] else torch.zeros(1, dtype=torch.float64)
        slack_h = a["scale"] * (64 * U * n_y * (w.double() * g.double()).abs()) + 4 * U * branch + U * (h64.abs() + s["h"].double().abs())
        close(h, h64, slack_h, what + " h")
    else:
        assert h is hd
    wx = torch.ones(1, dtype=torch.float64) if a["weight"] is None else s["args"]["weight"].double().abs()
    slack_n = 64 * U * (top(h64) * r + 1) + (slack_h + top(slack_h) * (1 + n64.abs())) * r
    close(x, x64, slack_n * wx + 2 * U * x64.abs(), what + " x")
    size = torch.cat([top(h64), r * 1, top(s["y"].double()) if s["y"] is not None else top(h64), r_y], 1)
    close(stats, st64, 64 * U * size + torch.cat([top(slack_h), top(slack_h) * r * r, torch.zeros_like(r), torch.zeros_like(r)], 1), what + " stats")


WIDTHS = [1, 2, 7, 8, 16, 129, 512, 520, 1000, 1024, 1032, 1600, 2048, 2056, 4096, 4104, 8192, 8200, 16384, 16392, 20001, 32768]


@pytest.mark.parametrize("E", WIDTHS)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_widths(E, kind):
    """Every number of waves and pieces a row can take, both sides of each, and widths without wide access."""
    if kind == "layer" and E == 1:
        return  # (one value has no deviation: 0 / sqrt(eps) either way, checked as a constant row below)
    for T in (1, 5) if E > 4096 else (1, 3, 70):
        check_forward(norm_inputs(E, T, E, kind, "bf16", "f32", "bf16", True, "vector", 0.5), f"{E} {T}")
        check_forward(norm_inputs(E, T, E, kind, "f32", None), f"{E} {T} alone")


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("h,y,params,post,gate", [("f32", "f32", "f32", False, None), ("bf16", "bf16", "bf16", False, "vector"),
                                                  ("bf16", "f32", "f32", False, "tokens"), ("f32", "bf16", "bf16", True, None),
                                                  ("bf16", "bf16", "f32", True, "tokens"), ("f32", "f32", "bf16", True, "vector")])
def test_norm_types_and_parts(kind, h, y, params, post, gate):
    for T, E in ((33, 264), (9, 1600), (4, 131)):
        check_forward(norm_inputs(E, T, E, kind, h, y, params, post, gate, 0.7), f"{T}x{E}")


def test_norm_without_parameters():
    s = norm_inputs(1, 6, 80, "layer", post=True)
    for k in ("weight", "bias", "post_weight", "post_bias"):
        s["args"][k] = None
    check_forward(s)


@pytest.mark.parametrize("E", [64, 131, 2048])
def test_norm_pitches_and_places(E):
    """Rows apart by wide and by odd pitches, odd addresses, the stream updated in place, fp32 output."""
    s = norm_inputs(5, 21, E, "rms", "f32", "bf16", "f32", True, "tokens")
    for extra, shift in ((8, 8), (3, 0), (0, 1)):
        check_forward(s, f"{extra} {shift}", h=wide(s["h"], extra, shift), y=wide(s["y"], extra, shift), h_out=wide(s["h"], extra + 8, shift),
                      out=wide(torch.zeros(21, E), extra, shift))
    stream = s["h"].to(DEV)
    check_forward(s, "in place", h=stream, h_out=stream)


@pytest.mark.parametrize("T,E,h,gate,cuts", [(4100, 4096, "bf16", None, (0, 7, 2000, 4100)), (1030, 16384, "bf16", "tokens", (0, 300, 301, 1030)),
                                             (2050, 8200, "f32", "vector", (0, 1000, 2050)),
                                             (2 ** 26 + 5, 8, "bf16", "tokens", (0, 2 ** 25, 2 ** 25 + 1, 2 ** 26 + 5))])
def test_norm_of_many_rows_is_that_of_its_parts(T, E, h, gate, cuts):
    """Streams beyond the L2s, and more rows than a launch has lanes for: bit for bit what calls on runs of the rows give, one
    run of which is held against the definition."""
    g = torch.Generator(device=DEV).manual_seed(T)
    make = lambda *shape, dtype=torch.bfloat16: torch.randn(shape, generator=g, device=DEV, dtype=dtype)
    hd, yd, w = make(T, E, dtype=TYPES[h]), make(T, E), make(E)
    gd = None if gate is None else make(T, E) if gate == "tokens" else make(E)
    part = lambda t, a, b: t if t is None or t.dim() == 1 else t[a:b]
    new_h, x, stats = api.norm_residual(hd, yd, weight=w, gate=gd, scale=0.5, with_stats=True)
    for a, b in zip(cuts, cuts[1:]):
        ph, px, ps = api.norm_residual(hd[a:b], yd[a:b], weight=w, gate=part(gd, a, b), scale=0.5, with_stats=True)
        assert torch.equal(ph, new_h[a:b]) and torch.equal(px, x[a:b]) and torch.equal(ps, stats[a:b])
    a = T - 5
    args = dict(norm_inputs(1, 5, E, "rms")["args"], weight=w.cpu(), gate=None if gd is None else part(gd, a, T).cpu(), scale=0.5)
    check_forward(dict(h=hd[a:].cpu(), y=yd[a:].cpu(), args=args), h=hd[a:].clone(), y=yd[a:].clone())
    assert torch.equal(api.norm_residual(hd[a:], yd[a:], **on_gpu(args))[1], x[a:])


def test_norm_hard_rows():
    """Rows whose mean is far from their deviation, constant rows, rows of zeros; one row's infinity or NaN stays in it."""
    T, E = 8, 1600
    s = norm_inputs(9, T, E, "layer", "f32", "f32")
    s["h"][0] += 3000.0  # the variance of the centred values: not the difference of two large means
    s["y"][1], s["h"][1] = 0.0, 2.5  # no deviation but eps
    s["y"][2], s["h"][2] = 0.0, 0.0
    h64, x64, st64, _ = forward64(s)
    check_forward(s)
    a = on_gpu(s["args"])
    h, x = api.norm_residual(s["h"].to(DEV), s["y"].to(DEV), **a)
    bad = s["h"].clone()
    bad[3, 17], bad[5, 1599] = float("inf"), float("nan")
    h2, x2 = api.norm_residual(bad.to(DEV), s["y"].to(DEV), **a)
    fine = [0, 1, 2, 4, 6, 7]
    assert torch.equal(x[fine], x2[fine]) and torch.equal(h[fine], h2[fine])
    assert torch.isnan(x2[5]).all() and torch.isnan(x2[3]).any() and h2[3, 17] == float("inf")


def check_backward(s, what="", with_dh=True, **places):
    """Against autograd of the definition in 64 bits, at the stored stream and with the statistics of that stream."""
    a = s["args"]
    h64, y64 = s["h"].double(), None if s["y"] is None else s["y"].double()
    _, nh, mean, r = norm64(h64, a["kind"], a["eps"], None, None)
    st = [mean, r, torch.zeros_like(mean), torch.zeros_like(mean)]
    if y64 is not None and a["post"]:
        _, m, mean_y, r_y = norm64(y64, a["kind"], a["eps"], None, None)
        st[2:] = [mean_y, r_y]
    stats = torch.cat(st, 1).float()
    given = s["dh"] if with_dh else None
    hd = places.get("h", s["h"].to(DEV))
    yd = None if s["y"] is None else places.get("y", s["y"].to(DEV))
    g = api.norm_residual_backward(hd, yd, stats.to(DEV), places.get("dx", s["dx"].to(DEV)),
                                   None if given is None else places.get("dh", given.to(DEV)), dh=places.get("to"), **on_gpu(a))
    torch.cuda.synchronize()
    T, E = h64.shape
    ones = torch.ones(1, dtype=torch.float64)
    f = lambda t: ones if t is None else t.double()  # noqa: E731
    leaves = {"h": h64.clone().requires_grad_()}
    for k in ("weight", "bias"):
        if a[k] is not None:
            leaves[k] = a[k].double().requires_grad_()
    x, _, _, _ = norm64(leaves["h"], a["kind"], a["eps"], leaves.get("weight"), leaves.get("bias"))
    x = x if "bias" in leaves else x
    grads = dict(zip(leaves, torch.autograd.grad(x, list(leaves.values()), s["dx"].double())))
    dh64 = grads["h"] + (0 if given is None else given.double())
    top = lambda t: t.abs().max(1, keepdim=True).values  # noqa: E731
    dn = (s["dx"].double() * f(a["weight"])).abs()
    # n errs by 64 u of its row's size; it enters linearly and in the projection on n
    n_off = 64 * U * (top(h64) * r + 1)
    slack = r * (dn.max(1, keepdim=True).values * (n_off * (2 + nh.abs()) + 64 * U * (1 + nh.abs() * top(nh)))) + 4 * U * (dh64.abs() + f(given).abs())
    close(g.dh, dh64, slack, what + " dh")
    col = lambda terms: U * (T + 64) * terms.abs().sum(0)  # noqa: E731
    if a["weight"] is not None:
        close(g.dweight, grads["weight"], col(s["dx"].double() * (nh.abs() + n_off / U / 64)), what + " dweight")
    else:
        assert g.dweight is None
    if a["bias"] is not None:
        close(g.dbias, grads["bias"], col(s["dx"].double()), what + " dbias")
    if y64 is None:
        assert g.dy is None and g.dgate is None
        return
    leaves = {"y": y64.clone().requires_grad_()}
    for k in ("gate", "post_weight", "post_bias"):
        if a[k] is not None:
            leaves[k] = a[k].double().requires_grad_()
    p = norm64(leaves["y"], a["kind"], a["eps"], leaves.get("post_weight"), leaves.get("post_bias"))[0] if a["post"] else leaves["y"]
    p_abs = p.detach().abs()
    branch = a["scale"] * (p * leaves["gate"] if "gate" in leaves else p)
    grads = dict(zip(leaves, torch.autograd.grad(branch, list(leaves.values()), dh64)))
    dp = (a["scale"] * dh64 * f(a["gate"])).abs()
    dp_off = a["scale"] * slack * f(a["gate"]).abs()  # what dh errs by
    m_off = 64 * U * (top(y64) * st[3] + 1) if a["post"] else 0 * top(y64)
    p_off = m_off * f(a["post_weight"]).abs() + 4 * U * p_abs
    if a["gate"] is not None:
        one = a["scale"] * (dh64.abs() * p_off + slack * p_abs) + 4 * U * (a["scale"] * dh64 * p_abs).abs()
        close(g.dgate, grads["gate"], one.sum(0) + col(a["scale"] * dh64 * p_abs) if a["gate"].dim() == 1 else one, what + " dgate")
    if a["post"]:
        m_abs = m.abs()
        if a["post_weight"] is not None:
            close(g.dpost_weight, grads["post_weight"], (dp_off * m_abs + dp * m_off).sum(0) + col(dp * (m_abs + 1)), what + " dpost_weight")
        if a["post_bias"] is not None:
            close(g.dpost_bias, grads["post_bias"], dp_off.sum(0) + col(dp), what + " dpost_bias")
        dm, dm_off = dp * f(a["post_weight"]).abs(), dp_off * f(a["post_weight"]).abs()
        most, off = dm.max(1, keepdim=True).values, dm_off.max(1, keepdim=True).values
        close(g.dy, grads["y"], st[3] * (most * (m_off * (2 + m_abs) + 64 * U * (1 + m_abs * top(m))) + off * (2 + m_abs * top(m))) + 4 * U * grads["y"].abs(), what + " dy")
    else:
        close(g.dy, grads["y"], dp_off + 4 * U * dp, what + " dy")


@pytest.mark.parametrize("E", [w for w in WIDTHS if w > 1])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_backward_widths(E, kind):
    for T in (1, 5) if E > 4096 else (1, 6, 300):
        check_backward(norm_inputs(E, T, E, kind, "bf16", "bf16", "bf16", True, "vector", 0.5), f"{E} {T}")
        check_backward(norm_inputs(E, T, E, kind, "f32", None), f"{E} {T} alone", with_dh=False)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("h,y,params,post,gate", [("f32", "f32", "f32", False, None), ("bf16", "bf16", "bf16", False, "vector"),
                                                  ("bf16", "f32", "f32", False, "tokens"), ("f32", "bf16", "bf16", True, None),
                                                  ("bf16", "bf16", "f32", True, "tokens"), ("f32", "f32", "bf16", True, "vector")])
@pytest.mark.parametrize("dh", [False, True])
def test_norm_backward_types_and_parts(kind, h, y, params, post, gate, dh):
    for T, E in ((33, 264), (600, 96), (4, 131), (9, 1600), (700, 2048)):
        check_backward(norm_inputs(E, T, E, kind, h, y, params, post, gate, 0.7), f"{T}x{E}", with_dh=dh)


@pytest.mark.parametrize("E", [64, 131])
def test_norm_backward_pitches_and_places(E):
    s = norm_inputs(5, 21, E, "layer", "f32", "bf16", "f32", True, "tokens")
    for extra, shift in ((8, 8), (3, 0), (0, 1)):
        check_backward(s, f"{extra} {shift}", h=wide(s["h"], extra, shift), y=wide(s["y"], extra, shift), dx=wide(s["dx"], extra, shift),
                       dh=wide(s["dh"], extra, shift), to=wide(s["dh"], extra + 8, shift))
    d = s["dh"].to(DEV)
    g = api.norm_residual_backward(s["h"].to(DEV), None, torch.cat([torch.zeros(21, 1), torch.ones(21, 3)], 1).to(DEV), s["dx"].to(DEV), d, dh=d)
    want = api.norm_residual_backward(s["h"].to(DEV), None, torch.cat([torch.zeros(21, 1), torch.ones(21, 3)], 1).to(DEV), s["dx"].to(DEV), s["dh"].to(DEV))
    assert g.dh is d and torch.equal(d, want.dh)


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 511, 512, 513, 1030])
@pytest.mark.parametrize("E", [8, 24, 40, 129, 520, 1600])
def test_norm_backward_sums_at_the_seams(T, E):
    """Row counts at which the columns' sums change hands, widths that end inside a workgroup's columns, with and without the
    branch's own sums."""
    for kind, y, post, gate in (("layer", None, False, None), ("rms", "bf16", False, "tokens"), ("layer", "bf16", False, "vector"),
                                ("layer", "f32", True, "tokens"), ("rms", "bf16", True, "vector")):
        check_backward(norm_inputs(T + E, T, E, kind, "f32", y, "f32", post, gate), f"{T}x{E} {kind} {post} {gate}")


def test_norm_backward_over_no_rows_and_repeatability():
    """Over no rows the sums are zeros; repeated calls give the same bits."""
    s = norm_inputs(3, 2, 96, "layer", post=True, gate="vector")
    a = on_gpu(s["args"])
    none = torch.zeros((0, 96), device=DEV)
    g = api.norm_residual_backward(none, none, torch.zeros((0, 4), device=DEV), none, none, **a)
    for t in (g.dweight, g.dbias, g.dgate, g.dpost_weight, g.dpost_bias):
        assert t.shape == (96,) and not t.any()
    h, x = api.norm_residual(none, none, **a)
    assert h.shape == x.shape == (0, 96)
    s = norm_inputs(4, 3000, 1600, "layer", "bf16", "bf16", "bf16", True, "vector")
    stats = torch.rand((3000, 4)).to(DEV)
    runs = [api.norm_residual_backward(s["h"].to(DEV), s["y"].to(DEV), stats, s["dx"].to(DEV), **on_gpu(s["args"])) for _ in range(3)]
    for g in runs[1:]:
        for k in ("dh", "dy", "dgate", "dweight", "dbias", "dpost_weight", "dpost_bias"):
            assert torch.equal(getattr(g, k), getattr(runs[0], k)), k


# ---- gradients against differences -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_act_backward_against_differences(act):
    """Directional derivatives of act(G) U from values a step apart in 64 bits.  The gradients are rounded to bf16: 2^-8 of their
    length times the direction's; the central difference errs by its step squared."""
    z, u, dy = (rand(k, (24, 40), torch.bfloat16) for k in range(3))
    g = api.gated_act_backward(z.to(DEV), u.to(DEV), dy.to(DEV), act=act)
    for wrt, grad in (("z", g.dG), ("u", g.dU)):
        d = rand(9, (24, 40)).double()
        step = 1e-4
        f = lambda s: ((act64(act, z.double() + s * d * (wrt == "z")) * (u.double() + s * d * (wrt == "u"))) * dy.double()).sum()  # noqa: E731
        grad = grad.double().cpu()
        assert abs((f(step) - f(-step)).item() / (2 * step) - (grad * d).sum().item()) <= 2.0 ** -8 * grad.norm() * d.norm() + 1e-5


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_backward_against_differences(kind):
    """The same for the whole step h' = h + s g norm(y), x = norm(h'), forward and backward calls of the library: the loss takes
    both outputs, the directions go through h, y, the gate and the weights.  Beside the rounding of the gradients (bf16 dy) there
    is that of the stored stream: fp32 here."""
    T, E = 12, 88
    s = norm_inputs(2, T, E, kind, "f32", "f32", "f32", True, "vector", 0.6)
    a = s["args"]
    c_h, c_x = s["dh"].double(), s["dx"].double()
    h_new, _, stats = api.norm_residual(s["h"].to(DEV), s["y"].to(DEV), with_stats=True, **on_gpu(a))
    g = api.norm_residual_backward(h_new, s["y"].to(DEV), stats, s["dx"].to(DEV), s["dh"].to(DEV), **on_gpu(a))
    grads = {"h": g.dh, "y": g.dy, "gate": g.dgate, "weight": g.dweight, "bias": g.dbias, "post_weight": g.dpost_weight,
             "post_bias": g.dpost_bias}
    for k, grad in grads.items():
        if grad is None:
            assert kind == "rms" and k.endswith("bias")
            continue
        base = (s[k] if k in ("h", "y") else a[k]).double()
        d = rand(11, tuple(base.shape)).double()

        def loss(step):
            t = {"args": dict(a), "h": s["h"], "y": s["y"]}
            kw = {}
            if k in ("h", "y"):
                kw[k] = base + step * d
            else:
                t["args"][k] = base + step * d
            h64, x64, _, _ = forward64(t, **kw)
            return (h64 * c_h).sum() + (x64 * c_x).sum()

        step = 1e-4
        grad = grad.double().cpu()
        off = abs((loss(step) - loss(-step)).item() / (2 * step) - (grad * d).sum().item())
        assert off <= 2.0 ** -8 * grad.norm() * d.norm() + 1e-4, (k, off)
