"""Edges of the operators around the MLP: parameters that come alone, gates laid out by a stride of 0, NaN before a ReLU, more
columns than a launch has owners for, the gradient's kernels that go over their rows, forward and backward calls in a row on a rounded stream.

Definitions and tolerances are those of test_gpu_block_ops.py; the ones of this file are derived where they stand.  Inputs of the large
cases are made, and compared in 64 bits, on the card."""
import pytest
import torch

from paper_2507_03117_amd import api
from tests import test_gpu_block_ops as ops

pytestmark = pytest.mark.gpu

U, DEV, TYPES = ops.U, ops.DEV, ops.TYPES


def close(got, want, slack, what=""):
    """ops.close without the way through host memory."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    g, w = got.detach().double(), want.double().to(got.device)
    allowed = torch.as_tensor(slack, dtype=torch.float64).to(got.device) + (2.0 ** -8 * 1.01 * w.abs() if got.dtype == torch.bfloat16 else 0)
    bad = ~((g - w).abs() <= allowed)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: " \
                          f"{g[bad][0].item()!r} for {w[bad][0].item()!r}, allowed {allowed.expand_as(w)[bad][0].item():.3g}"


@pytest.fixture
def on_card(monkeypatch):
    """The definitions and comparisons of test_gpu_block_ops.py, computed on the card."""
    monkeypatch.setattr(ops, "close", close)
    with torch.device(DEV):
        yield


def norm_inputs(seed, T, E, kind, h, y, params, post, gate, scale):
    """ops.norm_inputs, made on the card."""
    gen, p, layer = torch.Generator(DEV).manual_seed(seed), TYPES[params], kind == "layer"
    make = lambda shape, dtype, std=1.0, mean=0.0: (torch.randn(shape, generator=gen, device=DEV) * std + mean).to(dtype)  # noqa: E731
    return {"h": make((T, E), TYPES[h], 1.5, 0.3), "y": None if y is None else make((T, E), TYPES[y], 0.7, 0.1),
            "dx": make((T, E), torch.bfloat16), "dh": make((T, E), TYPES[h]),
            "args": {"kind": kind, "weight": make((E,), p, 0.3, 1.0), "bias": make((E,), p) if layer else None, "post": post,
                     "post_weight": make((E,), p, 0.3, 1.0) if post else None, "post_bias": make((E,), p) if post and layer else None,
                     "gate": None if gate is None else make((E,) if gate == "vector" else (T, E), p, 0.5, 0.4), "scale": scale, "eps": 1e-5}}


PARAMETERS = ("weight", "bias", "post_weight", "post_bias")


@pytest.mark.parametrize("E", [520, 4096, 8191, 8200, 16384, 16392])
@pytest.mark.parametrize("T", [1, 5, 300])
def test_norm_with_one_parameter(on_card, E, T):
    """Each of the four parameter arrays without the others, in either type, beside a bf16 stream and branch."""
    for params in ("f32", "bf16"):
        for keep in PARAMETERS:
            for y, post in ((None, False), ("bf16", False), ("bf16", True)):
                if keep.startswith("post") and not post:
                    continue
                s = norm_inputs(E + T, T, E, "layer", "bf16", y, params, post, None, 0.5)
                for k in PARAMETERS:
                    if k != keep:
                        s["args"][k] = None
                ops.check_forward(s, f"{keep} {params} {y} {post}")
                ops.check_backward(s, f"{keep} {params} {y} {post}")


@pytest.mark.parametrize("T", [1, 2, 6, 600])
@pytest.mark.parametrize("kind,post", [("rms", False), ("layer", True)])
def test_norm_gate_of_one_row_for_all_tokens_by_its_strides(on_card, T, kind, post):
    """A [T, width] gate whose rows are one row in memory: its gradient is that of the same gate with rows of its own."""
    for params, E in (("bf16", 72), ("f32", 131), ("bf16", 2048)):
        s = norm_inputs(T + E, T, E, kind, "bf16", "bf16", params, post, "vector", 0.7)
        s["args"]["gate"] = s["args"]["gate"].expand(T, E)
        ops.check_forward(s, f"{E} {params}")
        ops.check_backward(s, f"{E} {params}")
        s["args"]["gate"] = s["args"]["gate"][:1].clone().expand(T, E)
        ops.check_backward(s, f"{E} {params}, one row expanded")


def test_linear_keeps_nan_before_a_relu():
    """A NaN sum stays NaN through every activation, in every kernel; the other rows are as without it."""
    for b in (16, 32, 64, 128):
        packed, dense = ops.matrix(b, 4 * b, 3 * b, b, 0.6)
        rows, cols = dense.shape
        bias = ops.rand(1, (rows,)).to(DEV)
        bad = bias.clone()
        bad[5], bad[rows - 1] = float("nan"), float("nan")
        for T in (1, 20, 40, 300, 1030):
            x = ops.rand(T, (T, cols), torch.bfloat16).to(DEV)
            for act in ("relu", "gelu", "silu"):
                for layout in (api.TOKEN_MAJOR, api.FEATURE_MAJOR):
                    xl = x if layout == api.TOKEN_MAJOR else torch.empty((cols, T), dtype=x.dtype, device=DEV).copy_(x.t())
                    for out in (torch.float32, torch.bfloat16):
                        call = lambda v: api.bsr_linear(packed, xl, bias=v, act=act, layout=layout, out_dtype=out)  # noqa: E731
                        got, want = call(bad), call(bias).clone()
                        if layout == api.FEATURE_MAJOR:
                            got, want = got.t(), want.t()
                        assert torch.isnan(got[:, 5]).all() and torch.isnan(got[:, -1]).all(), (b, T, act, layout)
                        want[:, 5], want[:, -1] = float("nan"), float("nan")
                        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want)), (b, T, act, layout)


@pytest.mark.parametrize("T", [1, 70, 700])
def test_act_backward_keeps_nan(T):
    """What the activation of a NaN enters is NaN; relu' of it is 0, as of everything that is not positive."""
    N = 264
    z, u = ops.rand(1, (T, N), torch.bfloat16).to(DEV), ops.rand(2, (T, N), torch.bfloat16).to(DEV)
    dy = ops.rand(3, (T, N)).to(DEV)
    bad = z.clone()
    bad[T - 1, 17], bad[0, 263] = float("nan"), float("nan")
    at = torch.isnan(bad)
    for act in ("relu", "gelu", "silu"):
        for sums in (False, True):
            clean, got = (api.gated_act_backward(v, u, dy, act=act, bias_grad=sums) for v in (z, bad))
            for k in ("dU", "H", "dG"):
                g, c = getattr(got, k), getattr(clean, k)
                assert torch.equal(g[~at], c[~at]), (act, k)
                if act == "relu" and k == "dG":
                    assert not g[at].any()
                else:
                    assert torch.isnan(g[at]).all(), (act, k)
            one = api.act_backward(bad, dy, act=act, bias_grad=sums)
            assert torch.isnan(one.dZ[at]).all() if act != "relu" else not one.dZ[at].any()


@pytest.mark.parametrize("T,N", [(1, (1 << 29) + 72), (65, (1 << 27) + 72)])
def test_act_backward_sums_of_more_columns_than_a_launch_has_owners(T, N):
    """The gradient of a bias alone: small whole numbers, whose sums are exact."""
    dy = torch.randint(-3, 4, (1, N), generator=torch.Generator(DEV).manual_seed(T), device=DEV, dtype=torch.int8)
    want = dy[0].float() * (1 if T == 1 else T - 2)  # (of T rows one is taken away again)
    dy = dy.bfloat16().repeat(T, 1)
    if T > 1:
        dy[T // 2] *= -1
    got = torch.full((N,), float("nan"), device=DEV)
    api._act_backward(None, None, dy, None, None, None, None, got, None)
    assert torch.equal(got, want)


LOOP_WIDTHS = [2051, 2056, 4096, 8191, 8192, 8200, 12000, 16384, 16392, 20001, 32768]
LOOP_CASES = [("bf16", None, "bf16", False, None), ("f32", None, "f32", False, None), ("bf16", "bf16", "bf16", False, "tokens"),
              ("bf16", "bf16", "bf16", True, "vector"), ("bf16", "bf16", "bf16", True, "tokens"), ("f32", "bf16", "bf16", True, "vector"),
              ("f32", "f32", "f32", True, "tokens"), ("f32", "f32", "f32", False, "vector")]


@pytest.mark.parametrize("E", LOOP_WIDTHS)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_backward_over_many_rows(on_card, E, kind):
    """Workgroups that go over several rows, the last of them over fewer: every width class beyond 2048 features, with and without
    wide access, operands all in 16 bits and not, and every part of the branch."""
    for k, case in enumerate(LOOP_CASES):
        ops.check_backward(norm_inputs(E + k, 515 if k % 2 else 771, E, kind, *case, 0.5), f"{E} {case}", with_dh=k != 1)


@pytest.mark.parametrize("E", [8191, 8200, 12000, 16384, 16392, 20001, 32768])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_over_many_rows(on_card, E, kind):
    """The same of the forward call, whose workgroups go over the rows beyond 8192 features and 256 rows."""
    for k, case in enumerate(LOOP_CASES):
        ops.check_forward(norm_inputs(E + k, 257 if k % 2 else 600, E, kind, *case, 0.5), f"{E} {case}")


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("T,E", [(7, 72), (300, 1600), (600, 2048), (520, 4096), (520, 16384)])
@pytest.mark.parametrize("post,gate", [(False, None), (False, "tokens"), (True, "vector")])
def test_norm_forward_then_backward_on_a_rounded_stream(kind, T, E, post, gate):
    """Both calls in a row on a bf16 stream, as a training step makes them, against the derivative of the whole step in 64 bits.

    The forward call's statistics are those of the stream h' before it is rounded, the backward call normalises the stored one: its n is
    off by n_off = 2^-8 |h'| r (and 64 u of the row in fp32).  With dn = dx * weight, first order (1 % is added for the second):
      dh is off by r (n_off mean |dn n| + |n| mean(|dn| n_off)), and by 64 u of the terms' sizes;
      what is linear in dh is off by the same formula with sizes in place of values; dweight by sum_t |dx| n_off.
    dh itself is rounded to bf16 when it is stored; dy and the sums come of the unrounded values."""
    s = norm_inputs(T + E, T, E, kind, "bf16", "bf16", "f32", post, gate, 0.7)
    a = s["args"]
    h_new, x, stats = api.norm_residual(s["h"], s["y"], with_stats=True, **a)
    g = api.norm_residual_backward(h_new, s["y"], stats, s["dx"], s["dh"], **a)
    v = {k: s[k].double().requires_grad_() for k in ("h", "y")}
    v.update({k: a[k].double().requires_grad_() for k in PARAMETERS + ("gate",) if a[k] is not None})
    m, r_y, p = None, None, v["y"]
    if post:
        p, m, _, r_y = ops.norm64(v["y"], kind, a["eps"], v["post_weight"], v.get("post_bias"))
    h64 = v["h"] + a["scale"] * (p * v["gate"] if "gate" in v else p)
    x64, n, _, r = ops.norm64(h64, kind, a["eps"], v["weight"], v.get("bias"))
    loss = (x64 * s["dx"].double()).sum() + (h64 * s["dh"].double()).sum()
    want = dict(zip(v, torch.autograd.grad(loss, list(v.values()))))
    with torch.no_grad():
        top, mean = (lambda t: t.abs().max(1, keepdim=True).values), (lambda t: t.mean(1, keepdim=True))
        n, h64, p = n.abs(), h64.abs(), p.abs()
        n_off = 2.0 ** -8 * h64 * r + 64 * U * (top(h64) * r + 1)
        dn = (s["dx"].double() * v["weight"]).abs()
        fp32 = 64 * U * (r * (dn + n * mean(dn * n) + mean(dn)) + s["dh"].double().abs())
        dh_off = 1.01 * r * (n_off * mean(dn * n) + n * mean(dn * n_off)) + fp32
        dh = want["h"].abs()
        close(g.dh, want["h"], dh_off, "dh")
        col = lambda off, size: off.sum(0) + U * (T + 64) * size.sum(0)  # noqa: E731
        close(g.dweight, want["weight"], col(s["dx"].double().abs() * n_off * 1.01, s["dx"].double().abs() * n), "dweight")
        if kind == "layer":
            close(g.dbias, want["bias"], col(0 * n, s["dx"].double().abs()), "dbias")
        gate_size = v["gate"].abs() if gate else torch.ones(1, dtype=torch.float64, device=DEV)
        dp, dp_off = 0.7 * gate_size * dh, 0.7 * gate_size * dh_off
        if gate:
            p_off = 64 * U * ((top(v["y"]) * r_y + 1) * v["post_weight"].abs() + p) if post else 4 * U * p
            one_off, one = 0.7 * (dh_off * p + dh * p_off), 0.7 * dh * p
            close(g.dgate, want["gate"], col(one_off, one) if gate == "vector" else one_off + 4 * U * one, "dgate")
        if not post:
            close(g.dy, want["y"], dp_off + 4 * U * dp, "dy")
            return
        m, m_off = m.abs(), 64 * U * (top(v["y"]) * r_y + 1)
        close(g.dpost_weight, want["post_weight"], col(dp_off * m + dp * m_off, dp * (m + 1)), "dpost_weight")
        if kind == "layer":
            close(g.dpost_bias, want["post_bias"], col(dp_off, dp), "dpost_bias")
        w = v["post_weight"].abs()
        through = lambda d: d + m * mean(d * m) + (mean(d) if kind == "layer" else 0)  # noqa: E731
        off = through(dp_off * w) + m_off * mean(dp * w * m) + m * mean(dp * w * m_off) + 64 * U * through(dp * w)
        close(g.dy, want["y"], 1.01 * r_y * off, "dy")


def test_linear_without_an_epilogue_is_the_product():
    """bsr_linear with nothing in its epilogue multiplies as bsr_spmm does, in the same order: bit for bit, where rows are not cut."""
    for b in (16, 32, 64, 128):
        packed, dense = ops.matrix(b, 6 * b, 4 * b, b, 0.5)
        for T in (1, 16, 40, 300, 1030):
            x = ops.rand(T, (T, 4 * b), torch.bfloat16).to(DEV)
            got, want = (f(packed, x, out_dtype=torch.bfloat16) for f in (api.bsr_linear, api.bsr_spmm))
            assert torch.equal(got, want), (b, T)
