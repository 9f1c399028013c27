"""Sums of the products on scaled 8-bit tensors: held in 32 bits whatever is made of them, in every form of the kernels.

Forms: up to 128 pairs of a block row and 32 tokens by 32 rows (no 8-bit result asked for), more by whole block rows, many 128-token tiles by
lists of them.  A bf16 result is the fp32 one rounded, bit for bit: both come from the same sums.
"""
import pytest
import torch

from paper_2507_03117_amd import api
from tests import scaled8_reference as ref
from tests.test_gpu_scaled8 import BF16, F32, Matrix, activation, close, close8, eight, gen, masks

pytestmark = pytest.mark.gpu

# (block rows, tokens): parts of block rows, whole ones, tiles
FORMS = {"parts": (4, 40), "rows": (20, 300), "tiles": (25, 2100)}


@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
def test_terms_beside_larger_ones_that_cancel(b, form):
    """Two strong features whose products cancel beside weak ones: 448 w, -448 w and 2^-9 w, w = 1.  Every partial sum is a multiple of 2^-9 below
    3 * 448 + 1 < 2^11, three blocks a row: 20 bits, so that the sum of the weak ones is exact in 32 bits, in any order."""
    nr, T = FORMS[form]
    nc = 3
    ones = api.bsr_quantize_scaled8(api.bsr_pack(torch.ones((nr * b, nc * b), dtype=BF16, device="cuda"), b,
                                                 mask=torch.ones((nr, nc), dtype=torch.uint8, device="cuda")))
    x = torch.full((T, nc * b), 2.0 ** -9)
    g = gen(b)
    for c in range(nc):  # the strong two anywhere in a block
        two = torch.stack([torch.randperm(b, generator=g)[:2] + c * b for _ in range(T)])
        x.scatter_(1, two[:, :1], 448.0)
        x.scatter_(1, two[:, 1:], -448.0)
    q = api.quantize_scaled8(x.cuda(), group=b)
    assert torch.equal(api.dequantize_scaled8(q, out_dtype=F32).cpu(), x)
    want = torch.full((T, nr * b), nc * (b - 2) * 2.0 ** -9).cuda()
    assert torch.equal(api.bsr_linear_scaled8(ones, q), want)
    assert torch.equal(api.bsr_linear_scaled8(ones, q, out_dtype=BF16), want.to(BF16))
    assert torch.equal(api.bsr_gated_scaled8(ones, ones, q, act=None, out_fmt=None).H, (want * want).to(BF16))


@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("wfmt,xfmt", [("e4m3", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("bias,act,residual,kept", [(False, None, None, False), (True, "gelu", "bf16", False), (True, "silu", "f32", True)])
def test_bf16_results_are_the_fp32_ones_rounded(b, form, wfmt, xfmt, bias, act, residual, kept):
    nr, T = FORMS[form]
    g = gen(b + T)
    m = Matrix(g, masks(nr, 3, 5, 0.6), b, wfmt)
    q, x = eight(activation(g, T, m.cols, 0.3), b, xfmt)
    kw = {"act": act}
    if bias:
        kw["bias"] = torch.randn((m.rows,), generator=g).cuda()
    if residual:
        kw["residual"] = torch.randn((T, m.rows), generator=g).to(F32 if residual == "f32" else BF16).cuda()
    y = api.bsr_linear_scaled8(m.w8, q, **kw)
    assert torch.equal(api.bsr_linear_scaled8(m.w8, q, out_dtype=BF16, **kw), y.to(BF16))
    if kept:  # what is kept beside it changes nothing
        pre = api.empty_scaled8(T, m.rows, group=b)
        assert torch.equal(api.bsr_linear_scaled8(m.w8, q, out_dtype=BF16, pre=pre, **kw), y.to(BF16))
    if not bias:
        z, wide, _ = m.product(x)
        close(y, z, wide + 2.0 ** -24 * z.abs())


@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("wfmt,xfmt,act", [("e4m3", "e4m3", "silu"), ("e4m3", "e5m2", "gelu"), ("e5m2", "e4m3", "relu"), ("e5m2", "e5m2", None)])
def test_gated_bf16_results(b, form, wfmt, xfmt, act):
    """Against 64 bits with the bound of sums in 32 bits, and the same bits whether the two products are kept or not."""
    nr, T = FORMS[form]
    g = gen(b + T)
    mg, mu = (Matrix(g, masks(nr, 3, s, 0.6), b, wfmt) for s in (1, 2))
    q, x = eight(activation(g, T, mg.cols, 0.3), 128, xfmt)
    h = api.bsr_gated_scaled8(mg.w8, mu.w8, q, act=act, out_fmt=None).H
    kept = api.bsr_gated_scaled8(mg.w8, mu.w8, q, act=act, out_fmt=None, keep=True)
    assert torch.equal(h, kept.H)
    (zg, og, _), (zu, ou, _) = mg.product(x), mu.product(x)
    a = ref.act(act, zg)
    want = a * zu
    off = (1.13 * og + 2.0 ** -20 * zg.abs()) * (zu.abs() + ou) + a.abs() * ou + 2.0 ** -23 * want.abs()
    close(h, want, off + 2.0 ** -8 * (want.abs() + off))


@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("T", [5, 300, 4200])
def test_no_term_of_a_long_row_is_lost(b, T):
    """Rows of 70 blocks.  A sum is made of at most 70 b / 16 + 7 additions of instructions and waves to a partial sum, each off by 2^-23 of that at
    most; partial sums of random terms are in their root mean square no larger than the whole.  2^-8 / sqrt(3) is more than the root mean square of bf16's
    rounding.  A single feature left out would be sqrt(1 / (70 b)) of the sum, 0.01, and in bf16 results too more than that."""
    g = gen(b)
    mask = torch.ones((8, 70), dtype=torch.uint8)
    mask[5] = 0
    m = Matrix(g, mask, b, "e4m3", std=0.01)
    q, x = eight(torch.randn((T, m.cols), generator=g), b, "e4m3")
    z, _, _ = m.product(x)
    y = api.bsr_linear_scaled8(m.w8, q)
    rel = lambda v, w: float((v.double().cpu() - w).norm() / w.norm())  # noqa: E731
    off = (70 * b / 16 + 7) * 2.0 ** -23
    assert rel(y, z) <= off
    low = api.bsr_linear_scaled8(m.w8, q, out_dtype=BF16)
    assert torch.equal(low, y.to(BF16))
    assert rel(low, z) <= off + 2.0 ** -8 / 3 ** 0.5


@pytest.mark.parametrize("b,T", [(64, 90), (64, 1), (128, 40)])
def test_kept_intermediate_of_the_forward_pass(b, T):
    """H, G and U of a gated block whose weights differ, against 64 bits."""
    g = gen(5)
    mg, mu = (Matrix(g, masks(4, 5, s), b, "e4m3") for s in (1, 2))
    q, x = eight(activation(g, T, mg.cols, 0.3), b, "e4m3")
    r = api.bsr_gated_scaled8(mg.w8, mu.w8, q, keep=True)
    (zg, og, _), (zu, ou, _) = mg.product(x), mu.product(x)
    close8(r.G, zg, og, "G")
    close8(r.U, zu, ou, "U")
    a = ref.act("silu", zg)
    h = a * zu
    close8(r.H, h, (1.13 * og + 2.0 ** -20 * zg.abs()) * (zu.abs() + ou) + a.abs() * ou + 2.0 ** -23 * h.abs(), "H")
