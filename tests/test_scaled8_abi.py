"""Host-side checks of the operators on scaled 8-bit tensors: every refusal comes before the GPU is touched; and the reference that the
GPU tests compare with, against torch's own conversions."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2507_03117_amd import api
from tests import scaled8_reference as ref

F32, BF16 = api.F32, api.BF16
BUF = (C.c_int64 * 64)()  # (stands in for device pointers: no call below gets as far as using them)
P = C.c_void_p((C.addressof(BUF) + 15) // 16 * 16)
ODD = C.c_void_p(P.value + 1)


def matrix(rows=128, cols=128, b=64, nnz=1):
    return api.BsrView(rows, cols, b, 0, nnz, P, P if nnz else None, P, None, None)


def weight(vals=P, scales=P, fmt=0):
    return api.Weight8View(vals, scales, fmt)


def eight(codes=P, ld=128, scales=P, lds=16, fmt=0, group=64):
    return api.Scaled8View(codes, ld, scales, lds, fmt, group)


BAD_EIGHT = [{"codes": None}, {"scales": None}, {"ld": 127}, {"lds": 15}, {"lds": 24}, {"fmt": 2}, {"fmt": -1}, {"group": 32}, {"group": 0},
             {"scales": ODD}]


def quantise(X=P, ldx=128, t=F32, T=4, K=128, out=None):
    return api.lib().blast_quantize_scaled8(X, ldx, t, T, K, C.byref(eight() if out is None else out), None)


def dequantise(X=None, T=4, K=128, Y=P, ldy=128, t=F32):
    return api.lib().blast_dequantize_scaled8(C.byref(eight() if X is None else X), T, K, Y, ldy, t, None)


def test_quantiser_refusals():
    L = api.lib()
    for bad in ({"X": None}, {"ldx": 127}, {"t": 2}, {"T": -1}, {"K": -1}, {"T": 1 << 31}, {"K": 1 << 31}, {"T": 17}):
        assert quantise(**bad) == -1, bad
    for bad in ({"Y": None}, {"ldy": 127}, {"t": 2}, {"T": -1}, {"K": -1}, {"T": 17}):
        assert dequantise(**bad) == -1, bad
    for bad in BAD_EIGHT:
        assert quantise(out=eight(**bad)) == -1 and dequantise(eight(**bad)) == -1, bad
    assert L.blast_quantize_scaled8(P, 128, F32, 4, 128, None, None) == -1
    assert L.blast_dequantize_scaled8(None, 4, 128, P, 128, F32, None) == -1
    assert quantise(T=0, X=None) == 0 and quantise(K=0, X=None) == 0 and dequantise(T=0, Y=None) == 0
    assert quantise(T=0, out=eight(codes=None, scales=None)) == 0
    # more workgroups than a launch has
    assert quantise(T=(1 << 30) - 1, K=1 << 20, ldx=1 << 20, out=eight(ld=1 << 20, lds=1 << 30)) == -1

    def blocks(v=None, fmt=0, codes=P, scales=P):
        return L.blast_bsr_quantize_scaled8(C.byref(matrix() if v is None else v), fmt, codes, scales, None)

    assert L.blast_bsr_quantize_scaled8(None, 0, P, P, None) == -1
    assert blocks(fmt=2) == -1 and blocks(codes=None) == -1 and blocks(scales=None) == -1 and blocks(codes=ODD) == -1 and blocks(scales=ODD) == -1
    assert blocks(matrix(b=32)) == -3 and blocks(matrix(b=16)) == -3
    assert blocks(matrix(nnz=0), codes=None, scales=None) == 0
    bad = matrix()
    bad.vals = None
    assert blocks(bad) == -1


def linear(v=None, w=None, x=None, T=4, bias=None, act=-1, R=None, ldr=128, rt=F32, Y=P, ldy=128, yt=F32, Y8=None, Z8=None):
    ref_ = lambda s: None if s is None else C.byref(s)  # noqa: E731
    return api.lib().blast_bsr_linear_scaled8(C.byref(matrix() if v is None else v), C.byref(weight() if w is None else w),
                                              C.byref(eight() if x is None else x), T, bias, act, R, ldr, rt, Y, ldy, yt, ref_(Y8),
                                              ref_(Z8), None)


def gated(vg=None, wg=None, vu=None, wu=None, x=None, T=4, act=0, H=P, ldh=128, H8=None, G8=None, U8=None):
    ref_ = lambda s: None if s is None else C.byref(s)  # noqa: E731
    one = lambda s, d: C.byref(d if s is None else s)  # noqa: E731
    return api.lib().blast_bsr_gated_scaled8(one(vg, matrix()), one(wg, weight()), one(vu, matrix()), one(wu, weight()), one(x, eight()), T,
                                             act, H, ldh, ref_(H8), ref_(G8), ref_(U8), None)


@pytest.mark.parametrize("call", [linear, lambda v=None, w=None, **k: gated(vg=v, wg=w, **k), lambda v=None, w=None, **k: gated(vu=v, wu=w, **k)])
def test_product_refusals(call):
    assert call(matrix(100, 128)) == -2 and call(matrix(128, 100)) == -2
    for b in (16, 32, 48):
        assert call(matrix(96, 96, b)) == -3
    bad = matrix()
    bad.row_ptr = None
    assert call(bad) == -1
    bad = matrix()
    bad.col_idx = None
    assert call(bad) == -1
    for w in (weight(None), weight(ODD), weight(scales=None), weight(scales=ODD), weight(fmt=2), weight(fmt=-1)):
        assert call(w=w) == -1
    for kw in BAD_EIGHT + [{"codes": ODD}, {"ld": 136}]:
        assert call(x=eight(**kw)) == -1, kw
    assert call(T=-1) == -1 and call(T=1 << 31) == -1 and call(T=17) == -1
    assert call(act=-2) == -1 and call(act=3) == -1
    assert call(T=0, x=eight(codes=None, scales=None)) == 0
    for name in (("Y8", "Z8") if call is linear else ("G8", "U8")):
        for kw in BAD_EIGHT + [{"codes": ODD}, {"ld": 136}, {"group": 128}]:
            assert call(**{name: eight(**kw)}) == -1, (name, kw)


def test_linear_refusals():
    assert linear(Y=None) == -1 and linear(ldy=127) == -1 and linear(yt=2) == -1
    assert linear(R=P, rt=2) == -1 and linear(R=P, ldr=127) == -1
    big = matrix(256, 256, 128)
    assert linear(big, x=eight(ld=256, group=64), ldy=256) == -1  # groups smaller than a block
    L = api.lib()
    assert L.blast_bsr_linear_scaled8(None, None, None, 4, None, -1, None, 0, 0, P, 128, 0, None, None, None) == -1
    assert L.blast_bsr_linear_scaled8(C.byref(matrix()), C.byref(weight()), None, 4, None, -1, None, 0, 0, P, 128, 0, None, None, None) == -1


def test_gated_refusals():
    assert gated(H=None) == -1 and gated(ldh=127) == -1
    assert gated(H8=eight()) == -1  # both forms of H
    assert gated(vu=matrix(256, 128)) == -2 and gated(vu=matrix(128, 256)) == -2 and gated(vu=matrix(128, 128, 128)) == -2
    assert gated(wu=weight(fmt=1)) == -1


def test_gradient_refusals():
    L = api.lib()

    def grad(v=None, dY=P, ldy=128, x=None, T=4, out=P, ws=None, wsb=0):
        return L.blast_bsr_sddmm_scaled8(C.byref(matrix() if v is None else v), dY, ldy, C.byref(eight() if x is None else x), T, out, ws,
                                         wsb, None)

    assert grad(matrix(100, 128)) == -2 and grad(matrix(96, 96, 32)) == -3
    assert grad(dY=None) == -1 and grad(ldy=127) == -1 and grad(ldy=132) == -1 and grad(dY=ODD) == -1
    assert grad(out=None) == -1 and grad(out=ODD) == -1 and grad(T=-1) == -1 and grad(T=1 << 31) == -1
    for kw in BAD_EIGHT + [{"codes": ODD}, {"ld": 136}]:
        assert grad(x=eight(**kw)) == -1, kw
    assert grad(matrix(256, 256, 128), x=eight(ld=256, group=64), ldy=256) == -1
    assert grad(matrix(nnz=0), out=None, dY=None) == 0
    need = C.c_size_t(0)
    ask = L.blast_bsr_sddmm_scaled8_workspace
    assert ask(C.byref(matrix()), 4096, C.byref(need)) == 0 and need.value > 0
    many = eight(lds=4096)
    assert grad(x=many, T=4096) == -5 and grad(x=many, T=4096, ws=P, wsb=need.value - 1) == -5 and grad(x=many, T=4096, ws=ODD, wsb=need.value) == -5
    assert ask(C.byref(matrix()), 4, C.byref(need)) == 0 and need.value == 0
    assert ask(C.byref(matrix()), 4, None) == -1 and ask(None, 4, C.byref(need)) == -1 and ask(C.byref(matrix()), -1, C.byref(need)) == -1
    assert ask(C.byref(matrix(96, 96, 32)), 4, C.byref(need)) == -3


def test_activation_gradient_refusals():
    def act(Z=None, U=None, dY=P, lddy=128, t=F32, T=4, N=128, a=0, dZ=P, lddz=128, dU=None, lddu=128, H=None, ldh=128, dbz=None, dbu=None,
            ws=None, wsb=0):
        return api.lib().blast_act_backward_scaled8(C.byref(eight() if Z is None else Z), None if U is None else C.byref(U), dY, lddy, t, T, N, a, dZ,
                                                    lddz, dU, lddu, H, ldh, dbz, dbu, ws, wsb, None)

    assert api.lib().blast_act_backward_scaled8(None, None, P, 128, F32, 4, 128, 0, P, 128, None, 0, None, 0, None, None, None, 0, None) == -1
    for kw in BAD_EIGHT:
        assert act(Z=eight(**kw)) == -1 and act(U=eight(**kw)) == -1, kw
    assert act(T=-1) == -1 and act(N=-1) == -1 and act(T=17) == -1 and act(a=-2) == -1 and act(a=3) == -1 and act(t=2) == -1
    assert act(dY=None) == -1 and act(lddy=127) == -1 and act(lddz=127) == -1
    assert act(dU=P) == -1 and act(H=P) == -1 and act(dbu=P) == -1  # not gated
    assert act(U=eight(), dU=P, lddu=127) == -1 and act(U=eight(), H=P, ldh=127) == -1
    assert act(Z=eight(lds=4096), T=4096, dbz=P) == -5
    assert act(T=0) == 0 and act(N=0) == 0


def test_sizes_of_a_scaled_tensor():
    q = api.empty_scaled8(5, 200, group=64, device="cpu")
    assert q.codes.shape == (5, 200) and q.codes.stride() == (208, 1) and q.scales.shape == (4, 16)
    q = api.empty_scaled8(33, 256, device="cpu")
    assert q.codes.is_contiguous() and q.scales.shape == (2, 48)


@pytest.mark.parametrize("fmt,dtype", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_reference_agrees_with_torch(fmt, dtype):
    t = torch.arange(256, dtype=torch.uint8).view(dtype).double().numpy()
    mine = ref.table(fmt)
    assert np.array_equal(np.isnan(t), np.isnan(mine)) and np.array_equal(t[~np.isnan(t)], mine[~np.isnan(t)])
    v = torch.cat([torch.randn(20000, generator=torch.Generator().manual_seed(1)) * 2.0 ** k for k in range(-12, 8)]).double()
    v = v[v.abs() <= ref.FORMATS[fmt][2]]
    assert np.array_equal(ref.encode(v.numpy(), fmt), v.float().to(dtype).view(torch.uint8).numpy()[:len(v)]) or \
        np.array_equal(mine[ref.encode(v.numpy(), fmt)], v.float().to(dtype).double().numpy())


def test_reference_exponent_by_brute_force():
    for fmt in ref.FORMATS:
        for m in [448.0, 448.0000001, 57344.0, 57345.0, 1.0, 1.75, 1.7500001, 0.875, 2.0 ** -126, 3e38, 2.0 ** -100]:
            want = next(e for e in range(-100, 130) if m <= ref.FORMATS[fmt][2] * 2.0 ** e)
            assert ref.exponent(m, fmt) == want and ref.exponents(np.array([m]), fmt)[0] == want
        assert ref.exponents(np.array([0.0]), fmt)[0] == -100


def test_reference_codes_by_hand():
    v = np.array([[0.0, 1.0, -1.0, 448.0], [464.0, -0.001, 0.0009765625, 0.00146484375]])
    assert ref.encode(v.clip(-448, 448), "e4m3").tolist() == [[0, 0x38, 0xB8, 0x7E], [0x7E, 0x81, 0, 1]]
