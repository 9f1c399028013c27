"""Host-side checks of the operators around the MLP: every refusal comes before the GPU is touched."""
import ctypes as C

import pytest

from paper_2507_03117_amd import api

F32, BF16 = api.F32, api.BF16
BUF = (C.c_int64 * 64)()  # (stands in for device pointers: no call below gets as far as using them)
P = C.cast(BUF, C.c_void_p)
P16 = C.c_void_p((P.value + 15) // 16 * 16)


def matrix(rows=128, cols=128, b=64, nnz=0):
    ptr = C.cast(BUF, C.c_void_p)
    return api.BsrView(rows, cols, b, 0, nnz, ptr, ptr if nnz else None, None, None, None)


def linear(v=None, X=P, ldx=128, layout=0, T=4, bias=None, act=-1, R=None, ldr=128, rt=F32, Y=P, ldy=128, yt=F32, Z=None, ldz=128):
    v = matrix() if v is None else v
    return api.lib().blast_bsr_linear(C.byref(v), X, ldx, layout, T, bias, act, R, ldr, rt, Y, ldy, yt, Z, ldz, None, 0, None)


def test_linear_refusals():
    assert api.lib().blast_bsr_linear(None, P, 128, 0, 4, None, -1, None, 0, 0, P, 128, 0, None, 0, None, 0, None) == -1
    assert linear(matrix(100, 128)) == -2
    assert linear(matrix(96, 96, 48)) == -3
    assert linear(matrix(nnz=1)) == -1  # blocks without values
    assert linear(X=None) == -1 and linear(Y=None) == -1
    assert linear(ldx=127) == -1 and linear(ldy=127) == -1
    assert linear(layout=2) == -1 and linear(layout=-1) == -1
    assert linear(T=-1) == -1 and linear(T=1 << 31) == -1
    assert linear(act=-2) == -1 and linear(act=3) == -1
    assert linear(yt=2) == -1
    assert linear(R=P, rt=7) == -1 and linear(R=P, ldr=127) == -1
    assert linear(Z=P, ldz=127) == -1
    assert linear(layout=1, ldx=3) == -1  # feature-major rows hold T values
    assert linear(T=0, X=None, Y=None) == 0  # no token: nothing to do
    assert linear(matrix(rows=0)) == 0


def act(Z=P, ldz=64, U=None, ldu=64, dY=P, lddy=64, t=F32, T=4, N=64, a=0, dZ=P, lddz=64, dU=None, lddu=64, H=None, ldh=64, dbz=None,
        dbu=None, ws=None, wsb=0):
    return api.lib().blast_act_backward(Z, ldz, U, ldu, dY, lddy, t, T, N, a, dZ, lddz, dU, lddu, H, ldh, dbz, dbu, ws, wsb, None)


def test_act_backward_refusals():
    assert act(T=-1) == -1 and act(N=-1) == -1 and act(T=1 << 31) == -1 and act(N=1 << 31) == -1
    assert act(a=-2) == -1 and act(a=3) == -1 and act(t=2) == -1
    assert act(dY=None) == -1 and act(lddy=63) == -1
    assert act(Z=None) == -1 and act(Z=None, a=-1, U=P) == -1
    assert act(ldz=63) == -1 and act(U=P, ldu=63) == -1 and act(lddz=63) == -1
    assert act(U=P, dU=P, lddu=63) == -1 and act(U=P, H=P, ldh=63) == -1
    assert act(dU=P) == -1 and act(H=P) == -1 and act(dbu=P) == -1  # not gated
    need = C.c_size_t(0)
    ask = api.lib().blast_act_backward_workspace
    assert ask(4096, 64, 1, C.byref(need)) == 0 and need.value > 0
    assert act(T=4096, dbz=P) == -5 and act(T=4096, dbz=P, ws=P16, wsb=need.value - 1) == -5
    assert act(T=4096, dbz=P, ws=C.c_void_p(P16.value + 4), wsb=need.value) == -5
    two = C.c_size_t(0)
    assert ask(4096, 64, 2, C.byref(two)) == 0 and two.value == 2 * need.value
    assert ask(4096, 64, 0, C.byref(need)) == 0 and need.value == 0
    assert ask(0, 64, 2, C.byref(need)) == 0 and need.value == 0
    assert ask(-1, 64, 1, C.byref(need)) == -1 and ask(1, -1, 1, C.byref(need)) == -1
    assert ask(1, 1, 3, C.byref(need)) == -1 and ask(1, 1, 1, None) == -1
    assert act(T=0) == 0 and act(N=0, ldz=0) == 0


def view(width=64, kind=0, post=0, eps=1e-5, pt=F32, gt=F32, weight=None, bias=None, pw=None, pb=None, gate=None, ldg=0):
    return api.NormView(width, kind, post, eps, 1.0, pt, gt, weight, bias, pw, pb, gate, ldg)


def forward(v, h=P, ldh=64, ht=F32, y=None, ldy=64, yt=F32, T=4, ho=None, ldho=64, x=P, ldx=64, xt=BF16, stats=None):
    return api.lib().blast_norm_residual(C.byref(v), h, ldh, ht, y, ldy, yt, T, ho, ldho, x, ldx, xt, stats, None)


def backward(v, h=P, ldh=64, ht=F32, y=None, ldy=64, yt=F32, stats=P16, dx=P, lddx=64, dxt=BF16, dho=None, lddho=64, T=4, dh=P, lddh=64,
             dy=None, lddy=64, dyt=BF16, dg=None, lddg=64, dw=None, db=None, dpw=None, dpb=None, ws=None, wsb=0):
    return api.lib().blast_norm_residual_backward(C.byref(v), h, ldh, ht, y, ldy, yt, stats, dx, lddx, dxt, dho, lddho, T, dh, lddh, dy,
                                                  lddy, dyt, dg, lddg, dw, db, dpw, dpb, ws, wsb, None)


BAD_VIEWS = [dict(width=0), dict(width=-8), dict(width=32769), dict(kind=2), dict(kind=-1), dict(post=2), dict(eps=-1.0),
             dict(eps=float("nan")), dict(pt=2), dict(gt=-1), dict(kind=0, bias=P), dict(kind=0, post=1, pb=P)]


@pytest.mark.parametrize("bad", BAD_VIEWS)
def test_norm_refuses_bad_views(bad):
    need = C.c_size_t(0)
    assert forward(view(**bad)) == -1 and backward(view(**bad)) == -1
    assert api.lib().blast_norm_residual_backward_workspace(C.byref(view(**bad)), 4, C.byref(need)) == -1


def test_norm_refusals():
    L = api.lib()
    assert L.blast_norm_residual(None, P, 64, 0, None, 0, 0, 4, None, 0, P, 64, 1, None, None) == -1
    v = view()
    assert forward(v, h=None) == -1 and forward(v, x=None) == -1 and forward(v, ldh=63) == -1 and forward(v, ldx=63) == -1
    assert forward(v, ht=2) == -1 and forward(v, xt=2) == -1 and forward(v, y=P, ho=P, yt=5) == -1
    assert forward(v, T=-1) == -1 and forward(v, T=1 << 31) == -1
    assert forward(v, y=P) == -1  # nowhere to put the stream
    assert forward(v, y=P, ho=P, ldy=63) == -1 and forward(v, y=P, ho=P, ldho=63) == -1
    assert forward(v, stats=C.c_void_p(P16.value + 4)) == -1
    assert forward(view(gate=P, ldg=63), y=P, ho=P) == -1
    assert forward(v, T=0, h=None, x=None) == 0


def test_norm_backward_refusals():
    v = view()
    assert backward(v, h=None) == -1 and backward(v, dx=None) == -1 and backward(v, dh=None) == -1
    assert backward(v, ldh=63) == -1 and backward(v, lddx=63) == -1 and backward(v, lddh=63) == -1
    assert backward(v, dho=P, lddho=63) == -1 and backward(v, y=P, ldy=63) == -1 and backward(v, y=P, dy=P, lddy=63) == -1
    assert backward(v, ht=2) == -1 and backward(v, dxt=2) == -1 and backward(v, y=P, yt=2) == -1 and backward(v, y=P, dy=P, dyt=3) == -1
    assert backward(v, stats=None) == -1 and backward(v, stats=C.c_void_p(P16.value + 8)) == -1
    assert backward(v, T=-1) == -1
    # gradients of what is not there
    assert backward(v, dy=P) == -1 and backward(v, dg=P) == -1 and backward(v, dpw=P) == -1 and backward(v, dpb=P) == -1
    assert backward(v, y=P, dg=P) == -1 and backward(v, y=P, dpw=P) == -1 and backward(v, db=P) == -1
    assert backward(view(post=1), y=P, dpb=P) == -1
    assert backward(view(gate=P, ldg=64), y=P, dg=P, lddg=63) == -1
    need = C.c_size_t(0)
    ask = api.lib().blast_norm_residual_backward_workspace
    sizes = []
    for w in (v, view(kind=1), view(post=1), view(kind=1, post=1), view(kind=1, post=1, gate=P)):
        assert ask(C.byref(w), 4096, C.byref(need)) == 0
        sizes.append(need.value)
    assert sizes[1] == sizes[2] == 2 * sizes[0] and sizes[3] == 4 * sizes[0] and sizes[4] == 5 * sizes[0] and sizes[0] > 0
    assert ask(C.byref(view(gate=P, ldg=64)), 4096, C.byref(need)) == 0 and need.value == sizes[0]  # a gate per token has no sum
    assert ask(C.byref(v), 0, C.byref(need)) == 0 and need.value == 0
    assert ask(C.byref(v), -1, C.byref(need)) == -1 and ask(C.byref(v), 4, None) == -1
    assert backward(v, T=4096, dw=P) == -5 and backward(v, T=4096, dw=P, ws=P16, wsb=sizes[0] - 1) == -5
    assert backward(v, T=4096, dw=P, ws=C.c_void_p(P16.value + 4), wsb=sizes[0]) == -5
    assert backward(v, T=0, h=None, dx=None, dh=None) == 0  # no rows, no sums asked for


@pytest.mark.parametrize("T", [1, 2, 255, 256, 257, 100000])
def test_norm_workspace_never_shrinks_with_the_tokens(T):
    need, more = C.c_size_t(0), C.c_size_t(0)
    ask = api.lib().blast_norm_residual_backward_workspace
    assert ask(C.byref(view()), T, C.byref(need)) == 0 and ask(C.byref(view()), T + 1, C.byref(more)) == 0
    assert more.value >= need.value
