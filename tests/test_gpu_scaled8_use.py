"""Operators on scaled 8-bit tensors as a program uses them: together, captured and replayed, on several streams, at the sizes where counters
and offsets grow, and in the example network."""
import pytest
import torch

from examples.train_block import Network
from paper_2507_03117_amd import api
from tests import scaled8_reference as ref
from tests.test_gpu_scaled8 import BF16, F32, Matrix, activation, close, eight, gen, masks

pytestmark = pytest.mark.gpu


def plain_weight(g, nr, nc, b, keep=0.6):
    w = (torch.randn((nr * b, nc * b), generator=g) * 0.05).to(BF16)
    return api.bsr_pack(w.cuda(), b, mask=masks(nr, nc, nr + nc, keep).cuda())


@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("T", [5, 2560, 4200])
def test_rows_of_more_than_64_blocks(b, T):
    """Full rows of 70 blocks, an odd 67 and none, by waves that share them and by tiles."""
    g = gen(b)
    mask = torch.ones((8, 70), dtype=torch.uint8)
    mask[2, 3:6], mask[5] = 0, 0
    m = Matrix(g, mask, b, "e4m3", std=0.01)
    q, x = eight(activation(g, T, m.cols, 0.3), b, "e4m3")
    z, wide, low = m.product(x)
    close(api.bsr_linear_scaled8(m.w8, q), z, wide + 2.0 ** -24 * z.abs())
    close(api.bsr_linear_scaled8(m.w8, q, out_dtype=BF16), z, low + 2.0 ** -8 * (z.abs() + low))
    h = api.bsr_gated_scaled8(m.w8, m.w8, q, act=None, out_fmt=None).H
    off = 2 * low * (z.abs() + low)
    close(h, z * z, off + 2.0 ** -8 * (z * z + off))


@pytest.mark.parametrize("b", [64, 128])
def test_more_tiles_than_a_list_holds_at_once(b):
    """66000 tokens and 64 block rows: every workgroup has more than 64 tiles.  Each run of tokens gives what it gives by itself."""
    g = gen(b)
    T, cut = 66000, 8192
    w8 = api.bsr_quantize_scaled8(plain_weight(g, 64, 2, b))
    x = api.quantize_scaled8(torch.randn((T, 2 * b), generator=g).cuda(), group=b)
    y = api.bsr_linear_scaled8(w8, x, out_dtype=BF16)
    h = api.bsr_gated_scaled8(w8, w8, x)
    for t in list(range(0, T, cut))[::2]:
        n = min(cut, T - t)
        part = api.Scaled8(x.codes[t:t + n], x.scales[:, t:t + n + (-n) % 16].contiguous(), b, "e4m3")
        assert torch.equal(y[t:t + n], api.bsr_linear_scaled8(w8, part, out_dtype=BF16))
        hp = api.bsr_gated_scaled8(w8, w8, part)
        assert torch.equal(h.H.codes[t:t + n], hp.H.codes) and torch.equal(h.H.scales[:, t:t + n], hp.H.scales[:, :n])


def test_offsets_beyond_32_bits():
    """Codes, results and gradients whose last rows lie beyond 4 GiB."""
    b, T, K = 128, 300_000, 16384
    g = gen(3)
    mask = torch.zeros((1, K // b), dtype=torch.uint8)
    mask[0, [0, 77, K // b - 1]] = 1
    w = (torch.randn((b, K), generator=g) * 0.05).to(BF16)
    p = api.bsr_pack(w.cuda(), b, mask=mask.cuda())
    w8 = api.bsr_quantize_scaled8(p)
    x = torch.empty((T, K), dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    q = api.quantize_scaled8(x)
    tail = slice(T - 160, T)
    qt = api.quantize_scaled8(x[tail])
    assert torch.equal(q.codes[tail], qt.codes) and torch.equal(q.scales[:, tail], qt.scales)
    assert torch.equal(api.bsr_linear_scaled8(w8, q, out_dtype=BF16)[tail], api.bsr_linear_scaled8(w8, qt, out_dtype=BF16))
    assert torch.equal(api.dequantize_scaled8(q)[tail], api.dequantize_scaled8(qt))
    a = api.act_backward_scaled8(q, x, act="silu").dZ
    assert torch.equal(a[tail], api.act_backward_scaled8(qt, x[tail], act="silu").dZ)
    del a
    dy = torch.zeros((T, b), dtype=BF16, device="cuda")
    dy[tail] = 0.5
    assert torch.equal(api.bsr_sddmm_scaled8(p, dy, q), api.bsr_sddmm_scaled8(p, dy[tail].contiguous(), qt))


def chain(gate, up, down, down_t, w, x, dy, b):
    """Forward and backward pass of a gated block, as a training step runs it."""
    x8 = api.quantize_scaled8(x, group=b)
    inner = api.bsr_gated_scaled8(gate, up, x8, keep=True)
    y = api.bsr_linear_scaled8(down, inner.H, residual=x, out_dtype=F32)
    dh = api.bsr_linear_scaled8(down_t, api.quantize_scaled8(dy, group=b, fmt="e5m2"), out_dtype=BF16)
    through = api.gated_act_backward_scaled8(inner.G, inner.U, dh, bias_grad=True)
    return [y, inner.H.codes, inner.G.codes, inner.U.codes, dh, through.dG, through.dU, through.H, through.dbias_g, through.dbias_u,
            api.bsr_sddmm_scaled8(w, through.dG, x8), api.bsr_sddmm_scaled8(down.packed, dy, inner.H)]


def chain_inputs(b, T, seed=0):
    g = gen(b + T + seed)
    gate, up, down = plain_weight(g, 6, 4, b), plain_weight(g, 6, 4, b), plain_weight(g, 4, 6, b)
    w8 = [api.bsr_quantize_scaled8(p) for p in (gate, up, down, api.bsr_transpose(down))]
    x, dy = (torch.randn((T, 4 * b), generator=g).to(BF16).cuda() for _ in range(2))
    return (*w8, gate, x, dy, b)


@pytest.mark.parametrize("b,T", [(64, 1), (64, 100), (128, 3200), (128, 33)])
def test_captured_chain_equals_the_eager_one(b, T):
    args = chain_inputs(b, T)
    x, dy = args[5], args[6]
    chain(*args)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        chain(*args)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            out = chain(*args)
    for k in range(4):
        x.normal_(generator=torch.Generator("cuda").manual_seed(k))
        dy.normal_(generator=torch.Generator("cuda").manual_seed(k + 50))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, chain(*args)):
            assert torch.equal(got, want)


def test_two_streams_at_once():
    sets = [chain_inputs(64, 700, s) for s in range(2)]
    want = [chain(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for _ in range(3):
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                got.append(chain(*s))
    torch.cuda.synchronize()
    for k, g in enumerate(got):
        for a, w in zip(g, want[k % 2]):
            assert torch.equal(a, w)


@pytest.mark.parametrize("T", [1, 16, 300])
def test_prepared_calls(T):
    b = 64
    gate, up, down, _, _, x, _, _ = chain_inputs(b, T)
    x8 = api.empty_scaled8(T, 4 * b, group=b)
    h = api.empty_scaled8(T, 6 * b, group=b)
    keep = tuple(api.empty_scaled8(T, 6 * b, group=b) for _ in range(2))
    y = x.float()
    calls = [api.prepare_quantize_scaled8(x, x8), api.prepare_bsr_gated_scaled8(gate, up, x8, h, keep=keep),
             api.prepare_bsr_linear_scaled8(down, h, y, residual=y)]
    for c in calls:
        c()
    q = api.quantize_scaled8(x, group=b)
    r = api.bsr_gated_scaled8(gate, up, q, keep=True)
    assert torch.equal(x8.codes, q.codes)
    for got, want in zip((h, *keep), (r.H, r.G, r.U)):
        assert torch.equal(got.codes, want.codes) and torch.equal(got.scales[:, :T], want.scales[:, :T])
    assert torch.equal(y, api.bsr_linear_scaled8(down, r.H, residual=x.float()))


def test_kept_activations_against_64_bits_through_the_block():
    """The gradients of a gated block from what it kept, against the formulas in 64 bits on the values that the codes stand for: H of the
    forward pass, G and U, and the gradients that follow from those, a rounding at a time."""
    b, T = 64, 90
    g = gen(5)
    mg, mu = (Matrix(g, masks(4, 5, s), b, "e4m3") for s in (1, 2))
    q, x = eight(activation(g, T, mg.cols, 0.3), b, "e4m3")
    r = api.bsr_gated_scaled8(mg.w8, mu.w8, q, keep=True)
    gv, uv = (torch.from_numpy(ref.values(t.codes, t.scales, b, "e4m3")) for t in (r.G, r.U))
    dh = (torch.randn((T, mg.rows), generator=g) * 0.1).to(BF16)
    through = api.gated_act_backward_scaled8(r.G, r.U, dh.cuda())
    d = dh.double()
    want = d * uv * ref.slope("silu", gv)
    off = 2.0 ** -8 * want.abs() + 2.0 ** -18 * (d * uv).abs()
    close(through.dG, want, off)
    dw = api.bsr_sddmm_scaled8(mg.packed, through.dG, q)
    cut = lambda f: torch.stack([f[i * b:(i + 1) * b, c * b:(c + 1) * b] for i, c in mg.where])  # noqa: E731
    close(dw, cut(want.t() @ x), cut(off.t() @ x.abs()) + T * 2.0 ** -24 * cut((want.abs() + off).t() @ x.abs()))


def test_nan_codes_reach_the_gradient():
    T, N = 8, 256
    z = api.quantize_scaled8(torch.randn((T, N)).cuda(), group=64)
    z.codes[3, 5] = 0x7F
    dy = torch.ones((T, N), device="cuda")
    got = api.act_backward_scaled8(z, dy, act="silu", bias_grad=True)
    assert torch.isnan(got.dZ[3, 5]) and int(torch.isnan(got.dZ).sum()) == 1
    assert torch.isnan(got.dbias[5]) and int(torch.isnan(got.dbias).sum()) == 1


def test_example_network_in_eight_bits():
    """It runs, and its gradients are those of the 16-bit network but for the roundings: with 2^-4 at most a value in E4M3 and 2^-3 in E5M2,
    root mean squares of 0.026 and 0.052 over a binade, a gradient that six such tensors lead to is off by about 0.1 of its size."""
    nets = [Network(width=256, inter=512, blocks=2, seed=3, eight_bit=e) for e in (False, True)]
    h = torch.randn((200, 256), generator=gen(1)).cuda()
    dx = (torch.randn((200, 256), generator=gen(2)) * 0.05).to(BF16).cuda()
    outs, all_grads = [], []
    for net in nets:
        keep = []
        outs.append(net.forward(h.clone(), keep))
        all_grads.append(net.backward(dx, keep))
        assert torch.equal(net.forward(h.clone()), outs[-1])
        net.step(all_grads[-1][0], all_grads[-1][1], 0.01)
        assert torch.isfinite(net.forward(h.clone()).float()).all()
    rel = lambda a, w: float((a.double() - w.double()).norm() / w.double().norm())  # noqa: E731
    assert rel(outs[1], outs[0]) < 0.2
    (g16, f16, d16), (g8, f8, d8) = all_grads
    assert rel(f8, f16) < 0.2 and rel(d8, d16) < 0.2
    for a, w in zip(g8, g16):
        assert set(a) == set(w)
        for k in w:
            if w[k] is not None:
                assert a[k].shape == w[k].shape and 0 <= rel(a[k], w[k]) < 0.25, (k, rel(a[k], w[k]))
