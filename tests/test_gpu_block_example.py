"""The operators around the MLP as they are used together: the network of examples/train_block.py against the same network in
64 bits, its training, its calls for single tokens, and the calls on other streams and in recorded graphs."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2507_03117_amd import api

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EPS = 1e-5


def example():
    spec = importlib.util.spec_from_file_location("train_block", os.path.join(ROOT, "examples", "train_block.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def dense(weight):
    return api.bsr_unpack(weight.packed).double().cpu()


def norm64(v, kind, w, b=None):
    v = v - v.mean(1, keepdim=True) if kind == "layer" else v
    n = v / torch.sqrt(v.square().mean(1, keepdim=True) + EPS)
    return n * w if b is None else n * w + b


def forward64(net, p, h):
    x = norm64(h, "rms", p["first"])
    for k, blk in enumerate(net.blocks):
        q = {n: p[f"{k}.{n}"] for n in blk if f"{k}.{n}" in p}
        if blk["kind"] == "two":
            z = x @ q["w1"].t() + q["b1"]
            h = h + (z * 0.5 * torch.erfc(-z / math.sqrt(2.0))) @ q["w2"].t() + q["b2"]
            x = norm64(h, "layer", q["weight"], q["bias"])
        else:
            g, u = x @ q["gate"].t(), x @ q["up"].t()
            y = (g * torch.sigmoid(g) * u) @ q["down"].t()
            h = h + 0.7 * q["scale_gate"] * norm64(y, "rms", q["post_weight"])
            x = norm64(h, "rms", q["weight"])
    return x


@pytest.mark.parametrize("b,sparsity", [(64, 0.8), (128, 0.5), (32, 0.7)])
def test_network_against_64_bits(b, sparsity):
    """Output and every gradient.  The activations between the operators are bf16: a rounding (2^-8 of a value at most, 2^-8 /
    sqrt(3) of it on average) at each of about ten points on the way through four blocks and ten on the way back, which add up
    like independent errors: 20 of them, sqrt(20) 2^-8 / sqrt(3) = 0.010 of the length of a result; four times that is allowed."""
    mod = example()
    net = mod.Network(width=256, inter=768, blocks=4, b=b, sparsity=sparsity, seed=3)
    gen = torch.Generator().manual_seed(4)
    for blk in net.blocks:  # parameters off their starting values
        for k, v in blk.items():
            if isinstance(v, torch.Tensor):
                v += 0.2 * torch.randn(v.shape, generator=gen).cuda()
    tokens = 70
    h, c = torch.randn((tokens, 256), generator=gen), torch.randn((tokens, 256), generator=gen).to(torch.bfloat16)
    p = {"first": net.first.double().cpu()}
    for k, blk in enumerate(net.blocks):
        for n, v in blk.items():
            if isinstance(v, mod.Weight):
                p[f"{k}.{n}"] = dense(v)
            elif isinstance(v, torch.Tensor):
                p[f"{k}.{n}"] = v.double().cpu()
    for v in p.values():
        v.requires_grad_()
    h64 = h.double().requires_grad_()
    out64 = forward64(net, p, h64)
    out64.backward(c.double())
    keep = []
    out = net.forward(h.cuda(), keep)
    grads, first, dh = net.backward(c.cuda(), keep)
    off = lambda a, w: float((a.double().cpu() - w).norm() / w.norm())  # noqa: E731
    bound = 4 * math.sqrt(20) * 2.0 ** -8 / math.sqrt(3)
    assert off(out, out64.detach()) <= bound
    assert off(dh, h64.grad) <= bound and off(first, p["first"].grad) <= bound
    for k, (blk, grad) in enumerate(zip(net.blocks, grads)):
        for n, v in grad.items():
            if v is None:
                continue
            want = p[f"{k}.{n}"].grad
            if isinstance(blk[n], mod.Weight):
                m = blk[n].packed
                rows = torch.repeat_interleave(torch.arange(m.rows // b), m.row_ptr.cpu().diff())
                cols = m.col_idx[:m.nnz].cpu().long()
                want = want.view(m.rows // b, b, m.cols // b, b).permute(0, 2, 1, 3)[rows, cols]
            assert off(v, want) <= bound, (k, n, off(v, want))


def test_training_lowers_the_loss_and_tokens_match():
    mod = example()
    net = mod.Network(width=256, inter=512, blocks=2, seed=5)
    losses = mod.train(net, steps=25, tokens=128)
    assert losses[-1] < 0.7 * losses[0] and all(math.isfinite(v) for v in losses)
    for t in (1, 3):
        h = torch.randn((t, 256), device="cuda")
        want = net.forward(h.clone()).float()
        out = torch.empty((t, 256), dtype=torch.bfloat16, device="cuda")
        for call in net.token_calls(h, out):
            call()
        # the same kernels on the same values, but for the products of single tokens: a few roundings of bf16
        assert float((out.float() - want).abs().max()) <= 4 * 2.0 ** -8 * float(want.abs().max())


def pieces(seed, T=300, E=320):
    """One call of each operator: (function, outputs as a flat list)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, dt=torch.bfloat16: torch.randn(s, generator=g, device="cuda").to(dt)  # noqa: E731
    W = api.bsr_pack(r(512, E), 64, sparsity=0.5)
    s = {"x": r(T, E), "res": r(T, 512, dt=torch.float32), "z": r(T, 512), "dy": r(T, 512), "h": r(T, E, dt=torch.float32), "y": r(T, E),
         "dx": r(T, E), "w": r(E, dt=torch.float32), "gate": r(E, dt=torch.float32)}
    args = {"weight": s["w"], "post": True, "post_weight": s["w"], "gate": s["gate"]}

    def call():
        z = torch.empty((T, 512), dtype=torch.bfloat16, device="cuda")
        y = api.bsr_linear(W, s["x"], act="silu", residual=s["res"], pre=z)
        a = api.act_backward(s["z"], s["dy"], act="gelu", bias_grad=True)
        h, x, stats = api.norm_residual(s["h"], s["y"], with_stats=True, **args)
        n = api.norm_residual_backward(h, s["y"], stats, s["dx"], s["h"], **args)
        return [y, z, a.dZ, a.dbias, h, x, stats, n.dh, n.dy, n.dgate, n.dweight, n.dpost_weight]

    return s, call


def test_operators_on_a_stream_of_their_own():
    """Enqueued on the current stream and nowhere else: inputs written on that stream just before, results read on it."""
    s, call = pieces(1)
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    kept = {k: v.clone() for k, v in s.items()}
    with torch.cuda.stream(side):
        for v in s.values():
            v.zero_()
        torch.cuda._sleep(20_000_000)  # (the inputs come back only after a while)
        for k, v in s.items():
            v.copy_(kept[k])
        got = [t.clone() for t in call()]
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_operators_in_a_recorded_graph():
    """Recorded once and replayed on changing inputs, with eager work and synchronisations between: every replay has the bits of
    the eager calls."""
    s, call = pieces(2)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for k in range(4):
        g = torch.Generator(device="cuda").manual_seed(100 + k)
        for v in s.values():
            v.copy_(torch.randn(v.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, call()):
            assert torch.equal(a, b), k
