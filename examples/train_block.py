"""A small residual network of block-sparse MLPs, trained and then run token by token, on the operators around the MLP.

Two kinds of block alternate, as the two MLPs of the paper's models:
  two matrices   y = W2 gelu(W1 x + b1) + b2, added to the stream in the second product's epilogue, then a layer norm;
  gated          y = Wdown (silu(Wgate x) * Wup x), normalised, gated per feature, scaled and added by norm_residual, which
                 also takes the norm that the next block reads.
The gradient of every weight block is kept for the stored blocks only; G and U of the gated block are made again on the way
back instead of being kept.  Run: python examples/train_block.py
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)
from paper_2507_03117_amd import api  # noqa: E402

BF16 = torch.bfloat16


def _packed(gen, rows, cols, b, sparsity, std):
    w = torch.randn((rows, cols), generator=gen, device="cuda").mul_(std).to(BF16)
    return api.bsr_pack(w, b, sparsity=sparsity)


class Weight:
    """A packed matrix with fp32 masters of its stored blocks."""

    def __init__(self, gen, rows, cols, b, sparsity):
        self.packed = _packed(gen, rows, cols, b, sparsity, (1.0 / (cols * (1 - sparsity))) ** 0.5)
        n = self.packed.nnz * b * b
        self.values = self.packed.vals[:n].view(BF16).view(-1, b, b)
        self.master = self.values.float()

    def __call__(self, x, **kw):
        return api.bsr_linear(self.packed, x, out_dtype=BF16, **kw)

    def backward(self, dy, x, dx_dtype=BF16):
        """(gradient of x, gradient of the stored blocks)."""
        return api.bsr_spmm(api.bsr_transpose(self.packed), dy, out_dtype=dx_dtype), api.bsr_sddmm(self.packed, dy, x)

    def step(self, grad, rate):
        self.master -= rate * grad
        self.values.copy_(self.master)


class Network:
    def __init__(self, width=512, inter=2048, blocks=4, b=64, sparsity=0.8, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.width = width
        ones, zeros = (lambda n: torch.ones(n, device="cuda")), (lambda n: torch.zeros(n, device="cuda"))
        self.blocks = []
        for k in range(blocks):
            up = [Weight(gen, inter, width, b, sparsity)]
            if k % 2 == 0:
                blk = {"kind": "two", "w1": up[0], "w2": Weight(gen, width, inter, b, sparsity), "b1": zeros(inter), "b2": zeros(width)}
            else:
                blk = {"kind": "gated", "gate": up[0], "up": Weight(gen, inter, width, b, sparsity),
                       "down": Weight(gen, width, inter, b, sparsity), "post_weight": ones(width), "scale_gate": ones(width) * 0.5}
            # the norm after the block: what the next one (or the output) reads
            blk.update(weight=ones(width), bias=zeros(width) if blk["kind"] == "two" else None)
            self.blocks.append(blk)
        self.first = ones(width)

    def _norm(self, blk):
        if blk["kind"] == "two":
            return {"kind": "layer", "weight": blk["weight"], "bias": blk["bias"]}
        return {"kind": "rms", "weight": blk["weight"], "post": True, "post_weight": blk["post_weight"],
                "gate": blk["scale_gate"], "scale": 0.7}

    def forward(self, h, keep=None):
        """h: residual stream, fp32 [tokens, width].  Returns the last norm's output; `keep`, a list, receives what backward needs."""
        _, x, stats = api.norm_residual(h, weight=self.first, with_stats=True)
        if keep is not None:
            keep.append((h, stats))
        for blk in self.blocks:
            x_in = x
            if blk["kind"] == "two":
                z = torch.empty((h.shape[0], blk["b1"].numel()), dtype=BF16, device="cuda") if keep is not None else None
                a = blk["w1"](x, bias=blk["b1"], act="gelu", pre=z)
                h = api.bsr_linear(blk["w2"].packed, a, bias=blk["b2"], residual=h)  # fp32, a new stream: the old one is kept
                _, x, stats = api.norm_residual(h, with_stats=True, **self._norm(blk))
                saved = (x_in, z, a, h, None, stats)
            else:
                y = api.sparse_mlp(blk["gate"].packed, blk["up"].packed, blk["down"].packed, x, out_dtype=BF16)
                h, x, stats = api.norm_residual(h, y, with_stats=True, **self._norm(blk))
                saved = (x_in, None, None, h, y, stats)
            if keep is not None:
                keep.append(saved)
        return x

    def backward(self, dx, keep):
        """Gradients of all parameters from the gradient of the output (bf16 or fp32): a dict per block, and the first norm's."""
        dh, grads = None, []
        for blk, (x, z, a, h, y, stats) in zip(reversed(self.blocks), reversed(keep[1:])):
            g = api.norm_residual_backward(h, y, stats, dx, dh, **self._norm(blk))
            dh = g.dh
            if blk["kind"] == "two":
                # the block's output went onto the stream as it was: its gradient is the stream's, in bf16 for the products
                into = api.act_backward(None, dh, bias_grad=True)
                da, dw2 = blk["w2"].backward(into.dZ, a)
                through = api.act_backward(z, da, act="gelu", bias_grad=True)
                dx, dw1 = blk["w1"].backward(through.dZ, x)
                grads.append({"w1": dw1, "w2": dw2, "b1": through.dbias, "b2": into.dbias, "weight": g.dweight, "bias": g.dbias})
            else:
                gate, up = blk["gate"](x), blk["up"](x)
                dy = g.dy
                dact = api.bsr_spmm(api.bsr_transpose(blk["down"].packed), dy, out_dtype=BF16)
                through = api.gated_act_backward(gate, up, dact)
                ddown = api.bsr_sddmm(blk["down"].packed, dy, through.H)
                dx_gate, dgate = blk["gate"].backward(through.dG, x, torch.float32)
                up_t = api.bsr_transpose(blk["up"].packed)
                # both products' gradients of x meet in the second one's epilogue
                dx = api.bsr_linear(up_t, through.dU, residual=dx_gate, out_dtype=BF16)
                dup = api.bsr_sddmm(blk["up"].packed, through.dU, x)
                grads.append({"gate": dgate, "up": dup, "down": ddown, "weight": g.dweight, "post_weight": g.dpost_weight,
                              "scale_gate": g.dgate})
        h, stats = keep[0]
        g = api.norm_residual_backward(h, None, stats, dx, dh, weight=self.first)
        return grads[::-1], g.dweight, g.dh

    def step(self, grads, first, rate):
        for blk, grad in zip(self.blocks, grads):
            for k, v in grad.items():
                if isinstance(blk[k], Weight):
                    blk[k].step(v, rate)
                elif v is not None:
                    blk[k] -= rate * v
        self.first -= rate * first

    def token_calls(self, h, x_out):
        """The calls of one token (or a few) on kept buffers: h (fp32 [tokens, width]) is updated in place, x_out receives the output."""
        t, calls = h.shape[0], []
        x = torch.empty((t, self.width), dtype=BF16, device="cuda")
        calls.append(api.prepare_norm_residual(h, None, h, x, weight=self.first))
        ws = None
        for k, blk in enumerate(self.blocks):
            out = x_out if k + 1 == len(self.blocks) else x
            if blk["kind"] == "two":
                a = torch.empty((t, blk["b1"].numel()), dtype=BF16, device="cuda")
                calls.append(api.prepare_bsr_linear(blk["w1"].packed, x, a, bias=blk["b1"], act="gelu"))
                calls.append(api.prepare_bsr_linear(blk["w2"].packed, a, h, bias=blk["b2"], residual=h))
                calls.append(api.prepare_norm_residual(h, None, h, out, **self._norm(blk)))
            else:
                m = (blk["gate"].packed, blk["up"].packed, blk["down"].packed)
                y = torch.empty((t, self.width), dtype=BF16, device="cuda")
                if ws is None:
                    ws = torch.empty(max(api.mlp_workspace_bytes(*m, t), 256), dtype=torch.uint8, device="cuda")
                calls.append(api.prepare_sparse_mlp(*m, x, y, ws))
                calls.append(api.prepare_norm_residual(h, y, h, out, **self._norm(blk)))
        return calls


def train(net, steps=30, tokens=512, rate=0.02, seed=1):
    """Fits the network to a fixed random target; returns the losses (mean square error of the output)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn((tokens, net.width), generator=gen, device="cuda")
    want = torch.randn((tokens, net.width), generator=gen, device="cuda")
    losses = []
    for _ in range(steps):
        keep = []
        out = net.forward(h, keep).float()
        losses.append(float((out - want).square().mean()))
        dx = ((out - want) * (2.0 / tokens)).to(BF16)
        grads, first, _ = net.backward(dx, keep)
        net.step(grads, first, rate)
    return losses


def main():
    net = Network()
    losses = train(net)
    print("loss %.4f -> %.4f" % (losses[0], losses[-1]))
    h = torch.randn((1, net.width), device="cuda")
    want = net.forward(h.clone())
    out = torch.empty((1, net.width), dtype=BF16, device="cuda")
    for call in net.token_calls(h, out):
        call()
    torch.cuda.synchronize()
    print("one token: off by %.3g of the forward pass" % float((out.float() - want.float()).abs().max()))


if __name__ == "__main__":
    main()
