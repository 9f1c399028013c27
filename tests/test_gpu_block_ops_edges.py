"""Edges of the operators around the MLP: parameters that come alone, gates laid out by a stride of 0.

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
