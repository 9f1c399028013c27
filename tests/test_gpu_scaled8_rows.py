"""Scaled 8-bit operands of more rows or blocks than one launch has lanes for (2^32)."""
import pytest
import torch

from paper_2507_03117_amd import api

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_quantisers_of_many_tokens():
    """2^28 and some tokens of one feature, sixteen to a workgroup of 256 lanes."""
    T = (1 << 28) + 37
    x = torch.empty((T, 1), dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    q = api.quantize_scaled8(x, group=64)
    y = api.dequantize_scaled8(q)
    # a token's only value has its own scale, and three bits behind its first: off by 2^-4 of itself at most
    for t in range(0, T, 1 << 26):
        v, w = x[t:t + (1 << 26)].float(), y[t:t + (1 << 26)].float()
        assert bool(((v - w).abs() <= 2.0 ** -4 * v.abs()).all()), t
    for t in (0, (1 << 27) - 8, (1 << 28) - 16, T - 16):
        part = api.quantize_scaled8(x[t:t + 16], group=64)
        assert torch.equal(q.codes[t:t + 16], part.codes) and torch.equal(q.scales[:, t:t + 16].contiguous(), part.scales)
        assert torch.equal(y[t:t + 16], api.dequantize_scaled8(part))
