"""Scaled 8-bit operands of more rows or blocks than one launch has lanes for (2^32)."""
import ctypes as C

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


@pytest.mark.parametrize("out", ["bf16", "e4m3"])
def test_products_of_many_block_rows(out):
    """2^23 and some block rows for two tokens, a workgroup of 512 lanes to each where blocks are shared: four of them have a block.
    Integers: sums are exact in whatever order."""
    b, nbr, T = 64, (1 << 23) + 3, 2
    where = [0, 5, 1 << 22, nbr - 1]
    counts = torch.zeros(nbr + 1, dtype=torch.int32, device="cuda")
    counts[[r + 1 for r in where]] = 1
    row_ptr = counts.cumsum(0).to(torch.int32)
    col_idx = torch.tensor([0, 1, 1, 0], dtype=torch.int32, device="cuda")
    g = torch.Generator("cuda").manual_seed(2)
    vals = torch.randint(-3, 4, (4, b, b), generator=g, device="cuda").to(BF16)
    x8 = api.quantize_scaled8(torch.randint(-4, 5, (T, 2 * b), generator=g, device="cuda").float(), group=b)
    order = torch.arange(nbr, dtype=torch.int32, device="cuda")
    W = api.PackedBsr(nbr * b, 2 * b, b, 4, row_ptr, col_idx, vals.view(torch.int16), order, None, 0)
    w8 = api.bsr_quantize_scaled8(W)
    small = api.PackedBsr(4 * b, 2 * b, b, 4, torch.arange(5, dtype=torch.int32, device="cuda"), col_idx, W.vals, order[:4], None, 0)
    s8 = api.Weight8(small, w8.codes, w8.scales)
    if out == "bf16":
        y = torch.full((T, nbr * b), 7.0, dtype=BF16, device="cuda")
        h = torch.full((T, nbr * b), 7.0, dtype=BF16, device="cuda")
        api.bsr_linear_scaled8(w8, x8, out=y)
        api.bsr_gated_scaled8(w8, w8, x8, act=None, out=h)
        few = (api.bsr_linear_scaled8(s8, x8, out_dtype=BF16), api.bsr_gated_scaled8(s8, s8, x8, act=None, out_fmt=None).H)
        for got, want in zip((y, h), few):
            got = got.view(T, nbr, b)
            for k, r in enumerate(where):
                assert torch.equal(got[:, r], want[:, k * b:(k + 1) * b]), r
                got[:, r] = 0
            assert not got.any()
        return
    q, few = api.bsr_linear_scaled8(w8, x8, out_fmt="e4m3"), api.bsr_linear_scaled8(s8, x8, out_fmt="e4m3")
    codes = q.codes.view(T, nbr, b)
    for k, r in enumerate(where):
        assert torch.equal(codes[:, r], few.codes[:, k * b:(k + 1) * b]) and torch.equal(q.scales[r, :T], few.scales[k, :T]), r
        codes[:, r] = 0
        q.scales[r, :T] = 27
    assert not codes.any() and bool((q.scales[:, :T] == 27).all())


def test_gradient_of_many_blocks_over_no_tokens():
    """2^22 blocks of 64 x 64 and one: 64 GiB of zeros, four values to a lane."""
    b, nnz = 64, (1 << 22) + 1
    row_ptr = torch.tensor([0, nnz], dtype=torch.int32, device="cuda")
    col_idx = torch.arange(nnz, dtype=torch.int32, device="cuda")
    out = torch.ones((nnz, b * b), device="cuda")
    v = api.BsrView(b, nnz * b, b, 0, nnz, row_ptr.data_ptr(), col_idx.data_ptr(), None, None, None)
    x = api.Scaled8View(None, nnz * b, None, 16, 0, 64)
    rc = api.lib().blast_bsr_sddmm_scaled8(C.byref(v), None, b, C.byref(x), 0, out.data_ptr(), None, 0,
                                           torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    for q in range(0, nnz, 1 << 19):
        assert not out[q:q + (1 << 19)].any(), q
