"""The example network in eight bits, run token by token."""
import pytest
import torch

from examples.train_block import Network
from tests.test_gpu_scaled8 import BF16, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("T", [1, 3, 40])
def test_tokens_in_eight_bits_are_the_forward_pass(b, T):
    """The same calls on the same values: the output and the residual stream have the forward pass's bits."""
    net = Network(width=256, inter=512, blocks=4, b=b, seed=7, eight_bit=True)
    h = torch.randn((T, 256), generator=gen(T)).cuda()
    keep = []
    want = net.forward(h.clone(), keep)
    out = torch.empty((T, 256), dtype=BF16, device="cuda")
    stream = h.clone()
    calls = net.token_calls(stream, out)
    for _ in range(2):  # the calls are repeated on new tokens
        stream.copy_(h)
        out.fill_(7)
        for call in calls:
            call()
        assert torch.equal(out, want) and torch.equal(stream, keep[-1][3])
