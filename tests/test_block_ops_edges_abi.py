"""Host-side edges of the operators around the MLP: sizes of workspaces, calls over no rows.  No call gets as far as the GPU."""
import ctypes as C

import pytest

from paper_2507_03117_amd import api
from tests.test_block_ops_abi import P, backward, view


def norm_workspace(v, T):
    need = C.c_size_t(0)
    assert api.lib().blast_norm_residual_backward_workspace(C.byref(v), T, C.byref(need)) == 0
    return need.value


@pytest.mark.parametrize("width", [64, 4096, 16384, 32768])
def test_norm_backward_workspace_is_what_a_launch_fills(width):
    """A row of sums to a workgroup: a workgroup to a row up to 512 rows, beyond that 256 workgroups at most."""
    for v, sums in ((view(width=width), 1), (view(width=width, post=1), 2), (view(width=width, kind=1, post=1, gate=P), 5)):
        for T in (513, 4096, 1 << 20):
            assert norm_workspace(v, T) == sums * 256 * width * 4
        if sums > 1:  # (a single norm's sums need none up to 512 rows)
            assert norm_workspace(v, 300) == sums * 300 * width * 4 and norm_workspace(v, 512) == sums * 512 * width * 4
        assert norm_workspace(v, 1) == 0


def test_norm_backward_over_no_rows_needs_no_operands():
    """Operands of no rows may be null while outputs are not, the gradient of the branch among them."""
    none = dict(T=0, h=None, y=None, stats=None, dx=None, dh=None)
    for v in (view(), view(kind=1), view(post=1), view(gate=P, ldg=64)):
        assert backward(v, **none) == 0 and backward(v, dy=P, **none) == 0
    assert backward(view(gate=P, ldg=64), dy=P, dg=P, **none) == 0
    assert backward(view(), dg=P, **none) == -1  # no gate
    assert backward(view(), dy=P, **dict(none, T=4)) == -1
