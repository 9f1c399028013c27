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
