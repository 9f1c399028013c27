"""Host-side limits of the operators on scaled 8-bit tensors: refused before the GPU is touched."""
import ctypes as C

from paper_2507_03117_amd import api
from tests.test_scaled8_abi import P, eight, matrix


def test_gradient_of_more_blocks_than_a_launch_has_waves_for():
    """2^25 parts of 64 x 64 values are 512 GiB of gradients; one more is refused, whatever the width of a block."""
    L = api.lib()
    for b, nnz, group in ((64, (1 << 25) + 1, 64), (128, (1 << 23) + 1, 128)):
        v, x = matrix(128, 128, b, nnz), eight(group=group)
        assert L.blast_bsr_sddmm_scaled8(C.byref(v), P, 128, C.byref(x), 4, P, None, 0, None) == -1
