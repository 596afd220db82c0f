"""Linear attention: refusals of calls whose tensors are each well formed, but not together (no GPU: nothing here may reach a launch)."""
import ctypes

import pytest

import paper_2504_20490_amd as A
from paper_2504_20490_amd import binding as B

P = 1 << 20            # a pointer that is never followed


@pytest.mark.parametrize("rows", [12, 0])
def test_the_states_gradients_are_two_buffers(rows):
    """d_initial is written while other workgroups still read d_final."""
    lib, batch = A.load_library(), B._LinearBatchArgs(P, P, P, 4, rows, 5, 4, 2, 64)
    call = lambda d_final, d_initial: lib.hspmd_linear_attn_bwd(ctypes.byref(batch), P, P, P, P, P, 256, 128, 2, 0.0, None, d_final, P, P, P, 0, P, d_initial, P, 0, None)
    assert call(P, P) == 1 and b"d_initial" in lib.hspmd_last_error()
    assert call(P, 2 * P) == 3 and call(None, P) == 3          # (the workspace is too small: they came as far as that)
