"""Linear attention: d_initial is written while other workgroups of the launch still read d_final and the initial states.  Memory that they share is refused, and only
that (no GPU: nothing here may reach a launch)."""
import ctypes

import pytest

import paper_2504_20490_amd as A
from paper_2504_20490_amd import binding as B

P = 1 << 20            # a pointer that is never followed
STATE = 2 * 64 * 64    # elements of a sequence's states
N = 4                  # sequences


def call(d_final=None, d_initial=None, pool=None, stride=STATE, slots=9, named=True, rows=12, n=N):
    """1: refused; 3: as far as the workspace, which is too small."""
    batch = B._LinearBatchArgs(P, P if named else None, None, n, rows, 5, 4, 2, 64)
    states = None if pool is None else ctypes.byref(B._LinearStatesArgs(pool, stride, slots))
    return A.load_library().hspmd_linear_attn_bwd(ctypes.byref(batch), P, P, P, P, P, 256, 128, 2, 0.0, states, d_final, P, P, P, 0, P, d_initial, P, 0, None)


@pytest.mark.parametrize("rows", [12, 0])
def test_d_final(rows):
    size = 4 * N * STATE
    for apart in (16, size // 2, size - 16):
        assert call(P, P + apart, rows=rows) == 1 and b"d_initial" in A.load_library().hspmd_last_error()
        assert call(P + apart, P, rows=rows) == 1
    for apart in (size, size + 16, 3 * size):
        assert call(P, P + apart, rows=rows) == 3 and call(P + apart, P, rows=rows) == 3


@pytest.mark.parametrize("named", [True, False])
@pytest.mark.parametrize("rows", [12, 0])
def test_the_pool_of_initial_states(rows, named):
    size, pool = 4 * N * STATE, 4 * 9 * STATE
    far = P + (1 << 26)
    for at in (far, far + 16, far + 4 * STATE, far + pool - 16, far - 16, far - size + 16):
        assert call(None, at, far, rows=rows, named=named) == 1 and b"d_initial" in A.load_library().hspmd_last_error(), at - far
    for at in (far - size, far + pool, far + pool + 16):
        assert call(None, at, far, rows=rows, named=named) == 3, at - far


def test_between_the_slots_of_a_pool():
    """Slots of a state and room for another two: one sequence's gradient may lie in that room."""
    far, state = P + (1 << 26), 4 * STATE
    at = lambda places, **c: call(None, far + places, far, stride=3 * STATE, n=1, **c)
    assert at(state) == 3 and at(2 * state) == 3 and at(4 * state) == 3 and at(26 * state) == 3
    assert at(state - 16) == 1 and at(2 * state + 16) == 1 and at(3 * state) == 1 and at(24 * state) == 1 and at(25 * state - 16) == 1
    assert at(25 * state) == 3 and at(state, slots=1) == 3
    assert call(None, far + state, far, stride=3 * STATE, n=2) == 3 and call(None, far + state, far, stride=3 * STATE, n=3) == 1


def test_no_memory_in_common_where_there_is_none():
    assert call(P, None, P) == 3 and call(None, None, P) == 3          # d_final may be read as the initial states are: neither is written
    assert call(None, P) == 3


@pytest.mark.parametrize("stride", [1 << 61, 1 << 62, (1 << 63) - 4])
def test_slots_as_far_apart_as_can_be(stride):
    far = P + (1 << 26)
    assert call(None, far, far, stride=stride) == 1 and call(None, far + 4 * STATE, far, stride=stride) == 3 and call(None, far - 16, far, stride=stride) == 1


def test_no_sequence_has_no_gradient():
    """Nothing is written then, whatever the pointers are."""
    far = P + (1 << 26)
    for d_initial in (far, far + 16, far + 4 * STATE):
        assert call(None, d_initial, far, n=0, rows=0) == 0 and call(far + 32, d_initial, n=0, rows=0) == 0, d_initial - far
