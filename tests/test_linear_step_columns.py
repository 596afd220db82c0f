"""What a workgroup of the linear attention's single step takes of a state, from the kernels' own rule on the host: all columns are taken once, pieces of rows are whole
lines of memory wherever rows are, and rows that are not are cut for few states of many columns only."""
import ctypes
import subprocess

import pytest

from paper_2504_20490_amd import build as lib_build

SHIM = """
#include "linear_index.hpp"
extern "C" int columns(int head_dim, long states) { return hspmd::linear_step_columns(head_dim, states); }
"""


@pytest.fixture(scope="module")
def columns(tmp_path_factory):
    d = tmp_path_factory.mktemp("linear_step")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", f"-I{lib_build.CSRC}", "-o", str(d / "shim.so"), str(d / "shim.cpp")], check=True)
    f = ctypes.CDLL(str(d / "shim.so")).columns
    f.argtypes = [ctypes.c_int, ctypes.c_long]
    return f


@pytest.mark.parametrize("d", range(8, 129, 8))
def test_pieces(columns, d):
    for states in (1, 2, 7, 63, 64, 65, 500, 512, 513, 640, 4096, 8000, 1 << 22):
        c = columns(d, states)
        assert 0 < c <= d and c % 8 == 0
        assert states * -(-d // c) * 256 < 1 << 32                   # threads of the launch
        if d <= 64 or d % 32 and d <= 96:
            assert c == d
        elif d % 32 == 0:
            assert c % 32 == 0 and c < d
        else:
            assert c % 32 == 0 if states * d * d <= 1 << 20 else c == d


def test_more_states_never_take_narrower_pieces(columns):
    for d in range(8, 129, 8):
        seen = [columns(d, n) for n in (1, 10, 64, 100, 512, 513, 1000, 10000, 1 << 22)]
        assert seen == sorted(seen)


@pytest.mark.gpu
@pytest.mark.parametrize("n,group", [(3, 5), (30, 1), (600, 2)])
@pytest.mark.parametrize("d", [8, 40, 64, 72, 88, 96, 104, 112, 120, 128])
def test_steps_in_pieces(d, n, group):
    import numpy as np
    import torch
    import paper_2504_20490_amd as A
    from linear_util import Case, check_forward, host
    case = Case([1] * n, 2 * group, 2, d, 80 + d, False, True).to_device()
    o = torch.full((n, 2 * group, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    final = torch.full_like(case.tinitial, float("nan"))
    A.linear_attn_step(A.LinearBatch(), case.tq, case.tk, case.tv, case.tg, o, initial=case.tinitial, final=final)
    check_forward(case, o, final)
    # A product and a sum, the exponential: 2^-22.  The decay's exponent g log2(e) is rounded to half a step, and so is the constant: each 2^-24 of it at most, times
    # ln 2 for the decay: together 2^-23 |g|.  (g reaches -10 here, where that is 2^-20 of what the decay leaves.)
    want, most = case.forward()[1], case.forward(absolute=True)[1]
    room = (2.0 ** -22 + 2.0 ** -23 * np.abs(case.g))[:, :, None, None] * most
    assert (np.abs(host(final) - want) <= room).all()
