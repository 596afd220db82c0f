"""What the kernels of the linear attention rely on and the compiler does not check: registers (a wave holds its part of a state in them for a whole segment; a
few spilled scalars' lanes and bases are all that is let through), and the operations written out in `rest_of_rounding`, whose last result must not be read for
three operations."""
import re

import pytest

from test_kernel_invariants import _device_asm

FILES = ["linear_fwd_kernel.hip", "linear_bwd_kernel.hip", "linear_state_kernel.hip", "linear_step_kernel.hip"]
MOST_SPILLED = 32        # bytes of scratch memory per lane


@pytest.fixture(scope="module")
def asm():
    from concurrent.futures import ThreadPoolExecutor
    with ThreadPoolExecutor(max_workers=4) as pool:
        return dict(zip(FILES, pool.map(_device_asm, FILES)))


@pytest.mark.parametrize("source", FILES)
def test_registers(asm, source):
    found = re.findall(r"^\s*\.amdhsa_kernel\s+(\S+).*?\.amdhsa_private_segment_fixed_size\s+(\d+)", asm[source], flags=re.M | re.S)
    assert found
    for name, count in found:
        assert int(count) <= MOST_SPILLED, name


@pytest.mark.parametrize("source", FILES[:2])
def test_written_out_dot_products_end_in_a_wait(asm, source):
    blocks = re.findall(r"#ASMSTART(.*?)#ASMEND", asm[source], flags=re.S)
    dots = [b for b in blocks if "v_dot2_f32_bf16" in b]
    assert dots
    for b in dots:
        lines = [l.split(";")[0].strip() for l in b.splitlines() if l.split(";")[0].strip()]
        assert len(lines) == 9 and lines[-1] == "s_nop 2"
        written = [re.match(r"v_dot2_f32_bf16 (v\d+),", l).group(1) for l in lines[:8]]
        read = " ".join(l.split(",", 1)[1] for l in lines[:8])
        assert len(set(written)) == 8 and not any(re.search(rf"\b{w}\b", read) for w in written)


def test_no_memory_cleared_by_the_runtime():
    """Calls are captured into graphs: nothing is cleared but by kernels."""
    import os
    from paper_2504_20490_amd import build as lib_build
    for name in FILES + ["linear_walk.hpp", "linear_device.hpp"]:
        with open(os.path.join(lib_build.CSRC, name)) as f:
            assert "hipMemset" not in f.read()
