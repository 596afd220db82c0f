"""A buffer store of more than 64 bits reads its data after it has been issued.  The compiler leaves room in front of an instruction that overwrites them, but takes a store
whose offset is in a scalar register to need none; on this chip such a store has written what came behind it.  So the kernels have none of that form."""
import re

import pytest

from paper_2504_20490_amd import build as lib_build
from test_kernel_invariants import _device_asm

FILES = [s for s in lib_build.SOURCES if s.endswith(".hip")]


@pytest.fixture(scope="module")
def asm():
    from concurrent.futures import ThreadPoolExecutor
    with ThreadPoolExecutor(max_workers=8) as pool:
        return dict(zip(FILES, pool.map(_device_asm, FILES)))


@pytest.mark.parametrize("source", FILES)
def test_no_wide_store_with_an_offset_in_a_register(asm, source):
    found = [l.strip() for l in asm[source].splitlines() if re.search(r"\bbuffer_store_dwordx[34]\b.*\],\s*(s\d+|m0|ttmp\d+)\b(?!:)", l)]
    assert not found, found[:5]
