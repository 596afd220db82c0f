"""What the kernels of the paged attention rely on and the compiler does not check (see test_kernel_invariants): they keep nothing in M0 beside
the hand-written copies, and no register is spilled to scratch memory, whose traffic would upset the counts that the copies are waited for
by.  And in the loop over key tiles of few rows nothing but those waits, and the compiler's own for a row's first use, may wait for copies."""
import re

import pytest

from test_kernel_invariants import _device_asm

FILES = ["paged_attn_kernel.hip", "paged_many_kernel.hip", "rope_axes_kernel.hip", "kv_cache_kernel.hip"]


@pytest.fixture(scope="module")
def asm():
    from concurrent.futures import ThreadPoolExecutor
    with ThreadPoolExecutor(max_workers=3) as pool:
        return dict(zip(FILES, pool.map(_device_asm, FILES)))


def kernels(text):
    """(name, assembly) of every kernel."""
    names = re.findall(r"^\s*\.amdhsa_kernel\s+(\S+)", text, flags=re.M)
    return [(n, text[text.index(f"\n{n}:"):text.index(f".amdhsa_kernel {n}")]) for n in names]


@pytest.mark.parametrize("source", FILES)
def test_no_register_spills(asm, source):
    text = asm[source]
    assert kernels(text)
    assert not re.findall(r"^\s*scratch_(?:load|store)", text, flags=re.M)
    for name, count in re.findall(r"^\s*\.amdhsa_kernel\s+(\S+).*?\.amdhsa_private_segment_fixed_size\s+(\d+)", text, flags=re.M | re.S):
        assert int(count) == 0, name


@pytest.mark.parametrize("source", FILES[:2])
def test_compiler_keeps_nothing_in_m0(asm, source):
    inside, uses, ours = False, [], 0
    for line in asm[source].splitlines():
        if "#ASMSTART" in line:
            inside = True
        elif "#ASMEND" in line:
            inside = False
        elif re.search(r"\bm0\b", line.split(";")[0]):
            if inside:
                ours += 1
            else:
                uses.append(line.strip())
    assert ours > 0 and not uses, uses[:5]


def test_waits_in_the_tile_loop_of_few_rows(asm):
    """Between the first and the last product of a tile the wave waits for its copies with the counts written in the source only."""
    found = 0
    for name, text in kernels(asm["paged_attn_kernel.hip"]):
        if "paged_few" not in name:
            continue
        lines = text.splitlines()
        products = [i for i, l in enumerate(lines) if "v_mfma" in l]
        waits = [int(m.group(1)) for l in lines[products[0]:products[-1]] for m in [re.search(r"vmcnt\((\d+)\)", l)] if m]
        d, e4m3 = int(re.search(r"ILi(\d+)E", name).group(1)), "Lb1E" in name
        copies = 32 * d * (1 if e4m3 else 2) // 1024
        k, v = copies + (1 if e4m3 else 0), copies
        # the tile's K, its V with and without a further K under way; 0: the last tiles, once
        assert {k + v + k, k + v} <= set(waits) <= {k + v + v, k + v + k, k + v, 0} and waits.count(0) <= 1, (name, waits)
        found += 1
    assert found == 4
