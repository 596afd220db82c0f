"""Segments of the linear attention, from the kernels' own index arithmetic on the host: every segment has one slot of the launch, every state of
a long sequence an entry of its own, every long sequence one window; nothing leaves the grid or the workspace, whatever cu_rows holds."""
import ctypes
import random
import subprocess

import pytest

from paper_2504_20490_amd import build as lib_build

SHIM = """
#include "linear_index.hpp"
#include <vector>
using namespace hspmd;
// checks a batch; 0 or the number of the line that found a mistake
extern "C" int check(const int* cu, int num_seqs, int total_rows, int seg, int sane) {
    const long slots = linear_slots(total_rows, num_seqs, seg), entries = linear_entries(total_rows, seg), windows = linear_windows(total_rows, seg);
    std::vector<int> slot_of(slots, -1), entry_of(entries, -1), window_of(windows, -1);
    for (int s = 0; s < num_seqs; ++s) {
        const LinearRows r = linear_rows(cu[s], cu[s + 1], total_rows);
        if (r.start < 0 || r.n < 0 || r.start + r.n > total_rows) return __LINE__;
        const int count = linear_segments(r.n, seg), first = linear_first_slot(r.start, s, seg), entry = linear_first_entry(r.start, seg);
        if (count < 1 || (long)count * seg < r.n || (count > 1 && (long)(count - 1) * seg >= r.n)) return __LINE__;
        if (entry < 0 || (count > 1 && entry + count > entries)) return __LINE__;
        const int rows = linear_segment_rows(r.n, count);
        if (rows > seg || (r.n > 0 && ((long)(count - 1) * rows >= r.n || (long)count * rows < r.n || rows % kLinearChunk))) return __LINE__;
        if (!sane) continue;
        for (int b = 0; b < count; ++b) {
            if (first + b >= slots || slot_of[first + b] >= 0) return __LINE__;
            slot_of[first + b] = s;
            if (count == 1) continue;
            if (entry_of[entry + b] >= 0) return __LINE__;
            entry_of[entry + b] = s;
        }
        if (count > 1) window_of[r.start / seg] = s;
    }
    if (!sane) return 0;
    for (int s = 0; s + 1 < num_seqs; ++s)
        if (linear_first_slot(linear_rows(cu[s], 0, total_rows).start, s, seg) >= linear_first_slot(linear_rows(cu[s + 1], 0, total_rows).start, s + 1, seg)) return __LINE__;
    for (int s = 0; s < num_seqs; ++s) {
        const LinearRows r = linear_rows(cu[s], cu[s + 1], total_rows);
        if (linear_segments(r.n, seg) == 1) continue;
        int last = 0;                            // the launch's search: the last sequence that starts before the window's end
        for (int i = 0; i < num_seqs; ++i)
            if (linear_rows(cu[i], 0, total_rows).start < (long)(r.start / seg + 1) * seg) last = i;
        if (last != s) return __LINE__;
    }
    return 0;
}
extern "C" int check_items(long items, int granule) {
    std::vector<char> met(items, 0);
    long n = 0;
    for (long b = 0; b < linear_grid(items, granule); ++b) {
        const long i = linear_item(b, granule);
        if (i < 0) return __LINE__;
        if (i >= items) continue;
        if (met[i]++) return __LINE__;
        ++n;
    }
    return n == items ? 0 : __LINE__;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("linear_index")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", f"-I{lib_build.CSRC}", "-o", str(d / "shim.so"), str(d / "shim.cpp")], check=True)
    so = ctypes.CDLL(str(d / "shim.so"))
    so.check_items.argtypes = [ctypes.c_long, ctypes.c_int]
    return so


def check(lib, cu, total, seg, sane=True):
    return lib.check((ctypes.c_int * len(cu))(*cu), len(cu) - 1, total, seg, int(sane))


def test_every_segment_has_a_place_of_its_own(lib):
    rng = random.Random(1)
    for _ in range(3000):
        seg = 64 * rng.randint(4, 20)
        lengths = [rng.choice([0, 1, seg - 1, seg, seg + 1, 2 * seg, 2 * seg + 1, rng.randint(0, 5 * seg)]) for _ in range(rng.randint(1, 12))]
        cu = [0]
        for n in lengths:
            cu.append(cu[-1] + n)
        assert check(lib, cu, cu[-1] + rng.choice([0, 0, 1, 500]), seg) == 0, (lengths, seg)


def test_nothing_in_cu_rows_leads_out(lib):
    rng = random.Random(2)
    for _ in range(3000):
        seg, total = 64 * rng.randint(4, 20), rng.randint(0, 20000)
        cu = [rng.choice([0, total, rng.randint(-5, total + 5), -2 ** 31, 2 ** 31 - 1, rng.randint(-2 ** 31, 2 ** 31 - 1)]) for _ in range(rng.randint(2, 12))]
        assert check(lib, cu, total, seg, False) == 0, (cu, total, seg)


def test_the_largest_counts_fit(lib):
    top = 1 << 25
    assert check(lib, [0, top], top, 256) == 0
    assert check(lib, [0, 5, top - 7, top], top, 256) == 0


@pytest.mark.parametrize("items", [0, 1, 7, 8, 9, 100, 1001, 65536])
def test_items_are_dealt_out_once(lib, items):
    for granule in (4, 8, 12):
        assert lib.check_items(items, granule) == 0
