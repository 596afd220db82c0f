"""Anchors of the linear attention's decay gradients, from the kernels' own index arithmetic on the host: every anchor of every segment has an entry of its own, they
are as far apart as the routine that goes by them takes, and none is outside the workspace, whatever cu_rows holds."""
import ctypes
import random
import subprocess

import pytest

from paper_2504_20490_amd import build as lib_build

SHIM = """
#include "linear_index.hpp"
#include <vector>
using namespace hspmd;
// checks a batch (seg 0: sequences are not cut); 0 or the number of the line that found a mistake
extern "C" int check(const int* cu, int num_seqs, int total_rows, int seg, int sane) {
    const long entries = linear_anchors(total_rows);
    std::vector<char> met(entries, 0);
    for (int s = 0; s < num_seqs; ++s) {
        const LinearRows r = linear_rows(cu[s], cu[s + 1], total_rows);
        const int count = seg ? linear_segments(r.n, seg) : 1, each = seg ? linear_segment_rows(r.n, count) : 0;
        for (int b = 0; b < count; ++b) {
            const int start = r.start + b * each, rows = seg && r.n - b * each > each ? each : r.n - b * each;
            const int chunks = (rows + kLinearChunk - 1) / kLinearChunk;
            int since = 0;
            for (int c = chunks - 1; c >= 0; --c) {
                if (!linear_is_anchor(c, chunks)) {
                    if (++since >= kLinearAnchor && c > 0) return __LINE__;
                    continue;
                }
                if (c == 0 || since != kLinearAnchor - 1) return __LINE__;
                since = 0;
                const int at = linear_anchor(start, c, chunks);
                if (at < 0 || at >= entries) return __LINE__;
                if (sane && met[at]++) return __LINE__;
            }
        }
    }
    return 0;
}
extern "C" int elements(int head_dim) { return linear_anchor_elements(head_dim); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("linear_anchors")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", f"-I{lib_build.CSRC}", "-o", str(d / "shim.so"), str(d / "shim.cpp")], check=True)
    return ctypes.CDLL(str(d / "shim.so"))


def check(lib, cu, total, seg, sane=True):
    return lib.check((ctypes.c_int * len(cu))(*cu), len(cu) - 1, total, seg, int(sane))


def test_every_anchor_has_an_entry_of_its_own(lib):
    rng = random.Random(1)
    for _ in range(3000):
        seg = rng.choice([0, 64 * rng.randint(4, 20)])
        edge = seg or 64 * rng.randint(1, 20)
        lengths = [rng.choice([0, 1, 64, 65, 255, 256, 257, 512, 513, edge - 1, edge, edge + 1, 2 * edge + 1, rng.randint(0, 5 * edge)]) for _ in range(rng.randint(1, 12))]
        cu = [rng.choice([0, 0, 100])]
        for n in lengths:
            cu.append(cu[-1] + n)
        assert check(lib, cu, cu[-1] + rng.choice([0, 0, 1, 500]), seg) == 0, (lengths, seg)


def test_nothing_in_cu_rows_leads_out(lib):
    rng = random.Random(2)
    for _ in range(3000):
        seg, total = rng.choice([0, 64 * rng.randint(4, 20)]), rng.randint(0, 20000)
        cu = [rng.choice([0, total, rng.randint(-5, total + 5), -2 ** 31, 2 ** 31 - 1, rng.randint(-2 ** 31, 2 ** 31 - 1)]) for _ in range(rng.randint(2, 12))]
        assert check(lib, cu, total, seg, False) == 0, (cu, total, seg)


def test_the_largest_counts_fit(lib):
    top = 1 << 25
    for seg in (0, 256, 16384):
        assert check(lib, [0, top], top, seg) == 0
        assert check(lib, [0, 5, top - 7, top], top, seg) == 0


def test_what_an_anchor_keeps(lib):
    """The waves' part of a state: head_dim's columns in groups of 32, a wave each, its rows in groups of 16."""
    for d in range(8, 129, 8):
        assert lib.elements(d) == -(-d // 16) * 16 * -(-d // 32) * 32
