"""Shares of the attention over the paged cache, from the kernels' own index arithmetic on the host: every (row tile, KV head, chunk) of a
batch has one workgroup of the grid, partial results lie apart and inside the workspace, no page or row is out of range, whatever the
device arrays hold."""
import ctypes
import random
import subprocess

import pytest

from paper_2504_20490_amd import build as lib_build

SHIM = """
#include "paged_index.hpp"
#include <vector>
using namespace hspmd;
// checks a batch; 0 or the number of the line that found a mistake.  stats: slots, grid, tiles of partial results used, room for them
extern "C" int check(const int* cu, const int* len, int num_seqs, int total_rows, int width, int shift, int group, int kv_heads, int max_rows, long* stats) {
    const long most = (long)(max_rows > 0 && max_rows < total_rows ? max_rows : total_rows) * group;
    const bool few = most <= kFewRows || num_seqs > 1, many = most > kFewRows;
    const int limit = !many ? 0x7fffffff : few ? kFewRows : 0;
    std::vector<int> taken((long)total_rows * group * kv_heads, 0);
    for (int kind = 0; kind < 2; ++kind) {
        if (!(kind ? many : few)) continue;
        const int R = kind ? kManyRows : kFewRows;
        std::vector<SeqRows> s(num_seqs);
        std::vector<SeqTiles> t(num_seqs);
        long units = 0, slots = 0, parts = 0;
        for (int i = 0; i < num_seqs; ++i) {
            s[i] = seq_rows(cu[i], cu[i + 1], len[i], total_rows, width, shift);
            if (s[i].start < 0 || s[i].n < 0 || s[i].start + s[i].n > total_rows || s[i].kv < 0 || s[i].kv > ((long)width << shift)) return __LINE__;
            t[i] = seq_tiles(s[i], group, R, kind, limit);
            units += (long)t[i].tiles * t[i].units * kv_heads;
        }
        int per = units_per_chunk(units, kind);
        for (int raise = 0, first = per; raise < kRaises; ++raise) {
            long n = 0;
            for (int i = 0; i < num_seqs; ++i) n += (long)t[i].tiles * kv_heads * shares_of(t[i].units, per).chunks;
            const int next = raised(per, first, n, kind);
            if (next == per) break;
            per = next;
        }
        std::vector<long> first(num_seqs), first_part(num_seqs);
        for (int i = 0; i < num_seqs; ++i) {
            const Shares sh = shares_of(t[i].units, per);
            if ((long)sh.chunks * sh.units < t[i].units) return __LINE__;
            const long n = (long)t[i].tiles * kv_heads * sh.chunks;
            first[i] = slots, first_part[i] = parts;
            slots += n;
            parts += sh.chunks > 1 ? n : 0;
        }
        const GridBounds b = grid_bounds(total_rows, num_seqs, width, shift, group, kv_heads, kind, limit);
        const long room = kind ? grid_bounds(total_rows, num_seqs, width, shift, group, kv_heads, true, 0).part_tiles
                               : grid_bounds(total_rows, num_seqs, width, shift, group, kv_heads, false, 0x7fffffff).part_tiles;
        stats[4 * kind] = slots, stats[4 * kind + 1] = b.grid, stats[4 * kind + 2] = parts, stats[4 * kind + 3] = room;
        bool sane = true;                        // rows do not overlap: the bounds hold
        long sum = 0;
        for (int i = 0; i < num_seqs; ++i) sum += s[i].n;
        sane = sum <= total_rows;
        if (sane && (slots > b.grid || parts > room)) return __LINE__;
        std::vector<char> met(slots, 0), used(parts, 0);
        for (long block = 0; block < b.grid; ++block) {
            const long slot = block;
            if (slot >= slots) break;
            met[slot] = 1;
            int i = 0;
            while (i < num_seqs && !(slot >= first[i] && slot < first[i] + (i + 1 < num_seqs ? first[i + 1] : slots) - first[i])) ++i;
            if (i == num_seqs) return __LINE__;
            const Shares sh = shares_of(t[i].units, per);
            const SlotPlace at = place_of_slot(slot - first[i], t[i].tiles, sh.chunks, kv_heads);
            if (at.head < 0 || at.head >= kv_heads || at.chunk < 0 || at.chunk >= sh.chunks || at.tile < 0 || at.tile >= t[i].tiles) return __LINE__;
            if (sh.chunks > 1) {
                const long part = first_part[i] + part_of(at, t[i].tiles, sh.chunks) + at.chunk;
                if (part < 0 || part >= parts || used[part]++) return __LINE__;
            }
            if (at.chunk == 0 && sane)
                for (long rho = (long)at.tile * R; rho < (long)(at.tile + 1) * R && rho < (long)s[i].n * group; ++rho)
                    ++taken[((long)s[i].start * group + rho) * kv_heads + at.head];
        }
        if (sane)
            for (long x = 0; x < slots; ++x) if (!met[x]) return __LINE__;
    }
    bool rising = true;
    for (int i = 0; i < num_seqs; ++i) rising = rising && cu[i] <= cu[i + 1];
    if (rising)
        for (int i = 0; i < num_seqs; ++i) {
            const SeqRows s = seq_rows(cu[i], cu[i + 1], len[i], total_rows, width, shift);
            for (long x = (long)s.start * group * kv_heads; x < (long)(s.start + s.n) * group * kv_heads; ++x)
                if (taken[x] != 1) return __LINE__;
        }
    return 0;
}
"""


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("paged_index")
    src, so = tmp / "shim.cpp", tmp / "shim.so"
    src.write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", lib_build.CSRC, "-o", str(so), str(src)], check=True)
    lib = ctypes.CDLL(str(so))

    def call(cu, lens, total_rows, width, shift, group, kv_heads, max_rows):
        stats = (ctypes.c_long * 8)()
        ints = lambda x: (ctypes.c_int * max(len(x), 1))(*x)
        rc = lib.check(ints(cu), ints(lens), len(lens), total_rows, width, shift, group, kv_heads, max_rows, stats)
        assert rc == 0, (rc, cu, lens, total_rows, width, shift, group, kv_heads, max_rows)
        return list(stats)
    return call


def _cu(rows):
    out = [0]
    for n in rows:
        out.append(out[-1] + n)
    return out


def test_shares_of_random_batches(check):
    rng = random.Random(1)
    for _ in range(400):
        seqs, shift = rng.choice([1, 2, 5, 40, 300]), rng.randint(4, 10)
        group, heads = rng.choice([1, 1, 2, 4, 5, 12, 16, 24]), rng.choice([1, 2, 8])
        most = rng.choice([1, 1, 3, 20, 400 if seqs < 50 else 20])
        rows = [rng.randint(0, most) for _ in range(seqs)]
        lens = [rng.choice([rng.randint(0, 300), rng.randint(0, 20000), n]) for n in rows]
        width = max(1, -(-max(lens) >> shift)) + rng.randint(0, 3)
        T = sum(rows) + rng.randint(0, 3)
        if T * group * heads < 200000:
            check(_cu(rows), lens, T, width, shift, group, heads, rng.choice([0, 1, max(rows), 10000]))


def test_shares_of_batches_at_the_edges(check):
    for rows, lens, group, heads in (([1], [131001], 4, 8), ([1], [1], 1, 1), ([2048], [29082], 4, 8), ([1] * 64, [4000] * 64, 4, 8),
                                     ([16], [70000], 1, 1), ([17], [70000], 1, 1), ([4, 5], [9000, 9000], 4, 2), ([128] * 3, [128] * 3, 1, 5),
                                     ([0, 0], [5, 5], 4, 2), ([1000, 1], [1 << 20, 1 << 20], 1, 2)):
        for max_rows in (0, 1, max(rows)):
            check(_cu(rows), lens, sum(rows), -(-max(lens) // 16), 4, group, heads, max_rows)


def test_arrays_that_make_no_sense(check):
    big = (1 << 31) - 1
    rng = random.Random(2)
    for _ in range(300):
        seqs = rng.choice([1, 2, 7])
        wild = lambda: rng.choice([0, 1, 5, -1, -big - 1, big, rng.randint(-100, 100)])
        T = rng.randint(1, 60)
        check([wild() for _ in range(seqs + 1)], [wild() for _ in range(seqs)], T, rng.choice([0, 1, 3, 1000]), rng.randint(4, 10),
              rng.choice([1, 4, 5]), rng.choice([1, 3]), rng.choice([0, 1, T]))


def test_one_long_sequence_is_shared_out_and_equal_ones_are_not(check):
    slots, grid, parts, room = check(_cu([1]), [131001], 1, 8188, 4, 4, 8, 1)[:4]
    assert slots == parts and 800 <= slots <= grid
    slots, grid, parts, room = check(_cu([64] * 64), [4096 + 3 * i for i in range(64)], 64 * 64, 300, 4, 2, 8, 64)[4:]
    assert slots == 512 and parts == 0
