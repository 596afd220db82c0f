// Which rows, keys and pages a workgroup of the attention over the paged cache takes.  Plain index arithmetic, usable on the host as well:
// that every share is taken once and that nothing leads out of the grid or the workspace is tested there.
#pragma once
#include <stdint.h>

namespace hspmd {

#if defined(__HIPCC__)
#define HSPMD_INDEX __host__ __device__ __forceinline__ constexpr
#else
#define HSPMD_INDEX constexpr inline
#endif

constexpr int kUnitKeys = 128;       // keys are shared out in units of these
constexpr int kFewRows = 16;         // rows per tile of the kernel for few rows ...
constexpr int kManyRows = 128;       // ... and of the one for many
constexpr int kChunkTarget = 512;    // chunks to aim for: two for each of the 256 compute units
constexpr int kXcds = 8;             // workgroups go to the XCDs in turn
constexpr int kWindowPages = 2048;   // page numbers kept in LDS at a time (32768 keys of the smallest pages)

// A sequence's rows and keys as the device arrays give them, clamped to what there is.
struct SeqRows {
    int start, n, kv;
};
HSPMD_INDEX SeqRows seq_rows(int cu, int cu_next, int kv_len, int total_rows, int table_width, int page_shift) {
    const int start = cu < 0 ? 0 : cu > total_rows ? total_rows : cu;
    const int end = cu_next < start ? start : cu_next > total_rows ? total_rows : cu_next;
    const int64_t most = (int64_t)table_width << page_shift, cap = most < 0x7fffff00 ? most : 0x7fffff00;
    const int kv = kv_len < 0 ? 0 : kv_len > cap ? (int)cap : kv_len;
    return SeqRows{start, end - start, kv};
}

// Row tiles of a (sequence, KV head), and units of keys.  The kernel for few rows takes sequences with up to `few_limit` rows
// (new tokens x query heads of a KV head), the one for many the others.
struct SeqTiles {
    int tiles, units;
};
HSPMD_INDEX SeqTiles seq_tiles(const SeqRows& s, int group, int tile_rows, bool many, int few_limit) {
    const int64_t rows = (int64_t)s.n * group;
    if (rows == 0 || (rows > few_limit) != many) return SeqTiles{0, 0};
    const int units = (s.kv + kUnitKeys - 1) / kUnitKeys;
    return SeqTiles{(int)((rows + tile_rows - 1) / tile_rows), units > 1 ? units : 1};
}

// With U the units of all items together, a chunk is to take about U / kChunkTarget of them: the device then has about as many chunks as it
// takes at once, whatever the mix of lengths.
HSPMD_INDEX int units_per_chunk(int64_t all_units) {
    const int64_t per = (all_units + kChunkTarget - 1) / kChunkTarget;
    return per < 1 ? 1 : per > (1 << 24) ? (1 << 24) : (int)per;
}
// Chunks of an item: to the nearest number, so that an item a little longer than the others is not cut for it.
struct Shares {
    int chunks, units;   // units of each
};
HSPMD_INDEX Shares shares_of(int units, int per_chunk) {
    const int chunks = (int)((2 * (int64_t)units + per_chunk) / (2 * (int64_t)per_chunk));
    const int c = chunks < 1 ? 1 : chunks;
    return Shares{c, (units + c - 1) / c};
}

// Slots are dealt out to the XCDs in runs: neighbouring slots are row tiles that read the same keys, and meet in one L2.
// -1: the workgroup has none.
HSPMD_INDEX int64_t slot_of_block(int64_t block, int64_t slots) {
    const int64_t run = (slots + kXcds - 1) / kXcds, slot = block % kXcds * run + block / kXcds;
    return block / kXcds < run && slot < slots ? slot : -1;
}
// slot within a sequence -> KV head, chunk, row tile (tiles innermost)
struct SlotPlace {
    int head, chunk, tile;
};
HSPMD_INDEX SlotPlace place_of_slot(int64_t local, int tiles, int chunks) {
    const int64_t rest = local / tiles;
    return SlotPlace{(int)(rest / chunks), (int)(rest % chunks), (int)(local % tiles)};
}
// tile of partial results of an item's first chunk, counted from the sequence's first; its chunks follow each other
HSPMD_INDEX int64_t part_of(const SlotPlace& p, int tiles, int chunks) { return ((int64_t)p.head * tiles + p.tile) * chunks; }

// What the host can say about the number of workgroups and of partial results.  A chunk count is at most units / per_chunk + 1 and, where it is
// above one, at most 2 units / per_chunk; the sum of units / per_chunk is at most kChunkTarget.
struct GridBounds {
    int64_t grid, part_tiles;
};
HSPMD_INDEX GridBounds grid_bounds(int64_t total_rows, int64_t num_seqs, int64_t table_width, int page_shift, int64_t group, int64_t kv_heads,
                                   bool many, int few_limit) {
    const int64_t least_n = few_limit / group + 1;                     // tokens of a sequence that is not for the kernel for few rows
    const int64_t seqs = num_seqs < total_rows ? num_seqs : total_rows;
    const int64_t tile_rows = many ? kManyRows : kFewRows;
    int64_t full = total_rows * group / tile_rows, ends = seqs;        // full tiles, and one that may not be full per sequence
    if (many) {
        const int64_t fit = total_rows / least_n;
        ends = seqs < fit ? seqs : fit;
        if (ends == 0) full = 0;
    } else if (few_limit < total_rows * group) {
        const int64_t most = seqs * ((few_limit + tile_rows - 1) / tile_rows);
        full = full + ends < most ? full : most - ends;
        full = full < 0 ? 0 : full;
    }
    const int64_t items = kv_heads * (full + ends);
    const int64_t u = ((table_width << page_shift) + kUnitKeys - 1) / kUnitKeys, units = items * (u < 1 ? 1 : u);
    const int64_t slots = units < items + kChunkTarget ? units : items + kChunkTarget;
    return GridBounds{(slots + kXcds - 1) / kXcds * kXcds, units < 2 * kChunkTarget ? units : 2 * kChunkTarget};
}

}  // namespace hspmd
