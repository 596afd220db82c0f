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

constexpr int kFewRows = 16;         // rows per tile of the kernel for few rows ...
constexpr int kManyRows = 128;       // ... and of the one for many
// Keys are shared out in units of so many.
HSPMD_INDEX int unit_keys(bool many) { return many ? 128 : 32; }
// Chunks to aim for, over the 256 compute units.  Few rows: 8 waves each, as many as a unit holds with 8-bit tiles at D = 128; with 16-bit tiles
// (4 waves) that is two rounds, which even out lengths better than one (64 sequences of 500 .. 16000 keys, 32 heads on 8, one token: bf16 217
// against 231 us with half as many, e4m3 126 against 164; of 4265 keys each bf16 209 against 206, e4m3 121 against 116 to 133).  Many rows: 2 workgroups each, which
// is what a unit holds.
HSPMD_INDEX int chunk_target(bool many) { return many ? 512 : 2048; }

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
// Every row tile counts all keys of its sequence.  It walks those up to its last row only: the same but for the sequence's own new tokens, so exact for single tokens and close behind a long
// prefix; in a prompt without one the last chunks of the first tiles are empty and the last tiles have up to twice the mean (one of 2048, 16 heads: 52 us, the packed forward 34).
struct SeqTiles {
    int tiles, units;
};
HSPMD_INDEX SeqTiles seq_tiles(const SeqRows& s, int group, int tile_rows, bool many, int few_limit) {
    const int64_t rows = (int64_t)s.n * group;
    if (rows == 0 || (rows > few_limit) != many) return SeqTiles{0, 0};
    const int units = (int)(((int64_t)s.kv + unit_keys(many) - 1) / unit_keys(many));
    return SeqTiles{(int)((rows + tile_rows - 1) / tile_rows), units > 1 ? units : 1};
}

// With U the units of all items together, a chunk is to take U / chunk_target() of them, so that the device has as many chunks as it takes at
// once, whatever the mix of lengths; an item's chunks are equal.  Items that end in a short chunk make them more than that: the units per
// chunk are raised until they are not, by a factor of two at most (where there are more items than that, nothing is gained by it).
HSPMD_INDEX int units_per_chunk(int64_t all_units, bool many) {
    const int64_t per = (all_units + chunk_target(many) - 1) / chunk_target(many);
    return per < 1 ? 1 : per > (1 << 24) ? (1 << 24) : (int)per;
}
constexpr int kRaises = 3;
HSPMD_INDEX int raised(int per_chunk, int first, int64_t slots, bool many) {
    if (slots <= chunk_target(many)) return per_chunk;
    const int64_t more = (per_chunk * slots + chunk_target(many) - 1) / chunk_target(many);
    return more < 2 * (int64_t)first ? (int)more : 2 * first;
}
struct Shares {
    int chunks, units;   // units of each
};
HSPMD_INDEX Shares shares_of(int units, int per_chunk) {    // (32-bit: a 64-bit division takes a hundred instructions)
    const unsigned c = ((unsigned)units + (unsigned)per_chunk - 1u) / (unsigned)per_chunk;
    return Shares{c < 1 ? 1 : (int)c, c < 1 ? 0 : (int)(((unsigned)units + c - 1) / c)};
}

// slot within a sequence -> KV head, chunk, row tile.  The last row tiles, which see the most keys, come first (a workgroup that starts late has
// little to do); heads are innermost: workgroups go to the XCDs in turn, so that with 8 heads, or 16, the tiles and chunks of a head meet in one L2.
// 12 prompts of 300 .. 4000 tokens, 16 heads, 165 us against 215 with the heads outermost and first tiles first.
struct SlotPlace {
    int head, chunk, tile;
};
HSPMD_INDEX SlotPlace place_of_slot(uint32_t local, int tiles, int chunks, int heads) {
    const uint32_t rest = local / (uint32_t)heads;
    return SlotPlace{(int)(local % (uint32_t)heads), (int)(rest % (uint32_t)chunks), tiles - 1 - (int)(rest / (uint32_t)chunks)};
}
// tile of partial results of an item's first chunk, counted from the sequence's first; its chunks follow each other
HSPMD_INDEX int64_t part_of(const SlotPlace& p, int tiles, int chunks) { return ((int64_t)p.head * tiles + p.tile) * chunks; }

// With many sequences the sums over them are made once, by a launch in front, and kept in the workspace.  Words for each kernel: the units per chunk;
// the first slot of every sequence, and the end of the last one's; the first tile of partial results of every sequence.  Fewer: every workgroup
// sums for itself, up to 3 sequences per lane (one token each over 48 keys, 8 heads: 128 sequences 14 us against 18.6 with the launch, 192 19.4 against 21,
// 256 22.9 against 19, 2048 425 against 69; 4096 of 20 tokens 7.1 ms against 0.46).
constexpr int kPlanAbove = 192;
HSPMD_INDEX int64_t plan_words(int64_t num_seqs) { return 2 * num_seqs + 2; }

// What the host can say about the number of workgroups and of partial results.  A chunk count is at most units / per_chunk + 1 and, where it is
// above one, at most 2 units / per_chunk; the sum of units / per_chunk is at most chunk_target().
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
    const int64_t u = ((table_width << page_shift) + unit_keys(many) - 1) / unit_keys(many), units = items * (u < 1 ? 1 : u);
    const int64_t target = chunk_target(many), slots = units < items + target ? units : items + target;
    return GridBounds{slots, units < 2 * target ? units : 2 * target};
}

}  // namespace hspmd
