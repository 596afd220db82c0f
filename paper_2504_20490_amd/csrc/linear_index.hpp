// Which tokens, states and workspace entries a workgroup of the linear attention takes.  Plain index arithmetic, usable on the host as
// well: that every segment is taken once and that nothing leads out of the grid or the workspace is tested there.
#pragma once
#include <stdint.h>

namespace hspmd {

#if defined(__HIPCC__)
#define HSPMD_LINEAR_INDEX __host__ __device__ __forceinline__ constexpr
#else
#define HSPMD_LINEAR_INDEX constexpr inline
#endif

constexpr int kLinearChunk = 64;     // tokens whose pairs are formed; states pass from chunk to chunk

// A sequence's rows as the device array gives them, clamped to what there is.
struct LinearRows {
    int start, n;
};
HSPMD_LINEAR_INDEX LinearRows linear_rows(int cu, int cu_next, int total_rows) {
    const int start = cu < 0 ? 0 : cu > total_rows ? total_rows : cu;
    const int end = cu_next < start ? start : cu_next > total_rows ? total_rows : cu_next;
    return LinearRows{start, end - start};
}

// A sequence is cut into segments of at most seg_rows tokens (a multiple of the chunk, at least four), as few as that takes, of equal length in chunks but
// for the last, which is never empty; at least one.  Segment b of sequence s is slot
// start / seg_rows + s + b of the launch: the next sequence's first slot, (start + n) / seg_rows + s + 1, is never less than that of the
// last segment plus one, so every slot is taken once at most, by a rule that needs no sums over the sequences.
HSPMD_LINEAR_INDEX int linear_first_slot(int start, int seq, int seg_rows) { return start / seg_rows + seq; }
HSPMD_LINEAR_INDEX int linear_segments(int n, int seg_rows) { return n <= seg_rows ? 1 : (n + seg_rows - 1) / seg_rows; }
HSPMD_LINEAR_INDEX int linear_segment_rows(int n, int count) {
    return ((n + kLinearChunk - 1) / kLinearChunk + count - 1) / count * kLinearChunk;
}
HSPMD_LINEAR_INDEX int64_t linear_slots(int64_t total_rows, int64_t num_seqs, int64_t seg_rows) { return total_rows / seg_rows + num_seqs; }

// Sequences of several segments have an entry in the workspace for each (the state that reaches it): from 2 start / seg_rows on.  With n >
// seg_rows the next sequence's first entry is at least 2 (segments - 1) further, which is never less than the number of segments.
HSPMD_LINEAR_INDEX int linear_first_entry(int start, int seg_rows) { return (int)(2 * (int64_t)start / seg_rows); }
HSPMD_LINEAR_INDEX int64_t linear_entries(int64_t total_rows, int64_t seg_rows) { return 2 * total_rows / seg_rows + 1; }

// Anchors: chunks of a segment whose states are kept for the decays' gradients, the fourth from its end and every fourth in front of that, without the segment's first.
// A segment's number of them is at most (rows - 1) / 256, so they have entries of their own from start / 256 on.
constexpr int kLinearAnchor = 4;     // chunks
HSPMD_LINEAR_INDEX int linear_first_anchor(int start) { return start / (kLinearAnchor * kLinearChunk); }
HSPMD_LINEAR_INDEX int64_t linear_anchors(int64_t total_rows) { return total_rows / (kLinearAnchor * kLinearChunk); }
HSPMD_LINEAR_INDEX bool linear_is_anchor(int chunk, int chunks) { return chunk > 0 && (chunks - chunk) % kLinearAnchor == 0; }
HSPMD_LINEAR_INDEX int linear_anchor(int start, int chunk, int chunks) { return linear_first_anchor(start) + (chunks - chunk) / kLinearAnchor - 1; }
// What an anchor keeps: a state's rows and columns that head_dim takes, in whole groups of 16 and 32
HSPMD_LINEAR_INDEX int linear_anchor_elements(int head_dim) { return (head_dim + 15) / 16 * 16 * ((head_dim + 31) / 32 * 32); }

// The sequence of several segments that starts in window w (tokens w * seg_rows .. + seg_rows - 1), if there is one, is the last that
// starts there; windows are what the launch that passes states from segment to segment goes by.
HSPMD_LINEAR_INDEX int64_t linear_windows(int64_t total_rows, int64_t seg_rows) { return total_rows / seg_rows + 1; }

// Columns of a state that a workgroup of the single step takes; `states` of the launch.  Narrow pieces of rows are read and written in more places at once, but a line of 128
// bytes that two of them share moves twice.  us at 4 query heads each (d = 104, 120: one, 96: four), pieces in the order 32, 64 columns, whole rows:
//   d = 128: 64 states 7.6, 8.3, 11.1; 512 states 16.0, 16.6, 18.7; 640 states 24.2, 21.3, 22.9; 4096 states 112, 111, 125: 32 to 2^23 elements, 64 from there on
//   d = 96: 64 states 6.7, 7.0, 8.6; 768 states 19.5, 19.7, 17.9; 4096 states 70, 72, 79: likewise
//   d = 104: 64 states 9.9, 7.0, 7.5; 128 states 10.9, 8.3, 8.3; 512 states 17.6, 15.2, 14.1; 8192 states 224, 198, 144: 64 for few
//   d = 120: 64 states 7.9, 7.7, 8.4; 192 states 11.9, 11.2, 10.9; 8192 states 296, 264, 180: likewise
//   up to 88 and at 64: whole rows throughout (d = 64: 512 states 11.6, whole 8.3; d = 72: 128 states 11.1, 7.0, d = 40: 256 states 10.2, 5.0)
HSPMD_LINEAR_INDEX int linear_step_columns(int head_dim, int64_t states) {
    const int64_t elements = states * head_dim * head_dim;
    if (head_dim <= 64) return head_dim;
    if (head_dim % 32 == 0) return elements <= (1 << 23) ? 32 : 64;
    return head_dim > 96 && elements <= (1 << 20) ? 64 : head_dim;
}

// Workgroups go to the 8 XCDs in turn.  Items do so four heads at a time (`granule` items: four heads, all that is computed for them): neighbouring heads share
// lines of the decays and the edges of rows, which then meet in one L2, and every XCD has as many items as another but for one granule.  (All heads of a slot
// on one XCD, ranges of slots, left some with a round of workgroups more.)  The grid is 8 * granule * rounds; items from `items` on are none.
HSPMD_LINEAR_INDEX int64_t linear_grid(int64_t items, int granule) { return (items + 8 * granule - 1) / (8 * granule) * 8 * granule; }
HSPMD_LINEAR_INDEX int64_t linear_item(int64_t block, int granule) {
    const int64_t i = block / 8;
    return (i / granule * 8 + block % 8) * granule + i % granule;
}

}  // namespace hspmd
