// What a workgroup of the attention over the paged cache works on, and the tail that its kernels share (gfx950 only).
#pragma once
#include "paged_device.hpp"

namespace hspmd {

struct PagedItem {
    int seq;               // -1: none
    int row_start, n;      // the sequence's rows
    int kv;                // keys in the cache
    int tile, head;        // row tile, KV head
    int chunk, chunks;     // which share of the keys
    int units;             // units per share
    int part;              // tile of partial results of the item's first chunk (chunks > 1)
};

// Sums over the lanes up to each one (DPP: within rows of 16 lanes, then across them; no LDS)
__device__ __forceinline__ uint32_t lanes_up_to(uint32_t x) {
    auto add = [&](auto ctrl, auto row_mask) {
        x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(row_mask)::value, 0xf, false);
    };
    using std::integral_constant;
    add(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});   // row_shr 1, 2, 4, 8
    add(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
    add(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
    add(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
    add(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // the last lane of rows 0, 2 to rows 1, 3
    add(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});   // lane 31 to rows 2, 3
    return x;
}
__device__ __forceinline__ uint32_t all_lanes(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)lanes_up_to(x), 63); }

// the sequence's rows and keys, and its row tiles and units of keys; behind the last: a sequence without rows
template <bool MANY>
__device__ __forceinline__ void look_at(const PagedAttnParams& p, int seq, SeqRows& s, SeqTiles& t) {
    const int in = min(seq, p.rows.num_seqs - 1), begin = p.rows.cu_rows[in];
    s = seq_rows(begin, seq == in ? p.rows.cu_rows[in + 1] : begin, p.rows.kv_lens[in], p.rows.total_rows, p.rows.table_width, p.pool.page_shift);
    t = seq_tiles(s, p.group, MANY ? kManyRows : kFewRows, MANY, p.few_limit);
}

// The workgroup's item from the plan that a launch in front has made (more than kPlanAbove sequences)
template <bool MANY>
__device__ __forceinline__ PagedItem planned_item(const PagedAttnParams& p) {
    const uint32_t* const plan = p.plan + (MANY ? plan_words(p.rows.num_seqs) : 0);
    PagedItem it{};
    it.seq = __builtin_amdgcn_readfirstlane(interval_of(plan + 1, p.rows.num_seqs, (uint32_t)blockIdx.x));
    if (it.seq < 0) return it;
    SeqRows s;
    SeqTiles t;
    look_at<MANY>(p, it.seq, s, t);
    const Shares sh = shares_of(t.units, (int)plan[0]);
    const uint32_t local = blockIdx.x - plan[1 + it.seq];
    if (local >= (uint32_t)(t.tiles * p.pool.kv_heads * sh.chunks)) { it.seq = -1; return it; }
    const SlotPlace at = place_of_slot(local, t.tiles, sh.chunks, p.pool.kv_heads);
    const int64_t mine = plan[2 + p.rows.num_seqs + it.seq] + part_of(at, t.tiles, sh.chunks);
    return PagedItem{it.seq, s.start, s.n, s.kv, at.tile, at.head, at.chunk, sh.chunks, sh.units,
                     (int)min(mine, (int64_t)(0x7fffffff / (MANY ? kManyRows : kFewRows)))};
}

// The workgroup's item, worked out by every wave for itself from the lengths on the device (sums over the sequences, without LDS or a barrier;
// no launch in front).  A lane takes every 64th sequence, and slots go by lanes first.  The arrays hold anything: rows and lengths are clamped, and what a sum
// that overflows leads to stays inside its sequence's tiles.
template <bool MANY>
__device__ __forceinline__ PagedItem find_item(const PagedAttnParams& p) {
    if (p.plan) return planned_item<MANY>(p);
    constexpr int kRows = MANY ? kManyRows : kFewRows;
    const int lane = threadIdx.x & 63, kvh = p.pool.kv_heads;
    const int per_lane = (p.rows.num_seqs + 63) / 64;
    SeqRows s{};
    SeqTiles t{};
    auto look = [&](int i) { look_at<MANY>(p, i * 64 + lane, s, t); };      // the lane's sequence i
    int64_t units = 0;
    for (int i = 0; i < per_lane; ++i) {
        look(i);
        units += (int64_t)t.tiles * t.units * kvh;
    }
    // (a 64-bit sum in two parts that do not overflow)
    const int first_per = units_per_chunk(((int64_t)all_lanes((uint32_t)(units >> 20)) << 20) + all_lanes((uint32_t)units & 0xfffffu), MANY);
    auto slots_of = [&](const Shares& sh) { return (uint32_t)(t.tiles * kvh * sh.chunks); };
    int per_chunk = first_per;
    uint32_t slots = 0, parts = 0;
    for (int raise = 0;; ++raise) {
        slots = parts = 0;
        for (int i = 0; i < per_lane; ++i) {
            if (per_lane > 1) look(i);                      // (with one per lane it is still there)
            const Shares sh = shares_of(t.units, per_chunk);
            const uint32_t n = slots_of(sh);
            slots += n;
            parts += sh.chunks > 1 ? n : 0;
        }
        const int next = raise < kRaises ? raised(per_chunk, first_per, all_lanes(slots), MANY) : per_chunk;
        if (next == per_chunk) break;
        per_chunk = next;
    }
    const uint32_t slots_to = lanes_up_to(slots), parts_to = lanes_up_to(parts);
    const uint32_t slot = blockIdx.x;
    PagedItem it{};
    it.seq = -1;
    uint32_t first = slots_to - slots, part = parts_to - parts;
    if (slot >= first && slot < slots_to)
        for (int i = 0; i < per_lane; ++i) {
            if (per_lane > 1) look(i);
            const Shares sh = shares_of(t.units, per_chunk);
            const uint32_t n = slots_of(sh);
            if (slot - first < n) {
                const SlotPlace at = place_of_slot(slot - first, t.tiles, sh.chunks, kvh);
                const int64_t mine = part + part_of(at, t.tiles, sh.chunks);
                it = PagedItem{i * 64 + lane, s.start, s.n, s.kv, at.tile, at.head, at.chunk, sh.chunks, sh.units,
                               (int)min(mine, (int64_t)(0x7fffffff / kRows))};
                break;
            }
            first += n;
            part += sh.chunks > 1 ? n : 0;
        }
    const uint64_t owner = __ballot(it.seq >= 0);
    const int from = owner ? __builtin_ctzll(owner) : 0;
    int* const words = reinterpret_cast<int*>(&it);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(PagedItem) / 4); ++i) words[i] = __builtin_amdgcn_readlane(words[i], from);
    return it;
}

// Where a row's results are, for the join: tile of partial results of the first chunk and row in it, and number of chunks with the kind of tile
__device__ __forceinline__ int2 where_entry(int64_t first_row, int chunks, bool many) { return make_int2((int)first_row, chunks | (many ? 1 << 30 : 0)); }

}  // namespace hspmd
