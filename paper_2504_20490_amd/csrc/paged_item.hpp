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

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}

// The workgroup's item, worked out by every workgroup for itself from the lengths on the device (two sums over the sequences: a few
// microseconds at most, and no launch in front).  The arrays hold anything: sums are 64-bit, rows and lengths clamped.
template <bool MANY>
__device__ __forceinline__ PagedItem find_item(const PagedAttnParams& p) {
    __shared__ int64_t sums[2][4];
    __shared__ PagedItem found;
    constexpr int kRows = MANY ? kManyRows : kFewRows;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, kvh = p.pool.kv_heads;
    SeqRows s{};
    SeqTiles t{};
    auto look = [&](int seq) {
        t = SeqTiles{0, 0};
        if (seq >= p.rows.num_seqs) return;
        s = seq_rows(p.rows.cu_rows[seq], p.rows.cu_rows[seq + 1], p.rows.kv_lens[seq], p.rows.total_rows, p.rows.table_width, p.pool.page_shift);
        t = seq_tiles(s, p.group, kRows, MANY, p.few_limit);
    };
    auto block_sums = [&](int64_t x, int64_t y) {          // of the workgroup, left in sums[]
        x = wave_sum(x), y = wave_sum(y);
        __syncthreads();
        if (lane == 0) { sums[0][wave] = x; sums[1][wave] = y; }
        __syncthreads();
    };
    const int strips = (p.rows.num_seqs + kThreads - 1) / kThreads;
    int64_t units = 0, slots = 0;
    for (int i = 0; i < strips; ++i) {
        look(i * kThreads + threadIdx.x);
        units += (int64_t)t.tiles * t.units * kvh;
    }
    if (threadIdx.x == 0) found.seq = -1;
    block_sums(units, 0);
    const int per_chunk = units_per_chunk(sums[0][0] + sums[0][1] + sums[0][2] + sums[0][3]);
    auto slots_of = [&](const Shares& sh) { return (int64_t)t.tiles * kvh * sh.chunks; };
    for (int i = 0; i < strips; ++i) {
        if (strips > 1) look(i * kThreads + threadIdx.x);  // (with one strip the thread's sequence is still there)
        slots += t.tiles ? slots_of(shares_of(t.units, per_chunk)) : 0;
    }
    block_sums(slots, 0);
    const int64_t slot = slot_of_block(blockIdx.x, sums[0][0] + sums[0][1] + sums[0][2] + sums[0][3]);
    int64_t slot_base = 0, part_base = 0;
    for (int i = 0; i < strips && slot >= slot_base; ++i) {
        if (strips > 1) look(i * kThreads + threadIdx.x);
        const Shares sh = shares_of(t.units, per_chunk);
        const int64_t mine = t.tiles ? slots_of(sh) : 0, parts = sh.chunks > 1 ? mine : 0;
        int64_t x = mine, y = parts;                       // inclusive sums over the wave
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t a = __shfl_up(x, o, 64), b = __shfl_up(y, o, 64);
            if (lane >= o) { x += a; y += b; }
        }
        __syncthreads();
        if (lane == 63) { sums[0][wave] = x; sums[1][wave] = y; }
        __syncthreads();
        int64_t first = slot_base + x - mine, part = part_base + y - parts;
        for (int w = 0; w < wave; ++w) { first += sums[0][w]; part += sums[1][w]; }
        if (slot >= first && slot < first + mine) {
            const SlotPlace at = place_of_slot(slot - first, t.tiles, sh.chunks);
            part += part_of(at, t.tiles, sh.chunks);
            found = PagedItem{i * kThreads + (int)threadIdx.x, s.start, s.n, s.kv, at.tile, at.head, at.chunk, sh.chunks, sh.units,
                              (int)min(part, (int64_t)(0x7fffffff / kRows))};
        }
        for (int w = 0; w < 4; ++w) { slot_base += sums[0][w]; part_base += sums[1][w]; }
    }
    __syncthreads();
    PagedItem it = found;
    // the same in all lanes: scalar values from here on
    int* const words = reinterpret_cast<int*>(&it);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(PagedItem) / 4); ++i) words[i] = __builtin_amdgcn_readfirstlane(words[i]);
    return it;
}

// The numbers of pages first_page .. first_page + count - 1 of the item's sequence into LDS (all threads, no barrier).  A number that does
// not exist is replaced by 0 and the page's first key noted: what is read there is shown to nobody.
__device__ __forceinline__ void load_pages(const PagedAttnParams& p, int seq, int first_page, int count, int* pages, int* bad_key) {
    for (int i = threadIdx.x; i < count; i += kThreads) {
        int page = page_at(p.pool, p.rows, seq, first_page + i);
        if (page < 0) {
            atomicMin(bad_key, (first_page + i) << p.pool.page_shift);
            page = 0;
        }
        pages[i] = page;
    }
}

// Where a row's results are, for the join: tile of partial results of the first chunk and row in it, and number of chunks with the kind of tile
__device__ __forceinline__ int2 where_entry(int64_t first_row, int chunks, bool many) { return make_int2((int)first_row, chunks | (many ? 1 << 30 : 0)); }

}  // namespace hspmd
