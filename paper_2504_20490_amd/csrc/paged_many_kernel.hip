// Attention of new tokens over the paged cache: many rows per sequence and KV head (prompts, chunks of them).
//
// Bound by the matrix cores and the softmax beside them, like the forward over packed sequences, whose iteration over a 64-key
// tile it shares (fwd_iteration: S^T = K Q^T of the next tile under the exponentials of this one, then O^T += V^T P^T).  A workgroup takes 128
// rows of one KV head, token by token and within a token query head by query head: all query heads of a group use the same copy of a key
// tile, and a short chunk of a grouped model still fills the rows.  What differs is where a tile comes from: a wave's copy of 1 KB lies
// in one page (16 tokens at least), so its base is a scalar, worked out from page numbers that the workgroup keeps in LDS.
// 8-bit tiles go through registers: fetched an iteration ahead, scaled to bf16 (exact) and written to the tile, in the same places of the
// schedule where the 16-bit copies are issued; the tile and all that follows is the same.
// Weights are rounded to bf16 for their product with the values, as in the packed forward (O 2.3e-3 from the formula in 64 bits, 1.7e-3 of it its own rounding); two
// bf16 parts, as for few rows, take half as many matrix instructions again: 902 -> 1238 us for the first case below.
// 2048 tokens behind 27034, 32 heads on 8 of 128: bf16 877 to 923 us on six cards = 1020 to 1070 TFLOP/s of the visible pairs (a large bf16 matrix product here:
// 1330), e4m3 926 to 943 (the conversions are vector work beside the softmax).  8 prompts of 2048, 16 heads: 182 us = 757 TFLOP/s, the packed forward 151: items of 2 to 32 tiles, whose start
// (lengths, page numbers, first tiles) and masked tiles weigh more, dealt out as if each had all keys (seq_tiles).  16 sequences of 4 tokens, 64 heads on 8, 16000 keys (32 rows per
// KV head): bf16 202 us = 5.2 TB/s, e4m3 126 us = 4.2.
#include "fwd_iteration.hpp"
#include "paged_item.hpp"

namespace hspmd {

namespace {

constexpr int kTileKeys = kFwdKTile;
constexpr int kWindowPages = 2048;   // page numbers kept in LDS at a time (32768 keys of the smallest pages)

// Where the item's keys lie.  A copy of 1 KB (kRowsPerPiece rows) stays within a page.
template <int D, bool E4M3>
struct PagedSource {
    static constexpr int kRowBytes = D * (E4M3 ? 1 : 2);              // of a row as it is copied
    static constexpr int kRowsPerPiece = 1024 / kRowBytes;
    static constexpr int kPieces = kTileKeys / kRowsPerPiece / 4;     // per wave and tile
    const PagedPool* pool;
    const int* pages;          // LDS: page numbers from first_page on
    int first_page, end;       // end: first key behind the window
    int64_t head_row;          // head << page_shift
    int wave;

    __device__ __forceinline__ int first_row(int i) const { return (i * 4 + wave) * kRowsPerPiece; }
    // lane i: the page number of the wave's piece i of the tile that starts at key0 (pieces behind the end: the last page's)
    __device__ __forceinline__ int page_numbers(int key0) const {
        const int key = min(key0 + first_row((int)(threadIdx.x & 3)), end - 1);
        return pages[(key >> pool->page_shift) - first_page];
    }
    __device__ __forceinline__ int64_t row_of(int key0, int i) const {
        return head_row + ((key0 + first_row(i)) & ((1 << pool->page_shift) - 1));
    }
    __device__ __forceinline__ int64_t offset(int page, int key0, int i) const {
        return page * pool->page_bytes + row_of(key0, i) * pool->row_bytes;
    }
};

// 16-bit tiles: direct copies to LDS
template <int D>
struct DirectLoad {
    using Source = PagedSource<D, false>;
    static constexpr int kPieces = Source::kPieces;
    const Source* src;
    uint32_t lane_offset;      // of this lane's 16 bytes from the piece's first row
    uint32_t k_dst, v_dst;     // LDS
    int k_key0, v_key0;        // first keys of the tiles
    int k_pages, v_pages;      // lane i: page number of piece i
    __device__ __forceinline__ void piece(const uint8_t* base, uint32_t dst, int pages, int key0, int i) const {
        global_to_lds<16>(base + src->offset(__builtin_amdgcn_readlane(pages, i), key0, i), lane_offset, dst + (i * 4 + src->wave) * 1024);
    }
    __device__ __forceinline__ void k_piece(int i) const { piece(src->pool->k, k_dst, k_pages, k_key0, i); }
    __device__ __forceinline__ void v_piece(int i) const { piece(src->pool->v, v_dst, v_pages, v_key0, i); }
};

// 8-bit tiles: a piece that was fetched an iteration ago is converted and written, and the tile after it fetched
template <int D>
struct ConvertLoad {
    using Source = PagedSource<D, true>;
    static constexpr int kPieces = Source::kPieces;
    struct Raw {
        u32x4 bytes[kPieces];
        uint32_t scale[kPieces];
    };
    const Source* src;
    Raw* k_raw;
    Raw* v_raw;
    char* k_dst;               // the tiles that the pieces go to ...
    char* v_dst;
    int k_next, v_next;        // ... and first keys of those that are fetched,
    int k_pages, v_pages;      // with (lane i) the page number of piece i
    uint32_t lane_offset;      // of this lane's 16 bytes from the piece's first row
    __device__ __forceinline__ void fetch(Raw& raw, bool v, int pages, int key0, int i) const {
        const int page = __builtin_amdgcn_readlane(pages, i);
        const uint8_t* base = (v ? src->pool->v : src->pool->k) + src->offset(page, key0, i);
        raw.bytes[i] = *reinterpret_cast<const u32x4*>(base + lane_offset);
        const uint8_t* scales = (v ? src->pool->v_scale : src->pool->k_scale) + page * src->pool->scale_page_bytes + src->row_of(key0, i);
        raw.scale[i] = scales[(uint32_t)(threadIdx.x & 63) / (D / 16)];
    }
    __device__ __forceinline__ void convert(const Raw& raw, char* tile, int i) const {
        const int lane = threadIdx.x & 63, row = src->first_row(i) + lane / (D / 16), col = lane % (D / 16) * 16;
        const float scale = scale_of(raw.scale[i]);
        const u32x4 x = raw.bytes[i];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const u32x2 a = e4m3_to_bf16(x[2 * half], scale), b = e4m3_to_bf16(x[2 * half + 1], scale);
            *reinterpret_cast<u32x4*>(tile + tile_offset<D>(row, col + half * 8)) = u32x4{a[0], a[1], b[0], b[1]};
        }
    }
    __device__ __forceinline__ void k_piece(int i) const {
        convert(*k_raw, k_dst, i);
        fetch(*k_raw, false, k_pages, k_next, i);
    }
    __device__ __forceinline__ void v_piece(int i) const {
        convert(*v_raw, v_dst, i);
        fetch(*v_raw, true, v_pages, v_next, i);
    }
};

template <int D, int KD, bool E4M3>
__global__ __launch_bounds__(kThreads, 2) void paged_many_kernel(PagedAttnParams p) {
    using G = FwdGeom<D, KD>;
    using Source = PagedSource<D, E4M3>;
    using Load = typename std::conditional<E4M3, ConvertLoad<D>, DirectLoad<D>>::type;
    constexpr int KK = G::KK, DB = G::DB, BK = kTileKeys, kTileBytes = G::kTileBytes;
    __shared__ __attribute__((aligned(1024))) char lds[4 * kTileBytes];      // K tiles kt+1 / kt+2 and V tiles kt / kt+1
    __shared__ int pages[kWindowPages + 1];
    __shared__ int bad_key, taken_out;
    char* const kbuf0 = lds;
    char* const vbuf0 = lds + 2 * kTileBytes;

    const PagedItem it = find_item<true>(p);
    if (it.seq < 0) return;
    const int lane = threadIdx.x & 63, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hd = p.pool.head_dim, shift = p.pool.page_shift;
    const float c = p.scale_log2;

    // rows: this lane's, and the wave's first and last that exist
    const int wave_row0 = it.tile * kManyRows + wave * 32;
    const int rho = wave_row0 + (lane & 31);
    const int token = rho / p.group, q_head = it.head * p.group + rho % p.group;
    const bool real = token < it.n;
    const int offset = it.kv - it.n;                                  // position of the sequence's first row
    const int my_limit = real ? offset + token : -1;
    const bool wave_real = wave_row0 / p.group < it.n;
    const int first_limit = offset + wave_row0 / p.group, group_limit = offset + it.tile * kManyRows / p.group;   // ... and the workgroup's first
    const int last_limit = wave_real ? offset + min(it.n - 1, (wave_row0 + 31) / p.group) : -1;
    const int keys_end = max(0, offset + min(it.n - 1, (it.tile * kManyRows + kManyRows - 1) / p.group) + 1);
    const int64_t share = (int64_t)it.units * unit_keys(true);
    const int k0 = (int)min((int64_t)keys_end, it.chunk * share), k1 = (int)min((int64_t)keys_end, (it.chunk + 1) * share);

    FwdState<D, KD, 2> st;
    const uint16_t* const q_row = p.q + (int64_t)(it.row_start + token) * p.q_stride + (int64_t)q_head * hd;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        union { u32x4 u; bf16x8 v; } t;
        t.u = u32x4{0u, 0u, 0u, 0u};
        if (real && kk * 16 + hh * 8 < hd) t.u = *reinterpret_cast<const u32x4*>(q_row + kk * 16 + hh * 8);
        st.qf[kk] = t.v;
        st.rm[kk] = tile_offset<D>(lane & 31, kk * 16 + hh * 8);
    }
    {
        const int c16 = lane & 15, row = (hh << 2) + (c16 >> 2);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const int col = db * 32 + (((lane >> 4) & 1) << 4) + ((c16 & 3) << 2);
            st.tr[db][0] = tile_offset<D>(row, col);
            st.tr[db][1] = tile_offset<D>(row + 8, col);
        }
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.acc[db][i] = 0.f;
    st.m = -INFINITY;
    st.l = 0.f;
    if (threadIdx.x == 0) { bad_key = 0x7fffffff; taken_out = 0; }

    Source src;
    src.pool = &p.pool;
    src.pages = pages;
    src.head_row = (int64_t)it.head << shift;
    src.wave = wave;
    const uint32_t kdst0 = lds_address(lds), vdst0 = kdst0 + 2 * kTileBytes;
    typename ConvertLoad<D>::Raw k_raw, v_raw;                         // (E4M3 only)
    Load load;
    load.src = &src;
    const int last_chunk = p.pool.row_bytes / 16 - 1;
    if constexpr (E4M3) {
        load.k_raw = &k_raw;
        load.v_raw = &v_raw;
        load.lane_offset = (uint32_t)(lane / (D / 16) * p.pool.row_bytes + min(lane % (D / 16), last_chunk) * 16);
    } else {
        const int r = lane / (D / 8);
        load.lane_offset = (uint32_t)(r * p.pool.row_bytes + min(swizzle<D>(src.first_row(0) + r, lane % (D / 8)), last_chunk) * 16);
    }

    for (int w0 = k0; w0 < k1;) {
        const int first_page = w0 >> shift;
        const int w1 = (int)min((int64_t)k1, ((int64_t)first_page + kWindowPages) << shift);
        __syncthreads();                                              // every wave has left the previous window's tiles and numbers
        for (int i = threadIdx.x; i <= ((w1 - 1) >> shift) - first_page; i += kThreads) {
            int page = page_at(p.pool, p.rows, it.seq, first_page + i);
            if (page < 0) {
                atomicMin(&bad_key, (first_page + i) << shift);
                page = 0;                                             // (what is read there is shown to nobody)
            }
            pages[i] = page;
        }
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(st.qf[kk]));   // the row is here before copies are under way
        __syncthreads();
        src.first_page = first_page;
        src.end = w1;

        const int n_tiles = (w1 - w0 + BK - 1) / BK;
        // tiles that hold a key visible to one of the wave's rows; those of them that need no mask and have a successor
        const int n_tiles_w = min(n_tiles, (max(0, last_limit + 1 - w0) + BK - 1) / BK);
        const int n_plain = min(min(max(0, first_limit + 1 - w0), w1 - w0) / BK, n_tiles_w - 1);
        const int n_spread = max(0, min(n_plain, (w1 - w0) / BK - 2));
        auto key0 = [=](int kt) { return w0 + kt * BK; };

        // tile kt of K into K buffer kt & 1, of V into V buffer kt & 1
        auto direct = [&](bool v, int kt) {
            if constexpr (!E4M3) {
                const int numbers = src.page_numbers(key0(kt));
#pragma unroll
                for (int i = 0; i < Source::kPieces; ++i)
                    load.piece(v ? p.pool.v : p.pool.k, (v ? vdst0 : kdst0) + (kt & 1) * kTileBytes, numbers, key0(kt), i);
            }
        };
        auto fetch = [&](bool v, int kt) {
            if constexpr (E4M3) {
                const int numbers = src.page_numbers(key0(kt));
#pragma unroll
                for (int i = 0; i < Source::kPieces; ++i) load.fetch(v ? v_raw : k_raw, v, numbers, key0(kt), i);
            }
        };
        auto convert = [&](bool v, int kt) {
            if constexpr (E4M3) {
#pragma unroll
                for (int i = 0; i < Source::kPieces; ++i)
                    load.convert(v ? v_raw : k_raw, (v ? vbuf0 : kbuf0) + (kt & 1) * kTileBytes, i);
            }
        };
        // A weight of 0 hides a value only if the value is finite.  In tiles that some row of the workgroup does not see to the end (and in
        // what lies behind the last key) infinities and NaN are therefore taken out, each by the wave that brought it, and noted; the rows that do see
        // them get them back at the end.
        const int first_hiding = min(max(0, group_limit + 1 - w0), w1 - w0) / BK;
        auto finite_only = [&](int kt) {
            if (kt < first_hiding) return;
            constexpr int kPiece = Source::kRowsPerPiece * D * 2;
#pragma unroll
            for (int i = 0; i < Source::kPieces; ++i)
#pragma unroll
                for (int j = 0; j < kPiece / 1024; ++j) {
                    char* const at = vbuf0 + (kt & 1) * kTileBytes + (i * 4 + wave) * kPiece + j * 1024 + lane * 16;
                    u32x4 x = *reinterpret_cast<const u32x4*>(at);
                    uint32_t any = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t odd = ((x[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;   // an exponent of all ones
                        any |= odd;
                        x[e] &= ~((odd >> 15) * 0xffffu);
                    }
                    if (any) {
                        *reinterpret_cast<u32x4*>(at) = x;
                        taken_out = 1;
                    }
                }
        };

        // K(0), V(0), K(1); 8 bits: K(2) and V(1) are under way when the loop begins
        if constexpr (E4M3) {
            fetch(false, 0);
            fetch(true, 0);
            convert(false, 0);
            convert(true, 0);
            if (n_tiles > 1) {
                fetch(false, 1);
                fetch(true, 1);
                convert(false, 1);
                fetch(false, 2);
            }
        } else {
            direct(false, 0);
            direct(true, 0);
            if (n_tiles > 1) direct(false, 1);
            wait_tile_loads();
        }
        finite_only(0);
        __syncthreads();
        if (n_tiles_w > 0)
#pragma unroll
            for (int jb = 0; jb < 2; ++jb) {
#pragma unroll
                for (int i = 0; i < 16; ++i) st.s[jb][i] = 0.f;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
                    st.s[jb] = mfma(*reinterpret_cast<const bf16x8*>(kbuf0 + st.rm[kk] + jb * 32 * D * 2), st.qf[kk], st.s[jb]);
            }
        st.tnext = n_tiles_w > 0 ? lane_max(st.s) : -INFINITY;
        if (n_tiles > 2) __syncthreads();                             // iteration 0 brings K(2) where S(0) was read from

        // iteration kt: K(kt+1) and V(kt) are there; brings K(kt+2) and V(kt+1)
        auto arrive = [&](int kt) {
            if (kt > 0) {
                if constexpr (!E4M3) wait_tile_loads();
                finite_only(kt);
                __syncthreads();
            }
        };
        auto bring = [&](int kt) {
            if constexpr (E4M3) {
                if (kt + 2 < n_tiles) { convert(false, kt + 2); fetch(false, kt + 3); }
                if (kt + 1 < n_tiles) { convert(true, kt + 1); fetch(true, kt + 2); }
            } else {
                if (kt + 2 < n_tiles) direct(false, kt + 2);
                if (kt + 1 < n_tiles) direct(true, kt + 1);
            }
        };
        auto step = [&](int kt, auto masked, auto last) {
            arrive(kt);
            bring(kt);
            fwd_iteration<D, KD, 2, decltype(masked)::value, decltype(last)::value, false, true>(
                st, kbuf0 + ((kt + 1) & 1) * kTileBytes, vbuf0 + (kt & 1) * kTileBytes, c, my_limit - key0(kt) - 4 * hh, load);
        };
        auto step_spread = [&](int kt, auto parity) {
            const int par = parity;
            arrive(kt);
            if constexpr (E4M3) {
                load.k_dst = kbuf0 + par * kTileBytes;
                load.v_dst = vbuf0 + (1 - par) * kTileBytes;
                load.k_next = key0(kt + 3);
                load.v_next = key0(kt + 2);
                load.k_pages = src.page_numbers(load.k_next);
                load.v_pages = src.page_numbers(load.v_next);
            } else {
                load.k_dst = kdst0 + par * kTileBytes;
                load.v_dst = vdst0 + (1 - par) * kTileBytes;
                load.k_key0 = key0(kt + 2);
                load.v_key0 = key0(kt + 1);
                load.k_pages = src.page_numbers(load.k_key0);
                load.v_pages = src.page_numbers(load.v_key0);
            }
            fwd_iteration<D, KD, 2, false, false, true, true>(st, kbuf0 + (1 - par) * kTileBytes, vbuf0 + par * kTileBytes, c,
                                                              my_limit - key0(kt) - 4 * hh, load);
        };
        int kt = 0;
        for (; kt + 1 < n_spread; kt += 2) {
            step_spread(kt, std::integral_constant<int, 0>{});
            step_spread(kt + 1, std::integral_constant<int, 1>{});
        }
        for (; kt < n_spread; ++kt) step_spread(kt, kt & 1);
        for (; kt < n_plain; ++kt) step(kt, std::false_type{}, std::false_type{});
        for (; kt < n_tiles_w - 1; ++kt) step(kt, std::true_type{}, std::false_type{});
        if (n_tiles_w > 0) {
            step(kt, std::true_type{}, std::true_type{});
            ++kt;
        }
        for (; kt < n_tiles; ++kt) {
            arrive(kt);
            bring(kt);
        }
        w0 = w1;
    }

    // ---- results.  The row as a new value of the lane index, which the tile loop then does not have to keep.
    int lane_now = threadIdx.x & 63;
    asm volatile("" : "+v"(lane_now));
    const int r = lane_now & 31, half = lane_now >> 5;
    const int my_token = (wave_row0 + r) / p.group, my_head = it.head * p.group + (wave_row0 + r) % p.group;
    const bool exists = my_token < it.n;
    const int seen_to = exists ? offset + my_token : -1;
    float l_row = st.l + partner32(st.l);
    __syncthreads();                                                  // every wave has left the tiles
    if (seen_to >= bad_key) l_row = __builtin_nanf("");
    if (!wave_real) return;
    if (taken_out) {
        // the keys from the start of the first tile that was looked at, or before; 64 at once, one per lane, are searched for what was taken out (there may
        // be nothing: what lies behind the last key is taken out too, and nobody gets it back)
        for (int key0 = max(k0, group_limit + 1 - BK); key0 < k1; key0 += 64) {
            auto row_at = [&](int key, float& scale) {
                const int page = max(page_at(p.pool, p.rows, it.seq, key >> shift), 0);
                const int64_t at = src.head_row + (key & ((1 << shift) - 1));
                if constexpr (E4M3) scale = scale_of(p.pool.v_scale[page * p.pool.scale_page_bytes + at]);
                return p.pool.v + page * p.pool.page_bytes + at * p.pool.row_bytes;
            };
            uint32_t odd = 0;
            if (key0 + lane_now < k1) {
                float scale = 1.f;
                const uint8_t* const row = row_at(key0 + lane_now, scale);
                for (int b = 0; b < p.pool.row_bytes; b += 16) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(row + b);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        odd |= E4M3 ? ((x[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u : ((x[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                }
                if (E4M3 && scale > pow2(119)) odd = 1;                // (the largest scale, 2^120: from 256 times it on the value is infinite)
            }
            for (uint64_t left = __ballot(odd != 0); left; left &= left - 1) {
                const int key = key0 + __builtin_ctzll(left);
                float scale = 1.f;
                const uint8_t* const row = row_at(key, scale);
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const int col = db * 32 + i4 * 8 + half * 4;
                        u32x2 w = {0u, 0u};
                        if (col < hd) {
                            if constexpr (E4M3) w = e4m3_to_bf16(*reinterpret_cast<const uint32_t*>(row + col), scale);
                            else w = *reinterpret_cast<const u32x2*>(row + col * 2);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float x = __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
                            if (key <= seen_to && !is_finite(x)) st.acc[db][4 * i4 + j] += x;
                        }
                    }
            }
        }
    }
    const bool whole = it.chunks == 1;
    const int64_t part_row0 = p.few_part_rows + ((int64_t)it.part + it.chunk) * kManyRows + wave * 32;
    if (half == 0 && exists) {
        const int64_t row = it.row_start + my_token;
        if (it.chunk == 0) p.where[row * p.q_heads + my_head] = where_entry(part_row0 + r, it.chunks, true);
        if (whole && p.lse) p.lse[(int64_t)my_head * p.rows.total_rows + row] = l_row == 0.f ? -INFINITY : (st.m * c + __log2f(l_row)) * kLn2;
    }
    char* const area = lds + wave * (32 * D * 4);
    if (!whole) {
        if (part_row0 + 32 > p.part_rows) return;
        if (half == 0) p.part_stats[part_row0 + r] = make_float2(st.m, l_row);
        store_tile_f32<D, false>(area, st.acc, 1.f, p.part_o + part_row0 * D, D, 32, D, lane_now);
        return;
    }
    // O leaves through LDS as in store_tile_bf16, but a row's address follows from its token and query head
    constexpr int kChunks = D / 8, kRowsPerInstr = 64 / kChunks;
    const float inv = l_row == 0.f ? 0.f : 1.f / l_row;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
            const int col = db * 32 + i4 * 8 + half * 4;
            u32x2 w;
            w[0] = pack_bf16(st.acc[db][4 * i4 + 0] * inv, st.acc[db][4 * i4 + 1] * inv);
            w[1] = pack_bf16(st.acc[db][4 * i4 + 2] * inv, st.acc[db][4 * i4 + 3] * inv);
            *reinterpret_cast<u32x2*>(area + (r * kChunks + ((col / 8) ^ (r & (kChunks - 1)))) * 16 + (col & 4) * 2) = w;
        }
    const int chunk = lane_now % kChunks;
#pragma unroll
    for (int i = 0; i < 32 / kRowsPerInstr; ++i) {
        const int row = i * kRowsPerInstr + lane_now / kChunks, x = wave_row0 + row, t = x / p.group;
        if (t < it.n && chunk * 8 < hd)
            *reinterpret_cast<u32x4*>(p.o + ((int64_t)(it.row_start + t) * p.q_heads + it.head * p.group + x % p.group) * hd + chunk * 8) =
                *reinterpret_cast<const u32x4*>(area + (row * kChunks + (chunk ^ (row & (kChunks - 1)))) * 16);
    }
}

template <int D, int KD>
void launch_many(const PagedAttnParams& p, int64_t grid, bool e4m3, hipStream_t stream) {
    if (e4m3) hipLaunchKernelGGL((paged_many_kernel<D, KD, true>), dim3((unsigned)grid), dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((paged_many_kernel<D, KD, false>), dim3((unsigned)grid), dim3(kThreads), 0, stream, p);
}

}  // namespace

hipError_t launch_paged_many(const PagedAttnParams& p, int64_t grid, bool e4m3, hipStream_t stream) {
    if (grid == 0) return hipSuccess;
    const int hd = p.pool.head_dim;
    if (tile_width(hd) == 64) launch_many<64, 4>(p, grid, e4m3, stream);
    else if (contraction_steps(hd) <= 5) launch_many<128, 5>(p, grid, e4m3, stream);
    else if (contraction_steps(hd) == 6) launch_many<128, 6>(p, grid, e4m3, stream);
    else if (contraction_steps(hd) == 7) launch_many<128, 7>(p, grid, e4m3, stream);
    else launch_many<128, 8>(p, grid, e4m3, stream);
    return hipGetLastError();
}

}  // namespace hspmd
