// Attention of new tokens over the paged cache: few rows per sequence and KV head (single tokens, short runs of them), and
// the join of chunks' results.
//
// With few rows the keys and values are read once and used for little arithmetic: the kernel is bound by reading the cache.  A workgroup is
// one wave: it takes 16 rows (tokens x query heads of one KV head) and a range of keys, which it copies page by page to LDS, tiles of 32
// keys, two ahead.  Single waves on their own keep a compute unit busiest: nothing waits at a barrier, and while one finds its work (lengths,
// page numbers, first tiles: three trips to memory, some 5 us) the others of the unit (4 of them with 16-bit values at D = 128, 8 otherwise)
// stream.  Products are transposed (keys, then head columns along the rows of the result; the 16 rows along its columns): a lane owns
// one row, the weights of a tile are the second product's operand as they stand, and V's operand comes from the row-major tile through
// the LDS transpose read.
//   S^T = K Q^T (16x16x32, 2 key blocks x D/32 steps),  P = exp2(c S - c m),  O^T += V^T P^T (D/16 blocks, one step of 32 keys)
// 8-bit tiles are copied as they are; K is scaled to bf16 on its way from LDS (exact), V's scales go into the weights
// (exact), its bytes are converted as they are.  Weights go into their product in two bf16 parts, their upper 8 bits and the rest rounded (15 bits or more together):
// the matrix cores have the time.  Rounded to one part they leave the result 1.1 to 1.3 times as far from the formula in 64 bits (1.88e-3 to 2.16e-3 of it against
// 1.61e-3 to 1.68e-3, all of which is O's own rounding), at 127 against 129 us for the 64 sequences below and the same time for the others (with the join).
// Scores, maxima, sums and O are fp32.
// One token of a sequence of 131001 keys, 32 heads on 8 of 128, bf16: 101 us = 5.3 TB/s (and 7 us for the join); of 64 sequences with 272960 keys together,
// e4m3: 118 us = 4.8 TB/s (5 us); of one with 1058, 5 heads: 6.3 us (4), start and three trips to memory.  Counters: HBM reads 1.00 and 1.06 times the
// cache's bytes (the scales' lines are fetched by several units), matrix cores a tenth busy.
#include "paged_item.hpp"

namespace hspmd {

namespace {

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// all but the newest N of this wave's loads and copies have landed
template <int N>
__device__ __forceinline__ void wait_copies_except() {
    static_assert(N >= 0 && N < 64, "vmcnt field");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

// Tile geometry in LDS: rows of D elements, 16-byte chunks XOR-swizzled so that neither the row-wise operand reads (16 rows, the same
// 16 or 8 bytes of each) nor the transpose reads (8 rows, the same 32 bytes of each) meet in a bank.  With C chunks per row, 16 / C rows
// fill the 64 banks once; the swizzle is the row's number in units of that, its low bits moved up by one.
template <int D, bool E4M3>
struct PagedTile {
    static constexpr int kKeys = 32;
    static constexpr int kRowBytes = D * (E4M3 ? 1 : 2);
    static constexpr int kBytes = kKeys * kRowBytes;
    static constexpr int kChunks = kRowBytes / 16;
    static constexpr int kBits = kChunks == 16 ? 4 : kChunks == 8 ? 3 : 2;
    static constexpr int kRowsPerCopy = 1024 / kRowBytes;
    static constexpr int kCopies = kBytes / 1024;
    static __device__ __forceinline__ int swizzle(int row) {
        const int j = row / (16 / kChunks);
        return ((j << 1) & (kChunks - 1)) | ((j >> (kBits - 1)) & 1);
    }
    static __device__ __forceinline__ int at(int row, int byte) { return row * kRowBytes + (((byte >> 4) ^ swizzle(row)) << 4) + (byte & 15); }
};

// the largest of the values that lanes l, l ^ 16, l ^ 32 and l ^ 48 hold
__device__ __forceinline__ float quads_max(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// whether a tile holds an infinity or NaN (a whole wave)
template <int D, bool E4M3>
__device__ __forceinline__ bool tile_not_finite(const char* tile, int lane) {
    uint32_t found = 0;
#pragma unroll
    for (int i = 0; i < PagedTile<D, E4M3>::kCopies; ++i) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(tile + i * 1024 + lane * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (E4M3) {
                // a byte of seven ones beside the sign carries into its top bit when 1 is added
                found |= ((x[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            } else {
                found |= ((x[j] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;   // an exponent of all ones
            }
        }
    }
    return __any(found != 0);
}

template <int D, bool E4M3>
struct FewGeom {
    using Tile = PagedTile<D, E4M3>;
    static constexpr int kStages = 2;     // K and V tiles: 32 KB for 16-bit values at D = 128
    static constexpr int kScaleBytes = E4M3 ? 256 : 0;
    static constexpr int kStageBytes = 2 * Tile::kBytes + kScaleBytes;
    static constexpr int kBytes = kStages * kStageBytes;
    static constexpr int kCopiesK = Tile::kCopies + (E4M3 ? 1 : 0);     // the scales travel with K
    static constexpr int kCopiesV = Tile::kCopies;
    static constexpr int kCopiesRun = 16 / Tile::kRowsPerCopy;           // per run of 16 keys: the least that a page holds, and the swizzle's period
};

constexpr int kWave = 64;
constexpr int kFewPages = 512;     // page numbers kept in LDS at a time (8192 keys of the smallest pages)

template <int D, bool E4M3>
__global__ __launch_bounds__(kWave) void paged_few_kernel(PagedAttnParams p) {
    using G = FewGeom<D, E4M3>;
    using Tile = typename G::Tile;
    constexpr int R = kFewRows, KS = D / 32, DB = D / 16, NST = G::kStages;
    __shared__ __attribute__((aligned(1024))) char lds[G::kBytes];
    __shared__ int pages[kFewPages];

    const PagedItem it = find_item<false>(p);
    if (it.seq < 0) return;
    const int lane = threadIdx.x, r16 = lane & 15, quad = lane >> 4;
    const int hd = p.pool.head_dim, shift = p.pool.page_shift, page_mask = (1 << shift) - 1;
    const float c = p.scale_log2;

    // this lane's row
    const int rho = it.tile * R + r16;
    const int token = rho / p.group, q_head = it.head * p.group + rho % p.group;
    const bool real = token < it.n;
    const int limit = real ? it.kv - it.n + token : -1;           // last key that the row sees
    const int first_token = it.tile * R / p.group, last_token = min(it.n - 1, (it.tile * R + R - 1) / p.group);
    const int tile_limit = it.kv - it.n + first_token;             // last key that every real row sees
    const int keys_end = max(0, it.kv - it.n + last_token + 1);
    const int64_t share = (int64_t)it.units * unit_keys(false);
    const int k0 = (int)min((int64_t)keys_end, it.chunk * share), k1 = (int)min((int64_t)keys_end, (it.chunk + 1) * share);

    bf16x8 qf[KS];
    const uint16_t* const q_row = p.q + (int64_t)(it.row_start + token) * p.q_stride + (int64_t)q_head * hd;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        union { u32x4 u; bf16x8 v; } t;
        t.u = u32x4{0u, 0u, 0u, 0u};
        if (real && ks * 32 + quad * 8 < hd) t.u = *reinterpret_cast<const u32x4*>(q_row + ks * 32 + quad * 8);
        qf[ks] = t.v;
    }
    f32x4 acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    const uint32_t lds_at = lds_address(lds);
    const int64_t head_at = (int64_t)it.head << shift;
    const int last_chunk = (hd * (E4M3 ? 1 : 2) + 15) / 16 - 1;
    uint32_t lane_at[G::kCopiesRun];               // this lane's 16 bytes of a run's copies
#pragma unroll
    for (int i = 0; i < G::kCopiesRun; ++i) {
        const int r = i * Tile::kRowsPerCopy + lane / Tile::kChunks;
        lane_at[i] = (uint32_t)(r * p.pool.row_bytes + min((lane % Tile::kChunks) ^ Tile::swizzle(r), last_chunk) * 16);
    }
    int bad_key = 0x7fffffff;                      // first key of the first page that does not exist

    for (int w0 = k0; w0 < k1;) {
        // the window's page numbers; one that does not exist is replaced by 0: what is read there is shown to nobody
        const int first_page = w0 >> shift;
        const int w1 = (int)min((int64_t)k1, ((int64_t)first_page + kFewPages) << shift);
        const int count = ((w1 - 1) >> shift) - first_page + 1;
        for (int i0 = 0; i0 < count; i0 += kWave) {
            const int i = i0 + lane, page = i < count ? page_at(p.pool, p.rows, it.seq, first_page + i) : 0;
            const uint64_t bad = __ballot(page < 0);
            if (bad) bad_key = min(bad_key, (first_page + i0 + (int)__builtin_ctzll(bad)) << shift);
            if (i < count) pages[i] = max(page, 0);
        }
        // the row has to be here before copies are under way that the compiler does not count: it would wait for them too, in every tile
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
        const int tiles = (w1 - w0 + Tile::kKeys - 1) / Tile::kKeys;

        // Where tile t's two runs of 16 keys lie (each within a page), as byte offsets into k and v and into the scales.  Keys behind the last:
        // what the page holds there, or the same run of the last page; never seen.
        struct Where {
            int64_t at[2], scale_at[2];
        };
        auto locate = [&](int t) {
            const int key0 = w0 + t * Tile::kKeys;
            const int numbers = pages[(min(key0 + 16 * (lane & 1), w1 - 1) >> shift) - first_page];
            Where w;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int64_t page = __builtin_amdgcn_readlane(numbers, half), row = head_at + ((key0 + 16 * half) & page_mask);
                w.at[half] = page * p.pool.page_bytes + row * p.pool.row_bytes;
                w.scale_at[half] = E4M3 ? page * p.pool.scale_page_bytes + row : 0;
            }
            return w;
        };
        auto copy = [&](const uint8_t* base, const Where& w, uint32_t dst) {
#pragma unroll
            for (int i = 0; i < Tile::kCopies; ++i) global_to_lds<16>(base + w.at[i / G::kCopiesRun], lane_at[i % G::kCopiesRun], dst + i * 1024);
        };
        auto copy_k = [&](int t, const Where& w) {
            const uint32_t dst = lds_at + (t % NST) * G::kStageBytes;
            copy(p.pool.k, w, dst);
            // lanes 0 .. 7: K's scales of four keys each, lanes 8 .. 15: V's, the others the same again
            if constexpr (E4M3)
                global_to_lds<4>((lane & 8 ? p.pool.v_scale : p.pool.k_scale) + (lane & 4 ? w.scale_at[1] : w.scale_at[0]) + (lane & 3) * 4,
                                 dst + 2 * Tile::kBytes);
        };
        auto copy_v = [&](int t, const Where& w) { copy(p.pool.v, w, lds_at + (t % NST) * G::kStageBytes + Tile::kBytes); };

        for (int t = 0; t < min(NST, tiles); ++t) {
            const Where w = locate(t);
            copy_k(t, w);
            copy_v(t, w);
        }
        for (int t = 0; t < tiles; ++t) {
            const int key0 = w0 + t * Tile::kKeys;
            const char* const kt = lds + (t % NST) * G::kStageBytes;
            const char* const vt = kt + Tile::kBytes;
            const bool more = t + NST < tiles;
            // NST - 1 further tiles are under way, or the last ones
            if (t + NST <= tiles) wait_copies_except<(NST - 1) * (G::kCopiesK + G::kCopiesV) + G::kCopiesV>();
            else wait_copies_except<0>();
            asm volatile("" ::: "memory");
            Where next{};
            if (more) next = locate(t + NST);
            f32x4 s[2];
#pragma unroll
            for (int mb = 0; mb < 2; ++mb) {
                const int row = mb * 16 + r16;
                s[mb] = f32x4{0.f, 0.f, 0.f, 0.f};
                float k_scale = 1.f;
                if constexpr (E4M3) k_scale = scale_of(*reinterpret_cast<const uint8_t*>(kt + 2 * Tile::kBytes + row));
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    bf16x8 a;
                    if constexpr (E4M3) {
                        const u32x2 w = *reinterpret_cast<const u32x2*>(kt + Tile::at(row, ks * 32 + quad * 8));
                        const u32x2 x = e4m3_to_bf16(w[0], k_scale), y = e4m3_to_bf16(w[1], k_scale);
                        union { u32x4 u; bf16x8 v; } t4;
                        t4.u = u32x4{x[0], x[1], y[0], y[1]};
                        a = t4.v;
                    } else {
                        a = *reinterpret_cast<const bf16x8*>(kt + Tile::at(row, (ks * 32 + quad * 8) * 2));
                    }
                    s[mb] = mfma16(a, qf[ks], s[mb]);
                }
            }
            uint32_t v_scales[2] = {0u, 0u};
            if constexpr (E4M3) {
#pragma unroll
                for (int mb = 0; mb < 2; ++mb) v_scales[mb] = *reinterpret_cast<const uint32_t*>(kt + 2 * Tile::kBytes + 32 + mb * 16 + quad * 4);
            }
            // K's buffer is free once its reads have returned
            __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
            asm volatile("" : "+v"(v_scales[0]), "+v"(v_scales[1]) :: "memory");
            if (more) copy_k(t + NST, next);
            // element i of block mb: key key0 + 16 mb + 4 quad + i
            const bool masked = key0 + Tile::kKeys - 1 > min(tile_limit, w1 - 1);
            const int seen = min(limit, w1 - 1) - key0 - 4 * quad;
            if (masked) {
#pragma unroll
                for (int mb = 0; mb < 2; ++mb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (16 * mb + i > seen) s[mb][i] = -INFINITY;
            }
            float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            top = quads_max(top);
            const float m_new = fmaxf(m, top);
            const float m_ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = fast_exp2((m - m_ref) * c), mc = m_ref * c;
            m = m_new;
            float sum = 0.f;
            union { u32x4 u; bf16x8 v; } w, rest;      // the weights cut to bf16, and what is left of them
#pragma unroll
            for (int mb = 0; mb < 2; ++mb) {
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[i] = fast_exp2(fmaf(s[mb][i], c, -mc));
                    sum += e[i];
                    // (a scale behind the last key is whatever the page holds)
                    if constexpr (E4M3) {
                        e[i] *= scale_of((v_scales[mb] >> (8 * i)) & 0xffu);
                        if (masked) e[i] = 16 * mb + i > seen ? 0.f : e[i];
                    }
                }
                // (the upper halves of two words.  What is left is positive for every weight above 2^-102: 2^-24 of the weight is added, so that a value which
                // is infinite stays so in both products)
                w.u[2 * mb] = __builtin_amdgcn_perm(__float_as_uint(e[1]), __float_as_uint(e[0]), 0x07060302u);
                w.u[2 * mb + 1] = __builtin_amdgcn_perm(__float_as_uint(e[3]), __float_as_uint(e[2]), 0x07060302u);
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = fmaf(e[i], 0x1p-24f, e[i] - __uint_as_float(__float_as_uint(e[i]) & 0xffff0000u));
                rest.u[2 * mb] = pack_bf16(e[0], e[1]);
                rest.u[2 * mb + 1] = pack_bf16(e[2], e[3]);
            }
            l = l * alpha + sum;
            if (__any(alpha != 1.f)) {
#pragma unroll
                for (int i = 0; i < DB; ++i) acc[i] *= alpha;
            }
            if (more) wait_copies_except<(NST - 1) * (G::kCopiesK + G::kCopiesV) + G::kCopiesK>();
            else if (t + NST <= tiles) wait_copies_except<(NST - 1) * (G::kCopiesK + G::kCopiesV)>();
            asm volatile("" ::: "memory");
            const int v_row = quad * 4 + (r16 >> 2), v_byte = (r16 & 3) * 8;
            auto add_values = [&](f32x4 (&sum_of)[DB]) {
                if constexpr (E4M3) {
#pragma unroll
                    for (int cb = 0; cb < D / 32; ++cb) {
                        // two columns at a time as 16-bit elements: result row x of the first product is column 32 cb + 2 x, of the second 32 cb + 2 x + 1
                        union { s16x4 s; u32x2 u; } a, b;
                        a.s = lds_transpose_read(vt + Tile::at(v_row, cb * 32 + v_byte));
                        b.s = lds_transpose_read(vt + Tile::at(v_row + 16, cb * 32 + v_byte));
#pragma unroll
                        for (int odd = 0; odd < 2; ++odd) {
                            const uint32_t pick = odd ? 0x07050301u : 0x06040200u;
                            const u32x2 x = e4m3_to_bf16(__builtin_amdgcn_perm(a.u[1], a.u[0], pick), 1.f);
                            const u32x2 y = e4m3_to_bf16(__builtin_amdgcn_perm(b.u[1], b.u[0], pick), 1.f);
                            union { u32x4 u; bf16x8 v; } t4;
                            t4.u = u32x4{x[0], x[1], y[0], y[1]};
                            sum_of[2 * cb + odd] = mfma16(t4.v, rest.v, mfma16(t4.v, w.v, sum_of[2 * cb + odd]));
                        }
                    }
                } else {
#pragma unroll
                    for (int db = 0; db < DB; ++db) {
                        union { struct { s16x4 a, b; } s; bf16x8 v; } u;
                        u.s.a = lds_transpose_read(vt + Tile::at(v_row, db * 32 + v_byte));
                        u.s.b = lds_transpose_read(vt + Tile::at(v_row + 16, db * 32 + v_byte));
                        sum_of[db] = mfma16(u.v, rest.v, mfma16(u.v, w.v, sum_of[db]));
                    }
                }
            };
            // A weight of 0 hides a value only if the value is finite.  Where some row does not see all of a tile and one of its values is not,
            // the tokens take their products one by one, the last first, with the keys behind each set to zero.
            if (masked && tile_not_finite<D, E4M3>(vt, lane)) {
                char* const zeroed = lds + (vt - lds);
                for (int tk = last_token; tk >= first_token; --tk) {
                    for (int r = max(it.kv - it.n + tk + 1 - key0, 0); r < Tile::kKeys; ++r)
                        if (lane < Tile::kChunks) *reinterpret_cast<u32x4*>(zeroed + r * Tile::kRowBytes + lane * 16) = u32x4{0u, 0u, 0u, 0u};
                    f32x4 one[DB];
#pragma unroll
                    for (int i = 0; i < DB; ++i) one[i] = acc[i];
                    add_values(one);
#pragma unroll
                    for (int i = 0; i < DB; ++i)
                        if (token == tk) acc[i] = one[i];
                }
            } else {
                add_values(acc);
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): V's buffer is free as well
            asm volatile("" ::: "memory");
            if (more) copy_v(t + NST, next);
        }
        w0 = w1;
    }

    // ---- results: the lanes of a row hold a quarter of its weights' sum each
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (!real) return;
    if (limit >= bad_key) l = __builtin_nanf("");
    const int64_t row = it.row_start + token, part_row = ((int64_t)it.part + it.chunk) * R + r16;
    const bool whole = it.chunks == 1;
    if (!whole && part_row >= p.few_part_rows) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;            // no key: O = 0; a bad page: NaN
    auto store4 = [&](int col, float a, float b, float d, float e) {
        if (!whole) *reinterpret_cast<f32x4*>(p.part_o + part_row * D + col) = f32x4{a, b, d, e};
        else if (col < hd) *reinterpret_cast<u32x2*>(p.o + (row * p.q_heads + q_head) * hd + col) = u32x2{pack_bf16(a * inv, b * inv), pack_bf16(d * inv, e * inv)};
    };
    if constexpr (E4M3) {
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
            for (int i = 0; i < 4; i += 2) store4(cb * 32 + quad * 8 + 2 * i, acc[2 * cb][i], acc[2 * cb + 1][i], acc[2 * cb][i + 1], acc[2 * cb + 1][i + 1]);
    } else {
#pragma unroll
        for (int db = 0; db < DB; ++db) store4(db * 16 + quad * 4, acc[db][0], acc[db][1], acc[db][2], acc[db][3]);
    }
    if (quad == 0) {
        if (!whole) p.part_stats[part_row] = make_float2(m, l);
        else if (p.lse) p.lse[(int64_t)q_head * p.rows.total_rows + row] = l == 0.f ? -INFINITY : (m * c + __log2f(l)) * kLn2;
        if (it.chunk == 0) p.where[row * p.q_heads + q_head] = where_entry(part_row, it.chunks, false);
    }
}

// ---- the plan: a workgroup for each kernel that runs (find_item's sums with the sequences dealt out to 1024 threads)
constexpr int kPlanThreads = 1024;

struct UpTo {
    uint32_t mine, all;
};
// sums over the workgroup's threads up to each one, and over all; sums: LDS, one per wave
__device__ __forceinline__ UpTo threads_up_to(uint32_t x, uint32_t* sums) {
    const int wave = threadIdx.x >> 6;
    UpTo r{lanes_up_to(x), 0u};
    __syncthreads();                                       // the previous call's sums have been read
    if ((threadIdx.x & 63) == 63) sums[wave] = r.mine;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        r.mine += w < wave ? sums[w] : 0u;
        r.all += sums[w];
    }
    return r;
}

template <bool MANY>
__device__ __forceinline__ void make_plan(const PagedAttnParams& p, uint32_t* plan, uint32_t* sums) {
    const int n = p.rows.num_seqs, kvh = p.pool.kv_heads;
    SeqRows s{};
    SeqTiles t{};
    int64_t units = 0;
    for (int seq = threadIdx.x; seq < n; seq += kPlanThreads) {
        look_at<MANY>(p, seq, s, t);
        units += (int64_t)t.tiles * t.units * kvh;
    }
    const int64_t high = threads_up_to((uint32_t)(units >> 20), sums).all, low = threads_up_to((uint32_t)units & 0xfffffu, sums).all;
    const int first_per = units_per_chunk((high << 20) + low, MANY);
    int per_chunk = first_per;
    for (int raise = 0; raise < kRaises; ++raise) {
        uint32_t slots = 0;
        for (int seq = threadIdx.x; seq < n; seq += kPlanThreads) {
            look_at<MANY>(p, seq, s, t);
            slots += (uint32_t)(t.tiles * kvh * shares_of(t.units, per_chunk).chunks);
        }
        const int next = raised(per_chunk, first_per, threads_up_to(slots, sums).all, MANY);
        if (next == per_chunk) break;
        per_chunk = next;
    }
    uint32_t slots = 0, parts = 0;                         // of the sequences before
    for (int seq0 = 0; seq0 < n; seq0 += kPlanThreads) {
        const int seq = seq0 + threadIdx.x;
        look_at<MANY>(p, seq, s, t);
        const Shares sh = shares_of(t.units, per_chunk);
        const uint32_t mine = t.tiles * kvh * sh.chunks, mine_parts = sh.chunks > 1 ? mine : 0u;
        const UpTo a = threads_up_to(mine, sums), b = threads_up_to(mine_parts, sums);
        if (seq < n) {
            plan[1 + seq] = slots + a.mine - mine;
            plan[2 + n + seq] = parts + b.mine - mine_parts;
        }
        slots += a.all;
        parts += b.all;
    }
    if (threadIdx.x == 0) {
        plan[0] = per_chunk;
        plan[1 + n] = slots;
    }
}

__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(PagedAttnParams p, uint32_t* plan, int first) {
    __shared__ uint32_t sums[kPlanThreads / 64];
    if (first + (int)blockIdx.x == 0) make_plan<false>(p, plan, sums);
    else make_plan<true>(p, plan + plan_words(p.rows.num_seqs), sums);
}

// ---- chunks' results joined, for the (row, query head) pairs that have several
//   M = max m_i,  L = sum exp2(c (m_i - M)) l_i,  O = sum exp2(c (m_i - M)) o_i / L
// Sums, weights and the maximum are carried along the chunks together, so that nothing is read twice and nothing waits for a maximum; the order of a
// sum depends on the number of chunks alone.
struct Joined {
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, total = 0.f;
    __device__ __forceinline__ void add(float2 st, f32x4 x, float c) {
        const float m = fmaxf(top, st.x), ref = m == -INFINITY ? 0.f : m;
        const float keep = fast_exp2((top - ref) * c), f = fast_exp2((st.x - ref) * c);
        total = total * keep + f * st.y;
        sum = sum * keep + f * x;
        top = m;
    }
};

// A pair's entry; no chunks where there is nothing to join: the result is in o already, or the row belongs to no sequence (no entry then)
struct Pair {
    int first, chunks, stride;
};
__device__ __forceinline__ Pair pair_at(const PagedAttnParams& p, int64_t unit) {
    const int2 w = p.where[unit];
    const int64_t begin = (int64_t)max(p.rows.cu_rows[0], 0) * p.q_heads, end = (int64_t)p.rows.cu_rows[p.rows.num_seqs] * p.q_heads;
    Pair r{w.x, w.y & 0x3fffffff, w.y >> 30 & 1 ? kManyRows : kFewRows};
    if (unit < begin || unit >= end || r.chunks <= 1 || r.first < 0 || (int64_t)r.first + (int64_t)(r.chunks - 1) * r.stride >= p.part_rows) r.chunks = 0;
    return r;
}

// chunks from, from + step, ... of a pair, four of them read at a time; columns col .. col + 3
template <int D>
__device__ __forceinline__ Joined gather(const PagedAttnParams& p, const Pair& pair, int from, int step, int col) {
    constexpr int kAtOnce = 4;
    Joined r;
    for (int j = from; j < pair.chunks; j += step * kAtOnce) {
        float2 st[kAtOnce];
        f32x4 x[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int64_t at = pair.first + (int64_t)min(j + i * step, pair.chunks - 1) * pair.stride;
            st[i] = p.part_stats[at];
            x[i] = *reinterpret_cast<const f32x4*>(p.part_o + at * D + col);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
            if (j + i * step < pair.chunks) r.add(st[i], x[i], p.scale_log2);
    }
    return r;
}

__device__ __forceinline__ void put(const PagedAttnParams& p, const Joined& r, int64_t unit, int col) {
    const float inv = r.total == 0.f ? 0.f : 1.f / r.total;
    if (col < p.pool.head_dim)
        *reinterpret_cast<u32x2*>(p.o + unit * p.pool.head_dim + col) = u32x2{pack_bf16(r.sum[0] * inv, r.sum[1] * inv), pack_bf16(r.sum[2] * inv, r.sum[3] * inv)};
    if (col == 0 && p.lse)
        p.lse[unit % p.q_heads * p.rows.total_rows + unit / p.q_heads] = r.total == 0.f ? -INFINITY : (r.top * p.scale_log2 + __log2f(r.total)) * kLn2;
}

// Many pairs: a wave looks at `per_wave` of them at once, one per lane, and joins those that have something to join, a team of D / 4 lanes each, their
// chunks one after the other.  Bound by latency.
template <int D>
__global__ __launch_bounds__(kThreads, 8) void paged_join_kernel(PagedAttnParams p, int per_wave) {
    constexpr int kLanes = D / 4, kTeams = 64 / kLanes;
    const int lane = threadIdx.x & 63, team = lane / kLanes, col = lane % kLanes * 4;
    const int64_t units = (int64_t)p.rows.total_rows * p.q_heads, first = ((int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * per_wave;
    Pair mine{0, 0, 0};
    if (lane < per_wave && first + lane < units) mine = pair_at(p, first + lane);
    for (uint64_t left = __ballot(mine.chunks != 0); left;) {
        int at = -1;                                       // the team's: the first, second, ... of those left
#pragma unroll
        for (int t = 0; t < kTeams; ++t) {
            if (t == team && left) at = __builtin_ctzll(left);
            left &= left - 1;
        }
        const int from = max(at, 0);
        const Pair pair{__shfl(mine.first, from, 64), __shfl(mine.chunks, from, 64), __shfl(mine.stride, from, 64)};
        if (at >= 0) put(p, gather<D>(p, pair, 0, 1, col), first + at, col);
    }
}

// Few pairs, of many chunks perhaps: a workgroup for COLUMNS columns of one, the chunks dealt out to its teams.
template <int D, int COLUMNS>
__global__ __launch_bounds__(kThreads) void paged_join_pair_kernel(PagedAttnParams p) {
    constexpr int kLanes = COLUMNS / 4, kTeams = kThreads / kLanes;
    __shared__ f32x4 sums[kTeams][kLanes];
    __shared__ float2 stats[kTeams];
    const int lane = threadIdx.x % kLanes, team = threadIdx.x / kLanes, col = blockIdx.y * COLUMNS + lane * 4;
    const Pair pair = pair_at(p, blockIdx.x);
    if (pair.chunks == 0) return;
    Joined r = gather<D>(p, pair, team, kTeams, col);
    sums[team][lane] = r.sum;
    if (lane == 0) stats[team] = make_float2(r.top, r.total);
    __syncthreads();
    if (team) return;
    for (int g = 1; g < min(kTeams, pair.chunks); ++g) r.add(stats[g], sums[g][lane], p.scale_log2);
    put(p, r, blockIdx.x, col);
}

template <int D, bool E4M3>
void launch_few(const PagedAttnParams& p, const PagedSizes& sizes, hipStream_t stream) {
    hipLaunchKernelGGL((paged_few_kernel<D, E4M3>), dim3((unsigned)sizes.few_grid), dim3(kWave), 0, stream, p);
}

}  // namespace

// Which kernel takes a sequence.  With up to 16 rows per KV head the kernel for few rows reads the keys once; the one for many takes 128 rows
// in about the time that 16 take there, so two tiles of the former are already no faster.
PagedSizes paged_sizes(const PagedRows& rows, int max_rows, int page_shift, int q_heads, int kv_heads, int head_dim) {
    const int64_t group = q_heads / kv_heads, D = tile_width(head_dim);
    const int64_t most = (max_rows > 0 ? std::min(max_rows, rows.total_rows) : rows.total_rows) * group;
    PagedSizes s{};
    s.few = most <= kFewRows || rows.num_seqs > 1;
    s.many = most > kFewRows;
    // (one kernel alone takes every sequence, so that a wrong max_rows costs time and nothing else)
    s.join = ((int64_t)rows.table_width << page_shift) > unit_keys(false);       // (a single unit is not shared out)
    s.few_limit = !s.many ? 0x7fffffff : s.few ? kFewRows : 0;
    auto bounds = [&](bool many, int few_limit) {
        return grid_bounds(rows.total_rows, rows.num_seqs, rows.table_width, page_shift, group, kv_heads, many, few_limit);
    };
    s.few_grid = bounds(false, s.few_limit).grid;
    s.many_grid = bounds(true, s.few_limit).grid;
    // room for either choice: the size does not depend on the hint
    s.few_part_rows = bounds(false, 0x7fffffff).part_tiles * kFewRows;
    s.part_rows = s.few_part_rows + (rows.total_rows * group > kFewRows ? bounds(true, 0).part_tiles * kManyRows : 0);
    s.where_bytes = ((size_t)rows.total_rows * q_heads * sizeof(int2) + 255) / 256 * 256;
    s.stats_bytes = ((size_t)s.part_rows * sizeof(float2) + 255) / 256 * 256;
    s.part_bytes = (size_t)s.part_rows * D * sizeof(float);
    s.plan_bytes = rows.num_seqs > kPlanAbove ? 2 * (size_t)plan_words(rows.num_seqs) * sizeof(uint32_t) : 0;
    return s;
}

hipError_t launch_paged_attn(const PagedAttnParams& p, const PagedSizes& sizes, bool e4m3, hipStream_t stream) {
    const int width = tile_width(p.pool.head_dim);
    if (p.plan) {
        hipLaunchKernelGGL(paged_plan_kernel, dim3(sizes.few + sizes.many), dim3(kPlanThreads), 0, stream, p, const_cast<uint32_t*>(p.plan), sizes.few ? 0 : 1);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (sizes.few) {
        if (width == 128) {
            if (e4m3) launch_few<128, true>(p, sizes, stream);
            else launch_few<128, false>(p, sizes, stream);
        } else {
            if (e4m3) launch_few<64, true>(p, sizes, stream);
            else launch_few<64, false>(p, sizes, stream);
        }
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (sizes.many) {
        if (const hipError_t e = launch_paged_many(p, sizes.many_grid, e4m3, stream)) return e;
    }
    if (!sizes.join) return hipSuccess;
    // Chosen by the pairs of the call and the width of the table: the host does not know how many chunks a pair has.  (A few pairs of very many chunks in a large call wait for
    // one team's walk over them: a token over 131001 keys, 32 heads, 110 us by itself, 172 in a batch padded to 256 rows.)
    // up to 4096 pairs: a workgroup each (64 rows of 32 heads, 5 to 30 chunks 7 us); long contexts: several, 32 columns each (one row of 32
    // heads, 256 chunks 10 -> 7 us, but 5 heads of 34 chunks 3.7 -> 4.9); more: teams (22784 pairs of 2 or 3 chunks 11 us,
    // 19 us with a workgroup for 6), and as many pairs per wave as keep 8192 waves busy (131072 with nothing to join 4.7 us, 12.4 with one per team)
    const int64_t pairs = (int64_t)p.rows.total_rows * p.q_heads;
    const dim3 threads(kThreads);
    if (pairs > 4096) {
        const int teams = 64 / (width / 4), per_wave = (int)std::max<int64_t>(teams, std::min<int64_t>(64, pairs / 8192)), per_group = per_wave * (kThreads / 64);
        const dim3 grid((unsigned)((pairs + per_group - 1) / per_group));
        if (width == 128) hipLaunchKernelGGL(paged_join_kernel<128>, grid, threads, 0, stream, p, per_wave);
        else hipLaunchKernelGGL(paged_join_kernel<64>, grid, threads, 0, stream, p, per_wave);
    } else if (pairs <= 256 && ((int64_t)p.rows.table_width << p.pool.page_shift) >= 128 * unit_keys(false)) {
        const dim3 grid((unsigned)pairs, width / 32);
        if (width == 128) hipLaunchKernelGGL((paged_join_pair_kernel<128, 32>), grid, threads, 0, stream, p);
        else hipLaunchKernelGGL((paged_join_pair_kernel<64, 32>), grid, threads, 0, stream, p);
    } else {
        if (width == 128) hipLaunchKernelGGL((paged_join_pair_kernel<128, 128>), dim3((unsigned)pairs), threads, 0, stream, p);
        else hipLaunchKernelGGL((paged_join_pair_kernel<64, 64>), dim3((unsigned)pairs), threads, 0, stream, p);
    }
    return hipGetLastError();
}

}  // namespace hspmd
