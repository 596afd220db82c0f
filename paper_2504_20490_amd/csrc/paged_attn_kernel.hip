// Attention of new tokens over the paged cache: few rows per sequence and KV head (single tokens, short runs of them), and
// the join of chunks' results.
//
// With few rows the keys and values are read once and used for little arithmetic: the kernel is bound by reading the cache.  A
// workgroup takes 16 rows (tokens x query heads of one KV head) and a range of keys; its four waves take 32-key tiles in turn, each wave with
// LDS buffers of its own into which it copies pages directly, several tiles ahead, so that no wave waits for another and a compute
// unit has tens of KB under way.  Products are transposed (keys, then head columns along the rows of the result; the 16 rows along its
// columns): a lane owns one row, the weights of a tile are the second product's operand as they stand, and V's operand comes from the
// row-major tile through the LDS transpose read.
//   S^T = K Q^T (16x16x32, 2 key blocks x D/32 steps),  P = exp2(c S - c m),  O^T += V^T P^T (D/16 blocks, one step of 32 keys)
// 8-bit tiles are copied as they are; K is scaled to bf16 on its way from LDS (exact), V's scales go into the weights
// before they are rounded, its bytes are converted as they are.
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
    // K and V tiles per wave: 32 KB for 16-bit values at D = 128, 16 KB otherwise
    static constexpr int kStages = D == 128 && !E4M3 ? 2 : 4;
    static constexpr int kScaleBytes = E4M3 ? 256 : 0;
    static constexpr int kStageBytes = 2 * Tile::kBytes + kScaleBytes;
    static constexpr int kWaveBytes = kStages * kStageBytes;
    static constexpr int kCopiesK = Tile::kCopies + (E4M3 ? 1 : 0);     // the scales travel with K
    static constexpr int kCopiesV = Tile::kCopies;
};

template <int D, bool E4M3>
__global__ __launch_bounds__(kThreads) void paged_few_kernel(PagedAttnParams p) {
    using G = FewGeom<D, E4M3>;
    using Tile = typename G::Tile;
    constexpr int R = kFewRows, KS = D / 32, DB = D / 16, NST = G::kStages;
    static_assert(4 * R * D * 4 <= 4 * G::kWaveBytes, "the waves' sums fit where their tiles were");
    __shared__ __attribute__((aligned(1024))) char lds[4 * G::kWaveBytes];
    __shared__ int pages[kWindowPages + 1];
    __shared__ float2 stats[4][R];
    __shared__ int bad_key;                      // first key of the first page that does not exist

    const PagedItem it = find_item<false>(p);
    if (it.seq < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, quad = lane >> 4;
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
    const int64_t unit_keys = (int64_t)it.units * kUnitKeys;
    const int k0 = (int)min((int64_t)keys_end, it.chunk * unit_keys), k1 = (int)min((int64_t)keys_end, (it.chunk + 1) * unit_keys);

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

    char* const mine = lds + wave * G::kWaveBytes;
    const uint32_t mine_at = lds_address(lds) + wave * G::kWaveBytes;
    const int64_t head_at = (int64_t)it.head << shift;
    const int last_chunk = (hd * (E4M3 ? 1 : 2) + 15) / 16 - 1;
    if (threadIdx.x == 0) bad_key = 0x7fffffff;

    for (int w0 = k0; w0 < k1;) {
        // the window's page numbers
        const int first_page = w0 >> shift;
        const int w1 = (int)min((int64_t)k1, ((int64_t)first_page + kWindowPages) << shift);
        __syncthreads();
        load_pages(p, it.seq, first_page, ((w1 - 1) >> shift) - first_page + 1, pages, &bad_key);
        // the row has to be here before copies are under way that the compiler does not count: it would wait for them too, in every tile
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
        __syncthreads();
        const int tiles = (w1 - w0 + Tile::kKeys - 1) / Tile::kKeys;
        const int my_tiles = (tiles - wave + 3) / 4;

        auto issue = [&](int t) {
            const int key0 = w0 + (t * 4 + wave) * Tile::kKeys;
            const uint32_t dst = mine_at + (t % NST) * G::kStageBytes;
            int64_t off[Tile::kCopies];
#pragma unroll
            for (int i = 0; i < Tile::kCopies; ++i) {
                const int r = i * Tile::kRowsPerCopy + lane / Tile::kChunks;
                const int key = min(key0 + r, w1 - 1);               // (rows past the end repeat the last key: weight 0, finite)
                const int chunk = min((lane % Tile::kChunks) ^ Tile::swizzle(r), last_chunk);
                off[i] = pages[(key >> shift) - first_page] * p.pool.page_bytes + (head_at + (key & page_mask)) * p.pool.row_bytes + chunk * 16;
            }
#pragma unroll
            for (int i = 0; i < Tile::kCopies; ++i) global_to_lds<16>(p.pool.k + off[i], dst + i * 1024);
            if constexpr (E4M3) {
                // lanes 0 .. 7: K's scales of four keys each, lanes 8 .. 15: V's, the others the same again
                const int key = min(key0 + (lane & 7) * 4, (w1 - 1) & ~3);
                const int64_t at = pages[(key >> shift) - first_page] * p.pool.scale_page_bytes + head_at + (key & page_mask);
                global_to_lds<4>((lane & 8 ? p.pool.v_scale : p.pool.k_scale) + at, dst + 2 * Tile::kBytes);
            }
#pragma unroll
            for (int i = 0; i < Tile::kCopies; ++i) global_to_lds<16>(p.pool.v + off[i], dst + Tile::kBytes + i * 1024);
        };

        const int ahead = min(NST, my_tiles);
        for (int t = 0; t < ahead; ++t) issue(t);
        for (int t = 0; t < my_tiles; ++t) {
            const int key0 = w0 + (t * 4 + wave) * Tile::kKeys;
            const char* const kt = mine + (t % NST) * G::kStageBytes;
            const char* const vt = kt + Tile::kBytes;
            const bool steady = t + NST <= my_tiles;                  // NST - 1 further tiles are under way
            if (steady) wait_copies_except<(NST - 1) * (G::kCopiesK + G::kCopiesV) + G::kCopiesV>();
            else wait_copies_except<0>();
            asm volatile("" ::: "memory");
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
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float m_new = fmaxf(m, top);
            const float m_ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = fast_exp2((m - m_ref) * c), mc = m_ref * c;
            m = m_new;
            uint32_t v_scales[2] = {0u, 0u};
            if constexpr (E4M3) {
#pragma unroll
                for (int mb = 0; mb < 2; ++mb) v_scales[mb] = *reinterpret_cast<const uint32_t*>(kt + 2 * Tile::kBytes + 32 + mb * 16 + quad * 4);
            }
            float sum = 0.f;
            union { u32x4 u; bf16x8 v; } w;
#pragma unroll
            for (int mb = 0; mb < 2; ++mb) {
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[i] = fast_exp2(fmaf(s[mb][i], c, -mc));
                    sum += e[i];
                    // (a scale behind the last key is whatever the page holds)
                    if constexpr (E4M3) e[i] = masked && 16 * mb + i > seen ? 0.f : e[i] * scale_of((v_scales[mb] >> (8 * i)) & 0xffu);
                }
                w.u[2 * mb] = pack_bf16(e[0], e[1]);
                w.u[2 * mb + 1] = pack_bf16(e[2], e[3]);
            }
            l = l * alpha + sum;
            if (__any(alpha != 1.f)) {
#pragma unroll
                for (int i = 0; i < DB; ++i) acc[i] *= alpha;
            }
            if (steady) wait_copies_except<(NST - 1) * (G::kCopiesK + G::kCopiesV)>();
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
                            sum_of[2 * cb + odd] = mfma16(t4.v, w.v, sum_of[2 * cb + odd]);
                        }
                    }
                } else {
#pragma unroll
                    for (int db = 0; db < DB; ++db) {
                        union { struct { s16x4 a, b; } s; bf16x8 v; } u;
                        u.s.a = lds_transpose_read(vt + Tile::at(v_row, db * 32 + v_byte));
                        u.s.b = lds_transpose_read(vt + Tile::at(v_row + 16, db * 32 + v_byte));
                        sum_of[db] = mfma16(u.v, w.v, sum_of[db]);
                    }
                }
            };
            // A weight of 0 hides a value only if the value is finite.  Where rows of several tokens share a masked tile and one of its
            // values is not, the tokens take their products one by one, the last first, with the keys behind each set to zero.
            if (masked && first_token < last_token && tile_not_finite<D, E4M3>(vt, lane)) {
                char* const zeroed = mine + (vt - mine);
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
            // the tile's buffers are free once its reads have returned
            __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
            asm volatile("" ::: "memory");
            if (t + NST < my_tiles) issue(t + NST);
        }
        w0 = w1;
    }

    // ---- the four waves' shares meet in LDS
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    __syncthreads();                               // (every copy has been waited for by the wave that issued it)
    if (quad == 0) {
        if (limit >= bad_key) l = __builtin_nanf("");
        stats[wave][r16] = make_float2(m, l);
    }
    float* const sums = reinterpret_cast<float*>(lds) + wave * R * D;
    if constexpr (E4M3) {
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
            for (int i = 0; i < 4; i += 2)
                *reinterpret_cast<f32x4*>(sums + r16 * D + cb * 32 + quad * 8 + 2 * i) =
                    f32x4{acc[2 * cb][i], acc[2 * cb + 1][i], acc[2 * cb][i + 1], acc[2 * cb + 1][i + 1]};
    } else {
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(sums + r16 * D + db * 16 + quad * 4) = acc[db];
    }
    __syncthreads();
    const bool whole = it.chunks == 1;
    for (int e = threadIdx.x; e < R * (D / 4); e += kThreads) {
        const int r = e / (D / 4), col = e % (D / 4) * 4;
        const int rr = it.tile * R + r, tk = rr / p.group, hq = it.head * p.group + rr % p.group;
        if (tk >= it.n) continue;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, stats[w][r].x);
        const float ref = top == -INFINITY ? 0.f : top;
        float total = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 st = stats[w][r];
            const float f = fast_exp2((st.x - ref) * c);
            total += f * st.y;
            o += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(lds) + (w * R + r) * D + col);
        }
        const int64_t row = it.row_start + tk;
        if (whole) {
            const float inv = total == 0.f ? 0.f : 1.f / total;       // no key: O = 0; a bad page: NaN
            if (col < hd) {
                u32x2 x;
                x[0] = pack_bf16(o[0] * inv, o[1] * inv);
                x[1] = pack_bf16(o[2] * inv, o[3] * inv);
                *reinterpret_cast<u32x2*>(p.o + (row * p.q_heads + hq) * hd + col) = x;
            }
            if (col == 0 && p.lse) p.lse[(int64_t)hq * p.rows.total_rows + row] = total == 0.f ? -INFINITY : (top * c + __log2f(total)) * kLn2;
        }
        const int64_t part_row = ((int64_t)it.part + it.chunk) * R + r;
        if (!whole && part_row < p.few_part_rows) {
            *reinterpret_cast<f32x4*>(p.part_o + part_row * D + col) = o;
            if (col == 0) p.part_stats[part_row] = make_float2(top, total);
        }
        if (col == 0 && it.chunk == 0) p.where[row * p.q_heads + hq] = where_entry(part_row, it.chunks, false);
    }
}

// Chunks' results of a row joined: a wave per (row, query head).
//   M = max m_i, L = sum exp2(c (m_i - M)) l_i, O = sum exp2(c (m_i - M)) o_i / L
template <int D>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(PagedAttnParams p) {
    constexpr int kPer = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= (int64_t)p.rows.total_rows * p.q_heads) return;
    const int row = (int)(unit / p.q_heads), head = (int)(unit % p.q_heads);
    if (sequence_of(p.rows, row) < 0) return;
    const int2 at = p.where[unit];
    const bool many = at.y >> 30 & 1;
    const int chunks = at.y & 0x3fffffff, tile_rows = many ? kManyRows : kFewRows;
    if (chunks <= 1 || at.x < 0 || (int64_t)at.x + (int64_t)(chunks - 1) * tile_rows >= p.part_rows) return;
    const float c = p.scale_log2;
    float top = -INFINITY;
    for (int i = lane; i < chunks; i += 64) top = fmaxf(top, p.part_stats[at.x + i * tile_rows].x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float ref = top == -INFINITY ? 0.f : top;
    float total = 0.f, o[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) o[j] = 0.f;
    for (int i = 0; i < chunks; ++i) {
        const int64_t r = at.x + (int64_t)i * tile_rows;
        const float2 st = p.part_stats[r];
        const float f = fast_exp2((st.x - ref) * c);
        total += f * st.y;
#pragma unroll
        for (int j = 0; j < kPer; ++j) o[j] += f * p.part_o[r * D + lane * kPer + j];
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const int hd = p.pool.head_dim;
    uint16_t* const dst = p.o + unit * hd;
    if (lane * kPer < hd) {
        if constexpr (kPer == 2) *reinterpret_cast<uint32_t*>(dst + lane * 2) = pack_bf16(o[0] * inv, o[1] * inv);
        else dst[lane] = (uint16_t)pack_bf16(o[0] * inv, 0.f);
    }
    if (lane == 0 && p.lse) p.lse[(int64_t)head * p.rows.total_rows + row] = total == 0.f ? -INFINITY : (top * c + __log2f(total)) * kLn2;
}

template <int D, bool E4M3>
void launch_few(const PagedAttnParams& p, const PagedSizes& sizes, hipStream_t stream) {
    hipLaunchKernelGGL((paged_few_kernel<D, E4M3>), dim3((unsigned)sizes.few_grid), dim3(kThreads), 0, stream, p);
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
    return s;
}

hipError_t launch_paged_attn(const PagedAttnParams& p, const PagedSizes& sizes, bool e4m3, hipStream_t stream) {
    const int width = tile_width(p.pool.head_dim);
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
    const int64_t waves = (int64_t)p.rows.total_rows * p.q_heads;
    const dim3 grid((unsigned)((waves + 3) / 4)), threads(kThreads);
    if (width == 128) hipLaunchKernelGGL(paged_join_kernel<128>, grid, threads, 0, stream, p);
    else hipLaunchKernelGGL(paged_join_kernel<64>, grid, threads, 0, stream, p);
    return hipGetLastError();
}

}  // namespace hspmd
