// The write of new tokens into the paged cache (rotation and quantisation fused in) and the read back.
//
// HBM-bound copies: a row of k or v is read once and written once.  The write gives a row (one token) to a wave, or to several where there
// are few rows: the wave finds the row's place, then walks the heads of q (turned, if given), k (turned) and v, with a lane holding
// VEC pairs of columns of a head as the rotation pairs them.  A head's largest magnitude is one exchange among its lanes.
// Write, with q turned: 12351 rows, 32 + 8 + 8 heads of 128, bf16 65 us = 4.8 TB/s, e4m3 60 us = 4.7; 14100 rows, 16 + 16 + 16 heads of 104, bf16 71 us = 4.1; 64 rows
// (a generation step) 5.2 us.  Read: 131754 rows, 8 heads of 128, e4m3 159 us = 5.1 TB/s, bf16 210 us = 5.1; 83 rows 3.3 us.
#include "paged_device.hpp"

namespace hspmd {

namespace {

template <int VEC, bool E4M3>
__global__ __launch_bounds__(kThreads) void kv_cache_write_kernel(CacheWriteParams p) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = (int)(unit / p.shares), share = (int)(unit % p.shares);
    if (row >= p.rows.total_rows) return;
    const RowPlace at = place_of(p.pool, p.rows, row);
    if (at.seq < 0) return;
    const int hd = p.pool.head_dim, half = hd / 2, pieces = half / VEC, heads_at_once = 64 / pieces;
    const int sub = lane / pieces, piece = lane % pieces;
    const bool turned = p.rope.table != nullptr;
    float c[VEC], s[VEC];
    if (turned) {
        int pos[4] = {at.pos, at.pos, at.pos, at.pos};
        if (p.rope.positions) {
#pragma unroll
            for (int a = 0; a < 4; ++a)
                if (a < p.rope.num_axes) pos[a] = p.rope.positions[a * p.rope.positions_stride + row];
        }
        if (sub < heads_at_once) load_turn<VEC>(p.rope, pos, piece * VEC, half, c, s);
    }
    // rounds of heads, those of q, of k and of v: everything but the lane's place in a round is the same for the wave
    const int kv = p.pool.kv_heads, q_rounds = (p.q_heads + heads_at_once - 1) / heads_at_once, kv_rounds = (kv + heads_at_once - 1) / heads_at_once;
    const int mine = sub * hd + piece * VEC, shift = p.pool.page_shift;
    const uint32_t place = (uint32_t)(sub << shift) * (uint32_t)p.pool.row_bytes;      // of the lane's head in a page, from the round's first
    const bool lane_used = sub < heads_at_once;
    for (int round = share; round < q_rounds + 2 * kv_rounds; round += p.shares) {
        const bool is_q = round < q_rounds, is_v = round >= q_rounds + kv_rounds;
        const int h0 = (is_q ? round : is_v ? round - q_rounds - kv_rounds : round - q_rounds) * heads_at_once;
        const bool in = lane_used && h0 + sub < (is_q ? p.q_heads : kv);
        const uint16_t* const src = (is_q ? p.q : is_v ? p.v : p.k) + row * (is_q ? p.q_stride : p.kv_stride) + h0 * hd;
        float lo[VEC], hi[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) lo[j] = hi[j] = 0.f;
        if (in) {
            load_floats<VEC, false>(src, mine, lo);
            load_floats<VEC, false>(src, mine + half, hi);
        }
        if (turned && !is_v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) turn_pair(lo[j], hi[j], c[j], s[j], lo[j], hi[j]);
        if (is_q) {
            uint16_t* const to = p.q_out + row * p.q_out_stride + h0 * hd;
            if (in) {
                store_floats<VEC, false>(to, mine, lo);
                store_floats<VEC, false>(to, mine + half, hi);
            }
            continue;
        }
        if (at.page < 0) continue;
        const int64_t token = ((int64_t)h0 << shift) + at.slot;
        uint8_t* const dst = (is_v ? p.pool.v : p.pool.k) + at.page * p.pool.page_bytes + token * p.pool.row_bytes + place;
        if constexpr (E4M3) {
            float amax = 0.f;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (is_finite(lo[j])) amax = fmaxf(amax, fabsf(lo[j]));
                if (is_finite(hi[j])) amax = fmaxf(amax, fabsf(hi[j]));
            }
            // the maximum over the head's lanes, in cyclic steps of 1, 2, 4, ... (a lane may count twice: it is a maximum)
            for (int step = 1; step < pieces; step *= 2) {
                int from = piece + step;
                from = (from >= pieces ? from - pieces : from) + sub * pieces;
                amax = fmaxf(amax, __shfl(amax, lane_used ? from : lane, 64));
            }
            if (!in) continue;
            const int e = e4m3_exponent(amax);
            const float unit_of = pow2(-e);
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                uint32_t w[VEC / 4];
#pragma unroll
                for (int j = 0; j < VEC / 4; ++j) {
                    float x[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float y = part ? hi[4 * j + i] : lo[4 * j + i];
                        x[i] = is_finite(y) ? y * unit_of : __builtin_nanf("");
                    }
                    w[j] = pack_e4m3(x[0], x[1], x[2], x[3]);
                }
                uint8_t* const to = dst + part * half + piece * VEC;
                if constexpr (VEC == 8) *reinterpret_cast<u32x2*>(to) = u32x2{w[0], w[1]};
                else *reinterpret_cast<uint32_t*>(to) = w[0];
            }
            if (piece == 0) {
                if (hd & 8) *reinterpret_cast<u32x2*>(dst + hd) = u32x2{0u, 0u};   // the columns up to a multiple of 16
                (is_v ? p.pool.v_scale : p.pool.k_scale)[at.page * p.pool.scale_page_bytes + token + (sub << shift)] = (uint8_t)(e + 127);
            }
        } else if (in) {
            store_floats<VEC, false>(dst, piece * VEC, lo);
            store_floats<VEC, false>(dst, half + piece * VEC, hi);
        }
    }
}

// a wave per row: 8 columns of k and of v per lane and step
template <bool E4M3>
__global__ __launch_bounds__(kThreads) void kv_cache_read_kernel(CacheReadParams p) {
    const int lane = threadIdx.x & 63;
    const int row = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= p.rows.total_rows) return;
    const RowPlace at = place_of(p.pool, p.rows, row);
    if (at.seq < 0) return;
    const int chunks = p.pool.head_dim / 8;
    for (int e = lane; e < p.pool.kv_heads * chunks; e += 64) {
        const int head = e / chunks, chunk = e % chunks;
        const int64_t token = ((int64_t)head << p.pool.page_shift) + at.slot;
        u32x4 out[2];
#pragma unroll
        for (int is_v = 0; is_v < 2; ++is_v) {
            if (at.page < 0) {
                const uint32_t w = at.pos < 0 ? 0u : 0x7fc07fc0u;   // no place: zeros; no page: NaN
                out[is_v] = u32x4{w, w, w, w};
                continue;
            }
            const uint8_t* src = (is_v ? p.pool.v : p.pool.k) + at.page * p.pool.page_bytes + token * p.pool.row_bytes;
            if constexpr (E4M3) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(src + chunk * 8);
                const float scale = scale_of((is_v ? p.pool.v_scale : p.pool.k_scale)[at.page * p.pool.scale_page_bytes + token]);
                const u32x2 a = e4m3_to_bf16(w[0], scale), b = e4m3_to_bf16(w[1], scale);
                out[is_v] = u32x4{a[0], a[1], b[0], b[1]};
            } else {
                out[is_v] = *reinterpret_cast<const u32x4*>(src + chunk * 16);
            }
        }
        const int64_t to = row * p.kv_stride + e * 8;
        *reinterpret_cast<u32x4*>(p.k + to) = out[0];
        *reinterpret_cast<u32x4*>(p.v + to) = out[1];
    }
}

}  // namespace

hipError_t launch_cache_write(CacheWriteParams p, bool e4m3, hipStream_t stream) {
    if (p.rows.total_rows == 0 || p.rows.num_seqs == 0) return hipSuccess;
    const int half = p.pool.head_dim / 2, vec = half % 8 == 0 ? 8 : 4;
    const int heads_at_once = 64 / (half / vec);
    const int rounds = (p.q_heads + heads_at_once - 1) / heads_at_once + 2 * ((p.pool.kv_heads + heads_at_once - 1) / heads_at_once);
    p.shares = (int)std::max<int64_t>(1, std::min<int64_t>(rounds, (4096 + p.rows.total_rows - 1) / p.rows.total_rows));
    const int64_t units = (int64_t)p.rows.total_rows * p.shares;
    const dim3 grid((unsigned)((units + 3) / 4)), threads(kThreads);
    if (e4m3 && vec == 8) hipLaunchKernelGGL((kv_cache_write_kernel<8, true>), grid, threads, 0, stream, p);
    else if (e4m3) hipLaunchKernelGGL((kv_cache_write_kernel<4, true>), grid, threads, 0, stream, p);
    else if (vec == 8) hipLaunchKernelGGL((kv_cache_write_kernel<8, false>), grid, threads, 0, stream, p);
    else hipLaunchKernelGGL((kv_cache_write_kernel<4, false>), grid, threads, 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheReadParams& p, bool e4m3, hipStream_t stream) {
    if (p.rows.total_rows == 0 || p.rows.num_seqs == 0) return hipSuccess;
    const dim3 grid((unsigned)((p.rows.total_rows + 3) / 4)), threads(kThreads);
    if (e4m3) hipLaunchKernelGGL(kv_cache_read_kernel<true>, grid, threads, 0, stream, p);
    else hipLaunchKernelGGL(kv_cache_read_kernel<false>, grid, threads, 0, stream, p);
    return hipGetLastError();
}

}  // namespace hspmd
