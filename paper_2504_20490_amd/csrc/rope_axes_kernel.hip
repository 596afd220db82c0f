// Rotary embedding of q and k with positions given per token on up to four axes.
//
//   y_i = x_i cos(p_a theta_i) - x_{i+h} sin(p_a theta_i),  y_{i+h} = x_{i+h} cos(p_a theta_i) + x_i sin(p_a theta_i),  h = head_dim / 2, a = axis of pair i
// HBM-bound: every element of q and k is read once and written once.  A wave (or several, where there are few tokens) takes one token and
// walks its heads, those of q and then those of k; a lane owns VEC pairs of columns, so that their cosines and sines are fetched once
// per token and stay in registers, whatever axes the pairs belong to.  All but a lane's place in a round of heads is scalar.
// 32768 tokens, 24 + 24 heads of 128, bf16: 150 us = 5.4 TB/s; 16384 tokens, 32 + 8 heads, fp32: 130 us = 5.2 TB/s; 192 tokens, 2 + 2 heads of 64: 4.5 us.
// Heads of 104 (8-byte pieces, 52 of 64 lanes): 4.4 TB/s; several rounds of heads under way at once, or 16-byte pieces whose partners other lanes hold, are
// no faster (50.0 and 55.0 us against 50.1: 16384 tokens, 16 + 16 heads).
#include "paged_device.hpp"

namespace hspmd {

namespace {

// VEC pairs of every head per lane; F32: fp32 tensors
template <int VEC, bool F32>
__global__ __launch_bounds__(kThreads) void rope_axes_kernel(RopeAxesParams p) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token = (int)(unit / p.shares), share = (int)(unit % p.shares);
    if (token >= p.tokens) return;
    const int half = p.head_dim / 2, pieces = half / VEC, heads_at_once = 64 / pieces;
    const int sub = lane / pieces, piece = lane % pieces;
    if (sub >= heads_at_once) return;
    int pos[4] = {0, 0, 0, 0};
#pragma unroll
    for (int a = 0; a < 4; ++a)
        if (a < p.rope.num_axes) pos[a] = p.rope.positions[a * p.rope.positions_stride + token];
    float c[VEC], s[VEC];
    load_turn<VEC>(p.rope, pos, piece * VEC, half, c, s);
#pragma unroll
    for (int j = 0; j < VEC; ++j) s[j] *= p.sin_sign;
    // rounds of heads, those of q and then those of k: everything but the lane's place in a round is the same for the wave
    const int q_rounds = (p.q_heads + heads_at_once - 1) / heads_at_once, k_rounds = (p.kv_heads + heads_at_once - 1) / heads_at_once;
    const int mine = sub * p.head_dim + piece * VEC;
    for (int round = share; round < q_rounds + k_rounds; round += p.shares) {
        const bool is_k = round >= q_rounds;
        const int h0 = (is_k ? round - q_rounds : round) * heads_at_once;
        if (h0 + sub >= (is_k ? p.kv_heads : p.q_heads)) continue;
        constexpr int kBytes = F32 ? 4 : 2;
        const char* const src = static_cast<const char*>(is_k ? p.k : p.q) + (token * (is_k ? p.kv_stride : p.q_stride) + h0 * p.head_dim) * kBytes;
        char* const dst = static_cast<char*>(is_k ? p.k_out : p.q_out) + (token * (is_k ? p.kv_out_stride : p.q_out_stride) + h0 * p.head_dim) * kBytes;
        float lo[VEC], hi[VEC];
        load_floats<VEC, F32>(src, mine, lo);
        load_floats<VEC, F32>(src, mine + half, hi);
#pragma unroll
        for (int j = 0; j < VEC; ++j) turn_pair(lo[j], hi[j], c[j], s[j], lo[j], hi[j]);
        store_floats<VEC, F32>(dst, mine, lo);
        store_floats<VEC, F32>(dst, mine + half, hi);
    }
}

}  // namespace

hipError_t launch_rope_axes(RopeAxesParams p, bool f32, hipStream_t stream) {
    if (p.tokens == 0) return hipSuccess;
    const int half = p.head_dim / 2;
    const int vec = !f32 && half % 8 == 0 ? 8 : 4;
    const int heads_at_once = 64 / (half / vec);
    const int rounds = (p.q_heads + heads_at_once - 1) / heads_at_once + (p.kv_heads + heads_at_once - 1) / heads_at_once;
    // enough waves for the device: 16 for each of 256 compute units
    p.shares = (int)std::max<int64_t>(1, std::min<int64_t>(rounds, (4096 + p.tokens - 1) / p.tokens));
    const int64_t units = (int64_t)p.tokens * p.shares;
    const dim3 grid((unsigned)((units + 3) / 4)), threads(kThreads);
    if (f32) hipLaunchKernelGGL((rope_axes_kernel<4, true>), grid, threads, 0, stream, p);
    else if (vec == 8) hipLaunchKernelGGL((rope_axes_kernel<8, false>), grid, threads, 0, stream, p);
    else hipLaunchKernelGGL((rope_axes_kernel<4, false>), grid, threads, 0, stream, p);
    return hipGetLastError();
}

}  // namespace hspmd
