// Linear attention with a decay for each head, recurrent form: one token per sequence over a pool of states.
//   S' = e^g S + k v^T,   o_h = s S'^T q_h for each query head h of the group.
// Bound by reading and writing the states: 8 d^2 bytes for 3 d^2 + 2 d^2 group operations.  A workgroup takes a (sequence, KV head), or some
// of its columns (linear_step_columns); a thread owns four columns of every R-th row and keeps them in registers, so a state is read once and
// written once however many query heads share it, and all of a thread's reads are in flight at once.
#include "linear_device.hpp"

namespace hspmd {
namespace {

constexpr int kStepThreads = 256, kStepHeads = 4;    // query heads whose sums meet in LDS at a time

template <int PASSES>
__global__ __launch_bounds__(kStepThreads) void linear_step_kernel(LinearStepParams p, int columns, int parts) {
    __shared__ float q_rows[kStepHeads][128], k_row[128];
    __shared__ f32x4 sums[kStepHeads][kStepThreads];
    const int part = blockIdx.x % parts, kv_head = blockIdx.x / parts % p.kv_heads, seq = blockIdx.x / parts / p.kv_heads;
    const int d = p.head_dim, first_col = part * columns, lanes = min(columns, d - first_col) / 4, rows_per_pass = kStepThreads / lanes;
    const int row = threadIdx.x / lanes, col = first_col + threadIdx.x % lanes * 4;
    const bool works = row < rows_per_pass;
    bool from_exists, to_exists;
    const float* const from = state_of(p.initial, seq, kv_head, d, &from_exists);
    float* const to = state_of(p.final, seq, kv_head, d, &to_exists);
    f32x4 S[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int r = row + i * rows_per_pass;
        S[i] = f32x4{};
        if (from && works && r < d) S[i] = *reinterpret_cast<const f32x4*>(from + (int64_t)r * d + col);
        else if (from_exists && !from) S[i] = S[i] + __builtin_nanf("");
    }
    const float decay = fast_exp2(decay_log2(p.log_decay[seq * p.decay_stride + kv_head]));
    const auto value = [](uint16_t x) { return __uint_as_float((uint32_t)x << 16); };
    if (threadIdx.x < d) k_row[threadIdx.x] = value(p.k[seq * p.kv_stride + (int64_t)kv_head * d + threadIdx.x]);
    f32x4 v{};
    if (works) {
        const u32x2 raw = *reinterpret_cast<const u32x2*>(p.v + seq * p.kv_stride + (int64_t)kv_head * d + col);
        v = f32x4{__uint_as_float(raw[0] << 16), __uint_as_float(raw[0] & 0xffff0000u), __uint_as_float(raw[1] << 16), __uint_as_float(raw[1] & 0xffff0000u)};
    }
    for (int h0 = 0; h0 < p.group; h0 += kStepHeads) {
        const int heads = min(kStepHeads, p.group - h0);
        for (int i = threadIdx.x; i < heads * d; i += kStepThreads)
            q_rows[i / d][i % d] = value(p.q[seq * p.q_stride + (int64_t)(kv_head * p.group + h0) * d + i]);
        __syncthreads();
        if (works) {
            if (h0 == 0) {
#pragma unroll
                for (int i = 0; i < PASSES; ++i) {
                    const int r = row + i * rows_per_pass;
                    if (r < d) {
                        S[i] = S[i] * decay + v * k_row[r];
                        if (to) *reinterpret_cast<f32x4*>(to + (int64_t)r * d + col) = S[i];
                    }
                }
            }
            for (int h = 0; h < heads; ++h) {
                f32x4 sum{};
#pragma unroll
                for (int i = 0; i < PASSES; ++i) {
                    const int r = row + i * rows_per_pass;
                    if (r < d) sum += S[i] * q_rows[h][r];
                }
                sums[h][threadIdx.x] = sum;
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < heads * lanes; i += kStepThreads) {
            const int h = i / lanes, at = i % lanes;
            f32x4 sum = sums[h][at];
            for (int r = 1; r < rows_per_pass; ++r) sum += sums[h][r * lanes + at];
            store_grad4(p.o, ((int64_t)seq * p.q_heads + kv_head * p.group + h0 + h) * d + first_col + at * 4, false, sum[0] * p.scale, sum[1] * p.scale,
                        sum[2] * p.scale, sum[3] * p.scale);
        }
        // (the next heads' sums wait for the barrier behind their rows, which are read before this one's sums are written)
    }
}

}  // namespace

hipError_t launch_linear_step(const LinearStepParams& p, hipStream_t stream) {
    const int d = p.head_dim;
    const int64_t states = (int64_t)p.num_seqs * p.kv_heads;
    if (states == 0) return hipSuccess;
    const int columns = linear_step_columns(d, states), parts = (d + columns - 1) / columns;
    const unsigned grid = (unsigned)(states * parts);
    const int rows_per_pass = kStepThreads / (columns / 4), passes = (d + rows_per_pass - 1) / rows_per_pass;
    if (passes <= 4) linear_step_kernel<4><<<grid, kStepThreads, 0, stream>>>(p, columns, parts);
    else if (passes <= 8) linear_step_kernel<8><<<grid, kStepThreads, 0, stream>>>(p, columns, parts);
    else linear_step_kernel<16><<<grid, kStepThreads, 0, stream>>>(p, columns, parts);
    return hipGetLastError();
}

}  // namespace hspmd
