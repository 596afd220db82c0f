// Linear attention with a decay for each head, chunked form: the gradients.
#include "linear_walk.hpp"

namespace hspmd {
namespace {

// DECAYS: their gradients are wanted, and with them the dot products, which cost a sixth (headline pack, 24 heads: 965 us with, 860 without; fp32 gradients 1065 and 960,
// on 32 query heads of 8 KV heads 1460 and 1190).  The other gradients are the same bits.
template <int D, bool ONE, int WEIGHT_PARTS, int V_PARTS, int NB, bool DECAYS>
__global__ __launch_bounds__(D / 32 * 64, D == 128 && WEIGHT_PARTS == 3 && !ONE ? 1 : 2) void linear_bwd_kernel(LinearParams p) {
    __shared__ __align__(16) char lds[Lds<D, WEIGHT_PARTS, ONE>::bytes(true, DECAYS || Lds<D, WEIGHT_PARTS, ONE>::kLate)];
    int role, kv_head, slot;
    Segment seg;
    if (!item_of_block<true>(p.shape, 3, role, kv_head, slot) || !find_segment(p.shape, slot, seg)) return;
    if (role == 0) outputs_of<D, false, DECAYS, ONE, 3, WEIGHT_PARTS, NB>(p, dq_routine(p), seg, slot, kv_head, lds);
    else if (role == 1) outputs_of<D, true, DECAYS, ONE, 3, WEIGHT_PARTS, NB>(p, dk_routine(p), seg, slot, kv_head, lds);
    else outputs_of<D, true, false, ONE, V_PARTS, WEIGHT_PARTS, NB>(p, dv_routine(p), seg, slot, kv_head, lds);
}

// Gradients of the log decays, a workgroup per segment and KV head, from its last chunk to its first, a chunk per wave.  g_t weighs every pair of a
// token from t on and one before t.  Of these pairs, a chunk's own and those with a token on one side of the chunk come from the dot products;
// those across the whole chunk, <e^{G_L} S, R>, are what is left of <S, dS> at its end without its own keys.
constexpr int kDecayWaves = 8;
__global__ __launch_bounds__(kDecayWaves * 64) void linear_decay_kernel(LinearParams p) {
    __shared__ float keys[kDecayWaves], queries[kDecayWaves], dead[kDecayWaves], totals[kDecayWaves];
    const LinearShape& sh = p.shape;
    int role, kv_head, slot;
    if (!item_of_block(sh, 1, role, kv_head, slot)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)slot * sh.kv_heads + kv_head;
    const bool fixed = p.decay_stride == 0;
    Segment seg;
    if (!find_segment(sh, slot, seg)) {
        if (fixed && threadIdx.x == 0) p.decay_sums[item] = 0.f;
        return;
    }
    float across = p.across[item], total = 0.f;
    for (int last = (seg.rows + kLinearChunk - 1) / kLinearChunk - 1; last >= 0; last -= kDecayWaves) {
        const int chunk = last - wave;
        const int64_t row = seg.start + chunk * kLinearChunk + lane;
        const bool there = chunk >= 0 && chunk * kLinearChunk + lane < seg.rows;
        float near = 0.f, far_q = 0.f, far_k = 0.f, g = 0.f;
        if (there) {
            g = decay_log2(p.log_decay[row * p.decay_stride + kv_head]);
            far_k = p.k_far[(int64_t)kv_head * sh.total_rows + row];
            for (int h = 0; h < sh.group; ++h) {
                const int64_t at = (int64_t)(kv_head * sh.group + h) * sh.total_rows + row;
                near += p.q_near[at];
                far_q += p.q_far[at];
            }
            near -= p.k_near[(int64_t)kv_head * sh.total_rows + row];
        }
        const float all_k = wave_sum(far_k), all_q = wave_sum(far_q), all_g = wave_sum(g);
        __syncthreads();                       // (the others have read the round before)
        if (lane == 0) {
            keys[wave] = all_k;
            queries[wave] = all_q;
            // a decay that leaves nothing leaves no pairs across it either, not even rounding errors
            dead[wave] = fast_exp2(all_g) == 0.f ? 1.f : 0.f;
        }
        __syncthreads();
        float whole = 0.f, mine = 0.f;
#pragma unroll
        for (int w = 0; w < kDecayWaves; ++w) {
            whole = dead[w] != 0.f ? 0.f : across - keys[w];
            if (w == wave) mine = whole;
            across = whole + queries[w];
        }
        const float grad = sum_from(near + far_q, lane) + (sum_up_to(far_k) - far_k) + mine;
        if (there) {
            if (fixed) total += grad;
            else p.d_log_decay[row * sh.kv_heads + kv_head] = grad;
        }
    }
    if (fixed) {
        total = wave_sum(total);
        if (lane == 0) totals[wave] = total;
        __syncthreads();
        if (threadIdx.x == 0) {
            total = 0.f;
#pragma unroll
            for (int w = 0; w < kDecayWaves; ++w) total += totals[w];
            p.decay_sums[item] = total;
        }
    }
}

// A fixed decay's gradient is the sum over all tokens: one workgroup per KV head, in a fixed order.
__global__ __launch_bounds__(256) void linear_decay_sum_kernel(LinearParams p) {
    __shared__ float parts[4];
    float sum = 0.f;
    for (int64_t i = threadIdx.x; i < p.shape.slots; i += 256) sum += p.decay_sums[i * p.shape.kv_heads + blockIdx.x];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) p.d_log_decay[blockIdx.x] = parts[0] + parts[1] + parts[2] + parts[3];
}

template <int D, bool ONE, int NB, bool DECAYS>
void launch(const LinearParams& p, hipStream_t stream) {
    // dv rounded to bf16 needs two parts of the gradient of the state; that gradient itself, where it goes out, three
    const auto kernel = p.grad_f32 ? linear_bwd_kernel<D, ONE, 3, 3, NB, DECAYS>
                      : p.d_initial ? linear_bwd_kernel<D, ONE, 2, 3, NB, DECAYS> : linear_bwd_kernel<D, ONE, 2, 2, NB, DECAYS>;
    kernel<<<grid_of(p, 3), D / 32 * 64, 0, stream>>>(p);
}

}  // namespace

hipError_t launch_linear_bwd(const LinearParams& p, hipStream_t stream) {
    if (p.shape.slots > 0) {
        launch_linear_states(p, true, 3, stream);
        with_shape(p.shape, [&](auto d, auto blocks, auto one) {
            const auto with = p.d_log_decay ? launch<decltype(d)::value, decltype(one)::value, decltype(blocks)::value, true>
                                            : launch<decltype(d)::value, decltype(one)::value, decltype(blocks)::value, false>;
            with(p, stream);
        });
    }
    if (p.d_log_decay) {
        if (p.shape.slots > 0) linear_decay_kernel<<<grid_of(p, 1), kDecayWaves * 64, 0, stream>>>(p);
        if (p.decay_stride == 0) linear_decay_sum_kernel<<<(unsigned)p.shape.kv_heads, 256, 0, stream>>>(p);
    }
    return hipGetLastError();
}

}  // namespace hspmd
