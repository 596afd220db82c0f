// Linear attention with a decay for each head, chunked form: the gradients.
#include "linear_walk.hpp"

namespace hspmd {
namespace {

// DECAYS: their gradients are wanted, and with them the dot products and the anchors, which cost a quarter on one query head per KV head (headline pack, 24 heads: 1095 us with, 865
// without; fp32 gradients 1200 and 965; 32 query heads on 8 KV heads: 1130 and 940, fp32 1680 and 1340).  The other gradients are the same bits.
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
// token from t on and one before t.  Of these pairs, a chunk's own and those with a token on one side of the chunk come from the dot products.
// Those across the whole chunk are <e^{G_L} S, R>, S in front of it and R behind it.  Between two chunks <S, R> is
//   what lies across the left one + its keys' = what lies across the right one + its queries',
// so from a place where <S, R> is known, what lies across the chunks next to it follows by differences.  These keep the rounding errors of all terms on the way, where
// the value itself shrinks with the decays: carried along a segment of 8192 tokens they came to 1e-3 of a fixed decay's gradient, and to as much of rows near others
// with 10^4 times their gradients.  So <S, R> is known at the segment's ends and at every fourth chunk (its anchors), and a chunk in between takes the
// difference from the side where the terms on the way are smaller.  What this launch takes is reading them: 101 us for the headline pack, 4 TB/s.  (Against the definition in 64
// bits over 8192 rows: every 64 rows' gradients off by 1e-6 to 3e-6 of their norm, a fixed decay's by up to 8e-6 of its rows' norm.  Anchors at every second
// chunk: 5e-6 and 15 % more time for the backward, at every eighth 2e-5 and 6 % less.)
constexpr int kDecayWaves = 8, kDecayBlocks = kDecayWaves / kLinearAnchor;
static_assert(kLinearAnchor == 4 && kDecayWaves % kLinearAnchor == 0, "the waves of an anchor's chunks share its sum");

struct ChunkSums {
    float keys, queries;         // pairs of its keys with what is behind it, of its queries with what is in front
    float most_keys, most_queries;     // by their magnitudes
    float decay;                 // 0: it leaves nothing
};

// What lies across each chunk of a block, from the right (its last chunk) to the left, into whole[]; n chunks; *across: <S, R> at the block's right end, then at its left one.
// `left`: what lies across the leftmost chunk (anchored), or <S, R> at the left end
__device__ __forceinline__ void across_chunks(const ChunkSums* sums, int n, bool anchored, float left, float* across, float (&whole)[kLinearAnchor]) {
    float noise[kLinearAnchor], from = *across, most = fabsf(from);      // (noise: the largest term on the way)
#pragma unroll
    for (int i = 0; i < kLinearAnchor; ++i) {
        if (i >= n) break;
        // a decay that leaves nothing leaves no pairs across it either, not even rounding errors
        const bool none = sums[i].decay == 0.f;
        whole[i] = none ? 0.f : from - sums[i].keys;
        noise[i] = none ? 0.f : fmaxf(most, sums[i].most_keys);
        from = whole[i] + sums[i].queries;
        most = fmaxf(noise[i], sums[i].most_queries);
    }
    from = left, most = fabsf(left);
#pragma unroll
    for (int i = kLinearAnchor - 1; i >= 0; --i) {
        if (i >= n) continue;
        const bool known = anchored && i == kLinearAnchor - 1;
        const float x = known ? left : from - sums[i].queries, noise_x = known ? 0.f : fmaxf(most, sums[i].most_queries);
        // (a side that a NaN reaches is not taken while there is another)
        if (x == x && (whole[i] != whole[i] || noise_x < noise[i])) whole[i] = x, noise[i] = noise_x;
        from = whole[i] + sums[i].keys;
        most = fmaxf(noise[i], sums[i].most_keys);
    }
    *across = whole[kLinearAnchor - 1] + sums[kLinearAnchor - 1].queries;
}

__global__ __launch_bounds__(kDecayWaves * 64) void linear_decay_kernel(LinearParams p) {
    __shared__ ChunkSums sums[kDecayWaves];
    __shared__ float products[kDecayWaves];
    __shared__ double totals[kDecayWaves];
    const LinearShape& sh = p.shape;
    int role, kv_head, slot;
    if (!item_of_block(sh, 1, role, kv_head, slot)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)slot * sh.kv_heads + kv_head;
    const bool fixed = p.decay_stride == 0;
    Segment seg;
    if (!find_segment(sh, slot, seg)) {
        if (fixed && threadIdx.x == 0) p.decay_sums[item] = 0.;
        return;
    }
    const int chunks = (seg.rows + kLinearChunk - 1) / kLinearChunk, elements = linear_anchor_elements(sh.head_dim);
    float across = p.across[item];
    const float at_start = seg.index > 0 ? p.across[item - sh.kv_heads] : p.across[(int64_t)sh.slots * sh.kv_heads + item];
    double total = 0.;
    for (int last = chunks - 1; last >= 0; last -= kDecayWaves) {
        const int chunk = last - wave;
        const int64_t row = seg.start + chunk * kLinearChunk + lane;
        const bool there = chunk >= 0 && chunk * kLinearChunk + lane < seg.rows;
        // <S, R> of the anchor among the wave's four chunks, a quarter of the products
        const int anchor = last - (wave | (kLinearAnchor - 1));
        float product = 0.f;
        if (anchor > 0) {
            const int64_t from = ((int64_t)linear_anchor(seg.start, anchor, chunks) * sh.kv_heads + kv_head) * elements;
            f32x4 sum{};
            for (int i = (wave % kLinearAnchor) * 64 + lane; i < elements / 4; i += kLinearAnchor * 64)
                sum += reinterpret_cast<const f32x4*>(p.anchors + from)[i] * reinterpret_cast<const f32x4*>(p.d_anchors + from)[i];
            product = sum[0] + sum[1] + sum[2] + sum[3];
        }
        float near = 0.f, far_q = 0.f, far_k = 0.f;
        DecayLog2 g{0.f, 0.f};
        if (there) {
            g = split_decay_log2(p.log_decay[row * p.decay_stride + kv_head]);
            far_k = p.k_far[(int64_t)kv_head * sh.total_rows + row];
            for (int h = 0; h < sh.group; ++h) {
                const int64_t at = (int64_t)(kv_head * sh.group + h) * sh.total_rows + row;
                near += p.q_near[at];
                far_q += p.q_far[at];
            }
            near -= p.k_near[(int64_t)kv_head * sh.total_rows + row];
        }
        const ChunkSums mine = {wave_sum(far_k), wave_sum(far_q), wave_sum(fabsf(far_k)), wave_sum(fabsf(far_q)), fast_exp2(wave_sum(g.whole) + wave_sum(g.rest))};
        product = wave_sum(product);
        __syncthreads();                       // (the others have read the round before)
        if (lane == 0) {
            sums[wave] = mine;
            products[wave] = product;
        }
        __syncthreads();
        float whole_here = 0.f;
#pragma unroll
        for (int b = 0; b < kDecayBlocks; ++b) {
            const int first = b * kLinearAnchor, n = min(last - first + 1, kLinearAnchor);
            if (n <= 0) break;
            float left = at_start, whole[kLinearAnchor] = {};
            const bool anchored = last - first - (kLinearAnchor - 1) > 0;
            if (anchored) {
                left = 0.f;
#pragma unroll
                for (int i = 0; i < kLinearAnchor; ++i) left += products[first + i];
                left *= sums[first + kLinearAnchor - 1].decay;
            }
            across_chunks(sums + first, n, anchored, left, &across, whole);
#pragma unroll
            for (int i = 0; i < kLinearAnchor; ++i) whole_here = first + i == wave ? whole[i] : whole_here;
        }
        const float grad = sum_from(near + far_q, lane) + (sum_up_to(far_k) - far_k) + whole_here;
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
            total = 0.;
#pragma unroll
            for (int w = 0; w < kDecayWaves; ++w) total += totals[w];
            p.decay_sums[item] = total;
        }
    }
}

// A fixed decay's gradient is the sum over all tokens: one workgroup per KV head, in a fixed order.
__global__ __launch_bounds__(256) void linear_decay_sum_kernel(LinearParams p) {
    __shared__ double parts[4];
    double sum = 0.;
    for (int64_t i = threadIdx.x; i < p.shape.slots; i += 256) sum += p.decay_sums[i * p.shape.kv_heads + blockIdx.x];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) p.d_log_decay[blockIdx.x] = (float)(parts[0] + parts[1] + parts[2] + parts[3]);
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
