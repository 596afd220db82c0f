// Linear attention with a decay for each head, chunked form: the forward.
#include "linear_walk.hpp"

namespace hspmd {
namespace {

template <int D, bool ONE, int PARTS, int NB>
__global__ __launch_bounds__(D / 32 * 64, 2) void linear_fwd_kernel(LinearParams p) {
    __shared__ __align__(16) char lds[Lds<D, 2, ONE>::bytes(true, false)];
    int role, kv_head, slot;
    Segment seg;
    if (!item_of_block<true>(p.shape, 1, role, kv_head, slot) || !find_segment(p.shape, slot, seg)) return;
    outputs_of<D, false, false, ONE, PARTS, 2, NB>(p, forward_routine(p), seg, slot, kv_head, lds);
}

template <int D, bool ONE, int NB>
void launch(const LinearParams& p, hipStream_t stream) {
    // (o is rounded to bf16: two parts of the state suffice for it, a final state that is kept takes three)
    const auto kernel = p.final.data ? linear_fwd_kernel<D, ONE, 3, NB> : linear_fwd_kernel<D, ONE, 2, NB>;
    kernel<<<grid_of(p, 1), D / 32 * 64, 0, stream>>>(p);
}

}  // namespace

LinearSizes linear_sizes(int32_t total_rows, int32_t num_seqs, int32_t max_rows, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                         bool backward, bool decays) {
    LinearSizes s{};
    // As many segments as make one round of workgroups, 512 (a sequence ends in half a segment on average); fewer leave the device idle, more cost states
    // and a second round's end.  (The headline pack, 24 heads: 345 us in segments of 1024, 328 of 1856; ten prompts, 16 heads: 158 of 1024,
    // 131 of 640, 168 of 384.)  The backward, three workgroups for each, takes some more.  Sequences of up to two segments stay whole: that takes less
    // than a second reading of their keys and values.
    const int64_t longest = max_rows > 0 && max_rows < total_rows ? max_rows : total_rows;
    const int64_t round = (backward ? 576 : 512) - (int64_t)num_seqs * kv_heads / 2;
    int64_t seg = (int64_t)total_rows * kv_heads / (round < 256 ? 256 : round);
    seg = (seg + kLinearChunk - 1) / kLinearChunk * kLinearChunk;
    seg = seg < 256 ? 256 : seg > 16384 ? 16384 : seg;
    s.seg_rows = longest <= 2 * seg ? 0 : (int32_t)seg;
    if (s.seg_rows > 0) {
        s.slots = linear_slots(total_rows, num_seqs, seg);
        s.entries = linear_entries(total_rows, seg);
        s.windows = linear_windows(total_rows, seg);
    } else {
        s.slots = num_seqs;
    }
    const auto rounded = [](int64_t bytes) { return (size_t)((bytes + 255) / 256 * 256); };
    s.state_bytes = rounded(s.entries * kv_heads * head_dim * head_dim * 4);
    s.decay_bytes = rounded(s.entries * kv_heads * 4);
    s.q_row_bytes = rounded((int64_t)total_rows * q_heads * 4);
    s.k_row_bytes = rounded((int64_t)total_rows * kv_heads * 4);
    s.slot_bytes = rounded(s.slots * kv_heads * 8);
    s.anchor_bytes = rounded(decays ? linear_anchors(total_rows) * kv_heads * linear_anchor_elements(head_dim) * 4 : 0);
    return s;
}

hipError_t launch_linear_fwd(const LinearParams& p, hipStream_t stream) {
    if (p.shape.slots > 0) {
        launch_linear_states(p, false, p.final.data ? 3 : 2, stream);
        with_shape(p.shape, [&](auto d, auto blocks, auto one) { launch<decltype(d)::value, decltype(one)::value, decltype(blocks)::value>(p, stream); });
    }
    return hipGetLastError();
}

}  // namespace hspmd
