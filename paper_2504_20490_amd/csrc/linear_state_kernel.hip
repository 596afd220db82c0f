// Linear attention with a decay for each head: what segments of a long sequence add to the state, and the states from segment to segment.
#include "linear_walk.hpp"

namespace hspmd {
namespace {

// What a segment adds to the state, into the entry of the segment that it reaches next; `roles` 2: also what it adds to the gradient.
template <int D, int PARTS, int NB>
__global__ __launch_bounds__(D / 32 * 64, 2) void linear_state_kernel(LinearParams p, int roles) {
    __shared__ __align__(16) char lds[Lds<D, 2, true>::bytes(false, false)];
    int role, kv_head, slot;
    Segment seg;
    if (!item_of_block(p.shape, roles, role, kv_head, slot) || !find_segment(p.shape, slot, seg) || seg.count == 1) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), d = p.shape.head_dim;
    const bool last = seg.index == seg.count - 1;
    if (role == 0 ? last : seg.index == 0) return;
    State<NB> S;
    S.clear(0.f);
    const float decay = role == 0 ? walk<D, false, false, false, true, PARTS, 2, NB>(p, forward_routine(p), seg, kv_head, lds, S)
                                  : walk<D, true, false, false, false, PARTS, 2, NB>(p, dv_routine(p), seg, kv_head, lds, S);
    const int64_t own = (int64_t)(seg.entry + seg.index) * p.shape.kv_heads + kv_head;
    float* const to = role == 0 ? p.states + (own + p.shape.kv_heads) * d * d : p.d_states + (own - p.shape.kv_heads) * d * d;
    S.store(to, d, wave, lane);
    if (wave == D / 32 - 1 && lane == 0 && (role == 0 || last)) p.seg_decay[own] = decay;
}

// Passes states from segment to segment, elementwise: entry b holds what segment b - 1 adds and receives the state at the start of segment b.
// blockIdx.y: 0 states, forwards; 1 their gradients, backwards.
constexpr int kPassThreads = 256, kPassAhead = 4;
__global__ __launch_bounds__(kPassThreads) void linear_pass_kernel(LinearParams p, int parts) {
    const LinearShape& sh = p.shape;
    const int part = blockIdx.x % parts, kv_head = blockIdx.x / parts % sh.kv_heads, window = blockIdx.x / parts / sh.kv_heads;
    // the last sequence that starts in the window's tokens or before
    const int lane = threadIdx.x & 63;
    const int64_t end = ((int64_t)window + 1) * sh.seg_rows;
    int lo = 0, n = sh.num_seqs;
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        const bool before = at < n && linear_rows(sh.cu_rows[lo + at], 0, sh.total_rows).start < end;
        const uint64_t m = __ballot(before);
        const int found = m ? 63 - __builtin_clzll(m) : 0;
        lo += found * step;
        n = min(step, n - found * step);
    }
    const int seq = lo;
    const LinearRows r = linear_rows(sh.cu_rows[seq], sh.cu_rows[seq + 1], sh.total_rows);
    const int count = linear_segments(r.n, sh.seg_rows);
    if (count == 1 || r.start / sh.seg_rows != window) return;
    const int d = sh.head_dim, e = (part * kPassThreads + threadIdx.x) * 4;
    if (e >= d * d) return;
    const bool later = blockIdx.y == 1;
    const int64_t first = (int64_t)linear_first_entry(r.start, sh.seg_rows) * sh.kv_heads + kv_head;
    float* const base = (later ? p.d_states : p.states) + first * d * d + e;
    const float* const decay = p.seg_decay + first;
    const int64_t step = (int64_t)sh.kv_heads * d * d;
    bool exists;
    const float* const from = state_of(later ? p.final : p.initial, seq, kv_head, d, &exists);
    f32x4 s{};
    if (from) s = *reinterpret_cast<const f32x4*>(from + e);
    else if (exists) s = s + __builtin_nanf("");
    *reinterpret_cast<f32x4*>(base + (later ? count - 1 : 0) * step) = s;
    // number i of the way: entry i, or (later) count - 1 - i; the segment passed over between numbers i - 1 and i is that of number i - 1
    const int64_t way = later ? -1 : 1, begin = later ? count - 1 : 0;
    for (int i = 1; i < count; i += kPassAhead) {
        f32x4 x[kPassAhead];
        float g[kPassAhead];
#pragma unroll
        for (int j = 0; j < kPassAhead; ++j) {
            const int k = i + j;          // (all read before any is written)
            if (k >= count) break;
            x[j] = *reinterpret_cast<const f32x4*>(base + (begin + k * way) * step);
            g[j] = decay[(begin + (k - 1) * way) * sh.kv_heads];
        }
#pragma unroll
        for (int j = 0; j < kPassAhead; ++j) {
            if (i + j >= count) break;
            s = s * fast_exp2(g[j]) + x[j];
            *reinterpret_cast<f32x4*>(base + (begin + (i + j) * way) * step) = s;
        }
    }
}

template <int D, int NB>
void launch(const LinearParams& p, int roles, int parts, hipStream_t stream) {
    const auto kernel = parts == 3 ? linear_state_kernel<D, 3, NB> : linear_state_kernel<D, 2, NB>;
    kernel<<<grid_of(p, roles), D / 32 * 64, 0, stream>>>(p, roles);
}

}  // namespace

void launch_linear_states(const LinearParams& p, bool backward, int parts, hipStream_t stream) {
    if (p.shape.seg_rows == 0) return;
    const int roles = backward ? 2 : 1, d = p.shape.head_dim, blocks = (d * d / 4 + kPassThreads - 1) / kPassThreads;
    with_shape(p.shape, [&](auto width, auto blocks, auto) { launch<decltype(width)::value, decltype(blocks)::value>(p, roles, parts, stream); });
    linear_pass_kernel<<<dim3((unsigned)((int64_t)p.shape.windows * p.shape.kv_heads * blocks), roles), kPassThreads, 0, stream>>>(p, blocks);
}

}  // namespace hspmd
