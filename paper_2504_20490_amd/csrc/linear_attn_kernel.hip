// Linear attention with a decay for each head, chunked form, forward and backward.
//
// Per sequence and KV head, with G the running sum of the log decays from a chunk's start, S the state at that start and s the scale:
//   o_t  = s e^{G_t} S^T q_t + s sum_{j <= t} e^{G_t - G_j} <q_t, k_j> v_j,      S' = e^{G_L} S + sum_j e^{G_L - G_j} k_j v_j^T.
// The gradients are the same form with other tensors: dq looks backwards like o (targets dO, sources v and k, the transposed state),
// dk and dv look forwards (targets v and k, sources dO, q and q, dO) with R, the gradient of the state at the chunk's end:
//   dk_t = e^{G_L - G_t} R v_t + s sum_{i >= t} e^{G_i - G_t} <v_t, dO_i> q_i,    R' = e^{G_L} R + s sum_i e^{G_i} q_i dO_i^T.
// So one routine does all four: targets a, sources b and c, state sum b c^T.
#include "linear_device.hpp"

namespace hspmd {
namespace {

// Long sequences: segments of them go to different workgroups.  What each adds to the state is computed first (OUT false below), a small
// launch passes the states from segment to segment, and then every segment starts with the state that reaches it.

// What the routine below is given
struct Routine {
    const uint16_t* a;       // targets, [T, a_heads, d]
    const uint16_t* b;       // sources
    const uint16_t* c;
    const uint16_t* e;       // DOTS: the tensor whose gradient the output is
    int64_t a_stride, b_stride, c_stride, e_stride;
    float scale_in, scale_state;   // of what the state gives to a target, of what a source gives to the state
    void* out;
    bool out_f32;
    bool transposed;         // the state is b c^T transposed to how it lies in memory
    float* near;             // DOTS: [heads][total_rows], see LinearParams
    float* far;
};

template <int D>
struct Lds {
    static constexpr int kWaves = D / 32;
    static constexpr int kTile = kLinearChunk * D * 2;
    static constexpr int kB = 0, kC = kTile, kA = 2 * kTile, kP = 3 * kTile;
    static constexpr int kPairs = 3 * 4 * 1024;               // [block of pairs][step of 16 sources][part][lane]
    static constexpr int kSums = kP + kPairs;                 // running sums of the log decays, target and source weights
    static constexpr int kNear = kSums + 3 * kLinearChunk * 4;
    static constexpr int kFar = kNear + 3 * 32 * 4;
    static constexpr int kE = kFar + kWaves * kLinearChunk * 4;
    static constexpr int bytes(bool out, bool dots) { return dots ? kE + kTile : out ? kNear : kA + 3 * kLinearChunk * 4; }
};

typedef int i32x4 __attribute__((ext_vector_type(4)));

// A tile of a chunk's rows on its way from memory to LDS.  Rows behind the segment's end and columns behind head_dim read as zeros
// (an address outside the buffer resource), so that nothing behind a sequence ever meets a product.
template <int D>
struct TileLoad {
    static constexpr int kThreadsHere = D / 32 * 64, kRowsPerPass = kThreadsHere / (D / 8), kPasses = kLinearChunk / kRowsPerPass;
    u32x4 r[kPasses];
    __device__ __forceinline__ void issue(const uint16_t* first_row, int64_t stride, int rows, int head_dim) {
        const int row = threadIdx.x / (D / 8), col = threadIdx.x % (D / 8) * 8, there = col < head_dim ? rows : 0;
        const uint32_t off = (uint32_t)(row * (int)stride + col) * 2u;
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(first_row), 0, 0x7fffffff, 0x00020000);
#pragma unroll
        for (int i = 0; i < kPasses; ++i)
            r[i] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, row + i * kRowsPerPass < there ? off : 0x80000000u, i * kRowsPerPass * (int)stride * 2, 0);
    }
    // ends the life of what was put: a load that is not always made again would else keep its registers throughout the loop
    __device__ __forceinline__ void drop() {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) r[i] = u32x4{};
    }
    __device__ __forceinline__ void put(char* tile) const {
        const int row = threadIdx.x / (D / 8), col = threadIdx.x % (D / 8) * 8;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) *reinterpret_cast<u32x4*>(tile + tile_offset<D>(row + i * kRowsPerPass, col)) = r[i];
    }
};

// The wave's part of a state: columns 32 wave .. + 31 (of c) along the lanes, all D rows (of b) in registers; register i of
// block db holds row 32 db + 16 (i / 8) + 8 (lane / 32) + i % 8.
template <int D>
struct State {
    f32x16 x[D / 32];
    __device__ __forceinline__ void clear(float value) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[db][i] = value;
    }
    // as `in memory`: [row][col], or [col][row]
    __device__ __forceinline__ void load(const float* m, int d, bool transposed, int wave, int lane) {
        const int col = wave * 32 + (lane & 31);
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = db * 32 + h * 16 + (lane >> 5) * 8;
                const bool there = row < d && col < d;
                if (transposed) {
                    f32x4 u{}, v{};
                    if (there) {
                        u = *reinterpret_cast<const f32x4*>(m + (int64_t)col * d + row);
                        v = *reinterpret_cast<const f32x4*>(m + (int64_t)col * d + row + 4);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[db][8 * h + i] = u[i], x[db][8 * h + 4 + i] = v[i];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[db][8 * h + i] = there ? m[(row + i) * d + col] : 0.f;
                }
            }
    }
    __device__ __forceinline__ void store(float* m, int d, int wave, int lane) const {
        const int col = wave * 32 + (lane & 31);
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = db * 32 + h * 16 + (lane >> 5) * 8;
                if (row < d && col < d) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) m[(row + i) * d + col] = x[db][8 * h + i];
                }
            }
    }
    // this lane's share of the sum over all elements of this state times the one in memory
    __device__ __forceinline__ float dot(const float* m, int d, bool transposed, int wave, int lane) const {
        const int col = wave * 32 + (lane & 31);
        float sum = 0.f;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = db * 32 + h * 16 + (lane >> 5) * 8;
                if (row < d && col < d) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += x[db][8 * h + i] * (transposed ? m[(int64_t)col * d + row + i] : m[(row + i) * d + col]);
                }
            }
        return sum;
    }
};

// A hidden pair has the weight 0, and 0 times an infinity or NaN is NaN: sources that hold one are left out of the products, element by element, and
// added for the targets that see them.
__device__ __forceinline__ bool all_finite(const bf16x8 (&x)[4]) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 most{};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        union { bf16x8 v; u32x4 u; } c;
        c.v = x[t];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t m = c.u[i] & 0x7fff7fffu;
            most = __builtin_elementwise_max(most, *reinterpret_cast<const u16x2*>(&m));
        }
    }
    return !__any(most[0] >= 0x7f80 || most[1] >= 0x7f80);
}
__device__ __forceinline__ bf16x8 finite_part(bf16x8 x) {
    union { bf16x8 v; u32x4 u; } c;
    c.v = x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c.u[i] = (c.u[i] & 0x7f80u) == 0x7f80u ? c.u[i] & 0xffff0000u : c.u[i];
        c.u[i] = (c.u[i] & 0x7f800000u) == 0x7f800000u ? c.u[i] & 0xffffu : c.u[i];
    }
    return c.v;
}

// What the sources of the own chunk give: weights times c, (source block, target block) of 32 x 32 pairs by their number, see kPairs
template <int D, bool LATER, bool FINITE>
__device__ __forceinline__ void add_own_chunk(const char* lds, const bf16x8 (&sources)[4], int wave, int lane, f32x16 (&out)[2]) {
    const char* const weights = lds + Lds<D>::kP + lane * 16;
#pragma unroll
    for (int blk = 0; blk < 3; ++blk) {
        const int sb = LATER ? (blk > 0) : blk >> 1, tb = LATER ? blk >> 1 : (blk > 0);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const bf16x8 c = FINITE ? sources[2 * sb + tt] : finite_part(sources[2 * sb + tt]);
            out[tb] = mfma(c, *reinterpret_cast<const bf16x8*>(weights + (blk * 4 + tt * 2) * 1024), out[tb]);
            out[tb] = mfma(c, *reinterpret_cast<const bf16x8*>(weights + (blk * 4 + tt * 2 + 1) * 1024), out[tb]);
        }
    }
    if (FINITE) return;
    const char* const tile = lds + Lds<D>::kC;
    const int t32 = lane & 31, hh = lane >> 5;
#pragma unroll 1
    for (int s = 0; s < kLinearChunk; ++s) {
        const int sb = s / 32, r = s % 32;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            if (LATER ? sb < tb : sb > tb) continue;
            const bool sees = sb != tb || (LATER ? r >= t32 : r <= t32);
            // the weight of (s, t32) as it was laid out for the products: lane 32 (r / 4 % 2) + t32, element 4 (r / 8 % 2) + r % 4 of step r / 16
            const char* const at = lds + Lds<D>::kP + ((sb + tb) * 4 + (r / 16) * 2) * 1024 + (32 * (r / 4 % 2) + t32) * 16 + (4 * (r / 8 % 2) + r % 4) * 2;
            const float weight = (float)*reinterpret_cast<const __bf16*>(at) + (float)*reinterpret_cast<const __bf16*>(at + 1024);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int col = wave * 32 + 8 * (i / 4) + 4 * hh + i % 4;
                const uint32_t raw = *reinterpret_cast<const uint16_t*>(tile + tile_offset<D>(s, col & ~3) + (col & 3) * 2);
                if (sees && (raw & 0x7f80) == 0x7f80) out[tb][i] += weight * __uint_as_float(raw << 16);
            }
        }
    }
}

// Walks a segment's chunks, forwards or (LATER) backwards, with the state that reaches it in `S`.
//   LATER   targets see the tokens from themselves on, and a KV head's sources are those of all its query heads (dk, dv); else they see the
//           tokens up to themselves, and a KV head's targets are those of all its query heads (o, dq)
//   OUT     outputs are wanted, not only the state
//   DOTS    the dot products of the output with the tensor it is the gradient of, the part from the own chunk (without the token's own) and
//           the part from the state apart
//   ONE     a KV head has one query head
// Returns the log2 of the segment's decay.
template <int D, bool LATER, bool OUT, bool DOTS, bool ONE>
__device__ __forceinline__ float walk(const LinearParams& p, const Routine& f, const Segment& seg, int kv_head, char* lds, State<D>& S) {
    using L = Lds<D>;
    constexpr int kWaves = L::kWaves;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int d = p.shape.head_dim, group = ONE ? 1 : p.shape.group;
    const int hh = lane >> 5;
    TileReads<D> reads;
    reads.init(lane);
    char* const tile_a = lds + L::kA;
    char* const tile_b = lds + L::kB;
    char* const tile_c = lds + L::kC;
    char* const tile_e = lds + L::kE;
    float* const sums = reinterpret_cast<float*>(lds + (OUT ? L::kSums : L::kA));
    float* const in_weight = sums + kLinearChunk;
    float* const out_weight = in_weight + kLinearChunk;
    float* const near = reinterpret_cast<float*>(lds + L::kNear);
    float* const far = reinterpret_cast<float*>(lds + L::kFar);
    const bool has_columns = wave * 32 < d;

    const int chunks = (seg.rows + kLinearChunk - 1) / kLinearChunk;
    const int target_heads = LATER ? p.shape.kv_heads : p.shape.q_heads;
    float all_decay = 0.f;

    TileLoad<D> la, lb, lc, le;
    float next_g = 0.f;
    const int first_target = LATER ? kv_head : kv_head * group, first_source = LATER ? kv_head * group : kv_head;
    const uint16_t* const base_a = f.a + seg.start * f.a_stride + (int64_t)first_target * d;
    const uint16_t* const base_e = f.e + seg.start * f.e_stride + (int64_t)first_target * d;
    const uint16_t* const base_b = f.b + seg.start * f.b_stride + (int64_t)first_source * d;
    const uint16_t* const base_c = f.c + seg.start * f.c_stride + (int64_t)first_source * d;
    const float* const base_g = p.log_decay + seg.start * p.decay_stride + kv_head;
    // the tiles of chunk number n of the walk and query head h of the group, if there is that chunk
    auto issue = [&](int n, int h) {
        const int chunk = LATER ? chunks - 1 - n : n;
        const int first = n < chunks ? chunk * kLinearChunk : 0, rows = n < chunks ? seg.rows - first : 0;
        if (OUT) {
            if (ONE || !LATER || h == 0) {
                la.issue(base_a + first * f.a_stride + h * d, f.a_stride, rows, d);
                if (DOTS) le.issue(base_e + first * f.e_stride + h * d, f.e_stride, rows, d);
            } else {
                la.drop();
                if (DOTS) le.drop();
            }
        }
        if (ONE || LATER || h == 0) {
            lb.issue(base_b + first * f.b_stride + h * d, f.b_stride, rows, d);
            lc.issue(base_c + first * f.c_stride + h * d, f.c_stride, rows, d);
        } else {
            lb.drop();
            lc.drop();
        }
        if (ONE || h == 0) next_g = lane < rows ? base_g[(first + lane) * p.decay_stride] : 0.f;
    };
    if (chunks > 0) issue(0, 0);
    for (int n = 0; n < chunks; ++n) {
        const int chunk = LATER ? chunks - 1 - n : n;
        const int first = chunk * kLinearChunk;
        f32x16 out_of_heads[2];            // LATER: summed over the heads
        float chunk_decay = 0.f;
        for (int h = 0; h < group; ++h) {
            f32x16 out_of_head[2];
            f32x16 (&out)[2] = LATER ? out_of_heads : out_of_head;
            const bool first_head = h == 0, last_head = h == group - 1;
            int t32 = lane & 31;
            asm volatile("" : "+v"(t32));      // (as reads.fresh(): or the mask of every hidden pair is kept in registers)
            reads.fresh();
            if (OUT && (!LATER || first_head)) {
                la.put(tile_a);
                if (DOTS) le.put(tile_e);
            }
            if (LATER || first_head) {
                lb.put(tile_b);
                lc.put(tile_c);
            }
            if (first_head) {
                const float g = lane < seg.rows - first ? decay_log2(next_g) : 0.f;
                const float sum = sum_up_to(g, lane);
                chunk_decay = __shfl(sum, 63, 64);
                if (wave == 0) {
                    const float from_start = fast_exp2(sum), to_end = fast_exp2(chunk_decay - sum);
                    sums[lane] = sum;
                    in_weight[lane] = f.scale_in * (LATER ? to_end : from_start);
                    out_weight[lane] = f.scale_state * (LATER ? from_start : to_end);
                }
            }
            __syncthreads();
            if constexpr (OUT) {
                // pairs of sources (along the rows) and targets (along the lanes): of the four blocks of 32 x 32, the three that are not all hidden
#pragma unroll 1
                for (int blk = wave; blk < 3; blk += kWaves) {
                    const int sb = LATER ? (blk > 0) : blk >> 1, tb = LATER ? blk >> 1 : (blk > 0);
                    f32x16 w{};
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)
                        w = mfma(reads.along(tile_b, sb, kk), reads.along(tile_a, tb, kk), w);
                    f32x16 y{};
                    if constexpr (DOTS) {
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk)
                            y = mfma(reads.along(tile_c, sb, kk), reads.along(tile_e, tb, kk), y);
                    }
                    const float target_sum = sums[tb * 32 + t32];
                    float dot = 0.f;
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const f32x4 source_sum = *reinterpret_cast<const f32x4*>(sums + sb * 32 + 8 * i4 + 4 * hh);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int i = 4 * i4 + j, s = 8 * i4 + 4 * hh + j;
                            const float gap = LATER ? source_sum[j] - target_sum : target_sum - source_sum[j];
                            const bool hidden = sb == tb && (LATER ? s < t32 : s > t32);
                            w[i] = hidden ? 0.f : w[i] * (p.scale * fast_exp2(gap));
                            if constexpr (DOTS) dot += hidden || (sb == tb && s == t32) ? 0.f : w[i] * y[i];
                        }
                    }
                    if constexpr (DOTS) {
                        dot += partner32(dot);
                        if (lane < 32) near[blk * 32 + lane] = LATER && !first_head ? near[blk * 32 + lane] + dot : dot;
                    }
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt) {
                        float x[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = w[8 * tt + i];
                        const TwoParts parts = two_parts(x);
                        char* const at = lds + L::kP + (blk * 4 + tt * 2) * 1024 + lane * 16;
                        *reinterpret_cast<bf16x8*>(at) = parts.hi;
                        *reinterpret_cast<bf16x8*>(at + 1024) = parts.lo;
                    }
                }
                // what the state gives to the targets; the state goes into the product in two parts
                if (has_columns && (!LATER || first_head)) {
                    out[0] = out[1] = f32x16{};
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        float x[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = S.x[kk / 2][8 * (kk % 2) + i];
                        const TwoParts parts = two_parts(x);
#pragma unroll
                        for (int tb = 0; tb < 2; ++tb) {
                            const bf16x8 a = reads.along(tile_a, tb, kk);
                            out[tb] = mfma(parts.hi, a, out[tb]);
                            out[tb] = mfma(parts.lo, a, out[tb]);
                        }
                    }
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb) {
                        const float weight = in_weight[tb * 32 + t32];
                        float dot = 0.f;
#pragma unroll
                        for (int i4 = 0; i4 < 4; ++i4) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) out[tb][4 * i4 + j] *= weight;
                            if constexpr (DOTS) {
                                const u32x2 e = *reinterpret_cast<const u32x2*>(tile_e + tile_offset<D>(tb * 32 + t32, wave * 32 + 8 * i4 + 4 * hh));
                                dot += out[tb][4 * i4] * __uint_as_float(e[0] << 16) + out[tb][4 * i4 + 1] * __uint_as_float(e[0] & 0xffff0000u) +
                                       out[tb][4 * i4 + 2] * __uint_as_float(e[1] << 16) + out[tb][4 * i4 + 3] * __uint_as_float(e[1] & 0xffff0000u);
                            }
                        }
                        if constexpr (DOTS) {
                            dot += partner32(dot);
                            if (lane < 32) far[wave * kLinearChunk + tb * 32 + lane] = dot;
                        }
                    }
                }
                __syncthreads();
            }

            bf16x8 sources[4];     // c, 16 sources at a time down the operand's k
            if (has_columns) {
#pragma unroll
                for (int t = 0; t < 4; ++t) sources[t] = reads.down(tile_c, wave, t);
                if constexpr (OUT) {
                    if (all_finite(sources)) add_own_chunk<D, LATER, true>(lds, sources, wave, lane, out);
                    else add_own_chunk<D, LATER, false>(lds, sources, wave, lane, out);
                    if (!LATER || last_head) {
                        const int target_head = LATER ? kv_head : kv_head * group + h;
#pragma unroll
                        for (int tb = 0; tb < 2; ++tb) {
                            const int row = first + tb * 32 + t32;
                            if (row < seg.rows) {
                                const int64_t at = ((int64_t)(seg.start + row) * target_heads + target_head) * d + wave * 32 + 4 * hh;
#pragma unroll
                                for (int i4 = 0; i4 < 4; ++i4)
                                    if (wave * 32 + 8 * i4 < d)
                                        store_grad4(f.out, at + 8 * i4, f.out_f32, out[tb][4 * i4], out[tb][4 * i4 + 1], out[tb][4 * i4 + 2], out[tb][4 * i4 + 3]);
                            }
                        }
                    }
                }
            }
            // the next tiles: behind the outputs, whose registers they take, and in front of the state's products, which hide some of their way
            if (h + 1 < group) issue(n, h + 1);
            else issue(n + 1, 0);
            if (has_columns) {
                if (LATER || last_head) {
                    if (!LATER || first_head) {
                        const float left = fast_exp2(chunk_decay);
#pragma unroll
                        for (int db = 0; db < D / 32; ++db)
#pragma unroll
                            for (int i = 0; i < 16; ++i) S.x[db][i] *= left;
                    }
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const f32x4 w0 = *reinterpret_cast<const f32x4*>(out_weight + 16 * t + 4 * hh);
                        const f32x4 w1 = *reinterpret_cast<const f32x4*>(out_weight + 16 * t + 8 + 4 * hh);
                        union { bf16x8 v; u32x4 u; } c;
                        c.v = sources[t];
                        float x[8];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            x[2 * i] = __uint_as_float(c.u[i] << 16) * (i < 2 ? w0[2 * i] : w1[2 * i - 4]);
                            x[2 * i + 1] = __uint_as_float(c.u[i] & 0xffff0000u) * (i < 2 ? w0[2 * i + 1] : w1[2 * i - 3]);
                        }
                        const TwoParts parts = two_parts(x);
#pragma unroll
                        for (int db = 0; db < D / 32; ++db) {
                            const bf16x8 rows = reads.down_ordered(tile_b, db, t);
                            S.x[db] = mfma(rows, parts.hi, S.x[db]);
                            S.x[db] = mfma(rows, parts.lo, S.x[db]);
                        }
                    }
                }
            }
            if constexpr (DOTS) {
                if (wave == 0 && (!LATER || last_head) && lane < seg.rows - first) {
                    const int target_head = LATER ? kv_head : kv_head * group + h;
                    const int64_t at = (int64_t)target_head * p.shape.total_rows + seg.start + first + lane;
                    // blocks 0 | 1, 2 of the pairs have targets 0 .. 31 | 32 .. 63, or (LATER) 0, 1 | 2
                    f.near[at] = LATER ? (lane < 32 ? near[lane] + near[32 + lane] : near[32 + lane])
                                       : (lane < 32 ? near[lane] : near[lane] + near[32 + lane]);
                    float sum = 0.f;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) sum += w * 32 < d ? far[w * kLinearChunk + lane] : 0.f;
                    f.far[at] = sum;
                }
            }
            __syncthreads();
        }
        all_decay += chunk_decay;
    }
    return all_decay;
}

// the state at a segment's start (LATER: the gradient at its end) as it lies in memory; NULL: zeros.  *bad: it is one that does not exist
template <bool LATER>
__device__ __forceinline__ const float* reaching_state(const LinearParams& p, const Segment& seg, int kv_head, bool* bad) {
    const int d = p.shape.head_dim;
    *bad = false;
    if (seg.count > 1) return (LATER ? p.d_states : p.states) + ((int64_t)(seg.entry + seg.index) * p.shape.kv_heads + kv_head) * d * d;
    bool exists;
    const float* m = state_of(LATER ? p.final : p.initial, seg.seq, kv_head, d, &exists);
    *bad = exists && m == nullptr;
    return m;
}

template <int D, bool LATER, bool DOTS, bool ONE>
__device__ __forceinline__ void outputs_of(const LinearParams& p, const Routine& f, const Segment& seg, int slot, int kv_head, char* lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), d = p.shape.head_dim;
    State<D> S;
    bool bad;
    const float* const from = reaching_state<LATER>(p, seg, kv_head, &bad);
    if (from) S.load(from, d, f.transposed, wave, lane);
    else S.clear(bad ? __builtin_nanf("") : 0.f);
    walk<D, LATER, true, DOTS, ONE>(p, f, seg, kv_head, lds, S);
    if (!LATER && DOTS) {
        // <S, dS> behind the segment's last token: what the gradient of its decays starts from
        const float* const d_end = reaching_state<true>(p, seg, kv_head, &bad);
        float sum = d_end ? wave_sum(S.dot(d_end, d, f.transposed, wave, lane)) : 0.f;
        float* const parts = reinterpret_cast<float*>(lds);
        if (lane == 0) parts[wave] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            sum = 0.f;
            for (int w = 0; w < D / 32; ++w) sum += parts[w];
            p.across[(int64_t)slot * p.shape.kv_heads + kv_head] = sum;
        }
    }
    if (!DOTS && !f.transposed) {
        float* to = nullptr;
        if (LATER) {
            if (seg.index == 0 && p.d_initial) to = p.d_initial + ((int64_t)seg.seq * p.shape.kv_heads + kv_head) * d * d;
        } else if (seg.index == seg.count - 1) {
            bool exists;
            to = state_of(p.final, seg.seq, kv_head, d, &exists);
        }
        if (to) S.store(to, d, wave, lane);
    }
}

// what a workgroup works on: item -> (role, KV head, slot), roles innermost
__device__ __forceinline__ bool item_of_block(const LinearShape& shape, int roles, int& role, int& kv_head, int& slot) {
    const int64_t items = (int64_t)shape.slots * shape.kv_heads * roles, item = linear_item(blockIdx.x, items);
    if ((int64_t)blockIdx.x / 8 >= linear_share(items) || item >= items) return false;
    role = (int)(item % roles);
    kv_head = (int)(item / roles % shape.kv_heads);
    slot = (int)(item / roles / shape.kv_heads);
    return true;
}

__device__ __forceinline__ Routine forward_routine(const LinearParams& p) {
    return Routine{p.q, p.k, p.v, nullptr, p.q_stride, p.kv_stride, p.kv_stride, 0, p.scale, 1.f, p.o, false, false, nullptr, nullptr};
}
__device__ __forceinline__ Routine dq_routine(const LinearParams& p) {
    return Routine{p.d_o, p.v, p.k, p.q, p.do_stride, p.kv_stride, p.kv_stride, p.q_stride, p.scale, 1.f, p.dq, p.grad_f32 != 0, true, p.q_near, p.q_far};
}
__device__ __forceinline__ Routine dk_routine(const LinearParams& p) {
    return Routine{p.v, p.d_o, p.q, p.k, p.kv_stride, p.do_stride, p.q_stride, p.kv_stride, 1.f, p.scale, p.dk, p.grad_f32 != 0, true, p.k_near, p.k_far};
}
__device__ __forceinline__ Routine dv_routine(const LinearParams& p) {
    return Routine{p.k, p.q, p.d_o, nullptr, p.kv_stride, p.q_stride, p.do_stride, 0, 1.f, p.scale, p.dv, p.grad_f32 != 0, false, nullptr, nullptr};
}

template <int D, bool ONE>
__global__ __launch_bounds__(D / 32 * 64, 2) void linear_fwd_kernel(LinearParams p) {
    __shared__ __align__(16) char lds[Lds<D>::bytes(true, false)];
    int role, kv_head, slot;
    Segment seg;
    if (!item_of_block(p.shape, 1, role, kv_head, slot) || !find_segment(p.shape, slot, seg)) return;
    outputs_of<D, false, false, ONE>(p, forward_routine(p), seg, slot, kv_head, lds);
}

template <int D, bool ONE>
__global__ __launch_bounds__(D / 32 * 64, 2) void linear_bwd_kernel(LinearParams p) {
    __shared__ __align__(16) char lds[Lds<D>::bytes(true, true)];
    int role, kv_head, slot;
    Segment seg;
    if (!item_of_block(p.shape, 3, role, kv_head, slot) || !find_segment(p.shape, slot, seg)) return;
    if (role == 0) outputs_of<D, false, true, ONE>(p, dq_routine(p), seg, slot, kv_head, lds);
    else if (role == 1) outputs_of<D, true, true, ONE>(p, dk_routine(p), seg, slot, kv_head, lds);
    else outputs_of<D, true, false, ONE>(p, dv_routine(p), seg, slot, kv_head, lds);
}

// What a segment adds to the state, into the entry of the segment that it reaches next; `roles` 2: also what it adds to the gradient.
template <int D>
__global__ __launch_bounds__(D / 32 * 64, 2) void linear_state_kernel(LinearParams p, int roles) {
    __shared__ __align__(16) char lds[Lds<D>::bytes(false, false)];
    int role, kv_head, slot;
    Segment seg;
    if (!item_of_block(p.shape, roles, role, kv_head, slot) || !find_segment(p.shape, slot, seg) || seg.count == 1) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), d = p.shape.head_dim;
    const bool last = seg.index == seg.count - 1;
    if (role == 0 ? last : seg.index == 0) return;
    State<D> S;
    S.clear(0.f);
    const float decay = role == 0 ? walk<D, false, false, false, true>(p, forward_routine(p), seg, kv_head, lds, S)
                                  : walk<D, true, false, false, false>(p, dv_routine(p), seg, kv_head, lds, S);
    const int64_t own = (int64_t)(seg.entry + seg.index) * p.shape.kv_heads + kv_head;
    float* const to = role == 0 ? p.states + (own + p.shape.kv_heads) * d * d : p.d_states + (own - p.shape.kv_heads) * d * d;
    S.store(to, d, wave, lane);
    if (threadIdx.x == 0 && (role == 0 || last)) p.seg_decay[own] = decay;
}

// Passes states from segment to segment, elementwise: entry b holds what segment b - 1 adds and receives the state at the start of segment b.
// blockIdx.y: 0 states, forwards; 1 their gradients, backwards.
constexpr int kPassThreads = 256;
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
    for (int i = 1; i < count; ++i) {
        const int to = later ? count - 1 - i : i, over = later ? to + 1 : i - 1;     // the entry, and the segment that is passed over
        f32x4* const at = reinterpret_cast<f32x4*>(base + to * step);
        s = s * fast_exp2(decay[(int64_t)over * sh.kv_heads]) + *at;
        *at = s;
    }
}

// Gradients of the log decays, one wave per segment and KV head, from its last chunk to its first.  g_t weighs every pair of a token from t on
// and one before t.  Of these pairs, a chunk's own and those with a token on one side of the chunk come from the dot products;
// those across the whole chunk, <e^{G_L} S, R>, are what is left of <S, dS> at its end without its own keys.
__global__ __launch_bounds__(64) void linear_decay_kernel(LinearParams p) {
    const LinearShape& sh = p.shape;
    int role, kv_head, slot;
    if (!item_of_block(sh, 1, role, kv_head, slot)) return;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)slot * sh.kv_heads + kv_head;
    const bool fixed = p.decay_stride == 0;
    Segment seg;
    if (!find_segment(sh, slot, seg)) {
        if (fixed && lane == 0) p.decay_sums[item] = 0.f;
        return;
    }
    float across = p.across[item], total = 0.f;
    for (int chunk = (seg.rows + kLinearChunk - 1) / kLinearChunk - 1; chunk >= 0; --chunk) {
        const int64_t row = seg.start + chunk * kLinearChunk + lane;
        const bool there = chunk * kLinearChunk + lane < seg.rows;
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
        const float all_k = wave_sum(far_k);
        // (a decay that leaves nothing leaves no pairs across it either, not even rounding errors)
        const float whole = fast_exp2(wave_sum(g)) == 0.f ? 0.f : across - all_k;
        const float later = sum_from(near + far_q, lane);
        const float grad = later + (sum_up_to(far_k, lane) - far_k) + whole;
        if (there) {
            if (fixed) total += grad;
            else p.d_log_decay[row * sh.kv_heads + kv_head] = grad;
        }
        across = whole + wave_sum(far_q);
    }
    if (fixed) {
        total = wave_sum(total);
        if (lane == 0) p.decay_sums[item] = total;
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

unsigned grid_of(const LinearParams& p, int roles) { return (unsigned)(8 * linear_share((int64_t)p.shape.slots * p.shape.kv_heads * roles)); }

template <int D>
void launch_states(const LinearParams& p, int roles, hipStream_t stream) {
    if (p.shape.seg_rows == 0) return;
    linear_state_kernel<D><<<grid_of(p, roles), D / 32 * 64, 0, stream>>>(p, roles);
    const int d = p.shape.head_dim, parts = (d * d / 4 + kPassThreads - 1) / kPassThreads;
    linear_pass_kernel<<<dim3((unsigned)((int64_t)p.shape.windows * p.shape.kv_heads * parts), roles), kPassThreads, 0, stream>>>(p, parts);
}

template <int D>
void launch_fwd(const LinearParams& p, hipStream_t stream) {
    launch_states<D>(p, 1, stream);
    const auto kernel = p.shape.group == 1 ? linear_fwd_kernel<D, true> : linear_fwd_kernel<D, false>;
    kernel<<<grid_of(p, 1), D / 32 * 64, 0, stream>>>(p);
}
template <int D>
void launch_bwd(const LinearParams& p, hipStream_t stream) {
    launch_states<D>(p, 2, stream);
    const auto kernel = p.shape.group == 1 ? linear_bwd_kernel<D, true> : linear_bwd_kernel<D, false>;
    kernel<<<grid_of(p, 3), D / 32 * 64, 0, stream>>>(p);
}

}  // namespace

LinearSizes linear_sizes(int32_t total_rows, int32_t num_seqs, int32_t max_rows, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                         bool backward) {
    LinearSizes s{};
    const int64_t longest = max_rows > 0 && max_rows < total_rows ? max_rows : total_rows;
    int64_t seg = ((int64_t)total_rows * kv_heads / 768 + kLinearChunk - 1) / kLinearChunk * kLinearChunk;
    seg = seg < 256 ? 256 : seg > 4096 ? 4096 : seg;
    s.seg_rows = longest <= seg ? 0 : (int32_t)seg;
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
    s.slot_bytes = rounded(s.slots * kv_heads * 4);
    return s;
}

hipError_t launch_linear_fwd(const LinearParams& p, hipStream_t stream) {
    if (p.shape.slots > 0) p.shape.head_dim <= 64 ? launch_fwd<64>(p, stream) : launch_fwd<128>(p, stream);
    return hipGetLastError();
}

hipError_t launch_linear_bwd(const LinearParams& p, hipStream_t stream) {
    if (p.shape.slots > 0) p.shape.head_dim <= 64 ? launch_bwd<64>(p, stream) : launch_bwd<128>(p, stream);
    if (p.d_log_decay) {
        if (p.shape.slots > 0) linear_decay_kernel<<<grid_of(p, 1), 64, 0, stream>>>(p);
        if (p.decay_stride == 0) linear_decay_sum_kernel<<<(unsigned)p.shape.kv_heads, 256, 0, stream>>>(p);
    }
    return hipGetLastError();
}

}  // namespace hspmd
