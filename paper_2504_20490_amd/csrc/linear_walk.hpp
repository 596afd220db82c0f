// Linear attention with a decay for each head, chunked form: the routine of the forward and of the backward.
//
// Per sequence and KV head, with G the running sum of the log decays from a chunk's start, S the state at that start and s the scale:
//   o_t  = s e^{G_t} S^T q_t + s sum_{j <= t} e^{G_t - G_j} <q_t, k_j> v_j,      S' = e^{G_L} S + sum_j e^{G_L - G_j} k_j v_j^T.
// The gradients are the same form with other tensors: dq looks backwards like o (targets dO, sources v and k, the transposed state),
// dk and dv look forwards (targets v and k, sources dO, q and q, dO) with R, the gradient of the state at the chunk's end:
//   dk_t = e^{G_L - G_t} R v_t + s sum_{i >= t} e^{G_i - G_t} <v_t, dO_i> q_i,    R' = e^{G_L} R + s sum_i e^{G_i} q_i dO_i^T.
// So one routine does all four: targets a, sources b and c, state sum b c^T.
//
// Chunks of 64 tokens: per token the pairs cost 64 columns of products, the state 2 x 128, and making the state ready for the products (three operations per
// element, its parts) is shared by 64 targets; with two workgroups per compute unit their tiles fit LDS (62 KB forward, 80 KB backward).
// The state stays in registers: a wave holds 32 of its columns, 64 registers at head_dim 128, and everything it multiplies comes from LDS.
// What bounds it: memory in the forward (512 sequences of 1024 tokens, head_dim 128: 130 us, 4.1 TB/s; loads and stores alone 113 us, products
// alone 92), the chip's power in the backward (24 heads, 32768 tokens: 934 us, 0.56 PFLOP/s of products in their parts at 1.5 to 1.75 GHz).
#pragma once
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
    bool transposed;         // the state is b c^T transposed to how it lies in memory
    float* near;             // DOTS: [heads][total_rows], see LinearParams
    float* far;
    float* anchors;          // DOTS: where the states of anchors go
};

// What a workgroup keeps in LDS.  WEIGHT_PARTS: bf16 values per weight of a pair; ONE: a KV head has one query head
template <int D, int WEIGHT_PARTS, bool ONE>
struct Lds {
    static constexpr int kWaves = D / 32;
    static constexpr int kTile = kLinearChunk * D * 2;
    static constexpr int kB = 0, kC = kTile;
    static constexpr int kSums = 2 * kTile;                   // running sums of the log decays in two parts, weights of targets and of sources, `passing`, two addresses
    static constexpr int kLater = kSums + (4 * kLinearChunk + 8) * 4;
    static constexpr int kA = kSums + (4 * kLinearChunk + 8) * 4 + 16;
    static constexpr int kWeights = kA + kTile;               // of pairs: [block][step of 16 sources][part][lane]
    // D = 128: with a third part the area would leave room for one workgroup per compute unit.  It goes where the tile of e was, behind the last use of
    // that (with several heads, which share the tile of a KV head, there is no such time)
    static constexpr bool kLate = D == 128 && WEIGHT_PARTS == 3 && ONE;
    static constexpr int kAreaParts = kLate ? 2 : WEIGHT_PARTS;
    static constexpr int kNear = kWeights + 3 * 2 * kAreaParts * 1024;
    static constexpr int kFar = kNear + 3 * 32 * 4;
    static constexpr int kE = kFar + kWaves * kLinearChunk * 4;
    static constexpr int bytes(bool out, bool dots) { return dots ? kE + kTile : out ? kNear : kA; }
    // where the weights of a block's step are, for lane 0
    static constexpr int weights(int blk, int step, int part) {
        return part < kAreaParts ? kWeights + ((blk * 2 + step) * kAreaParts + part) * 1024 : kE + (blk * 2 + step) * 1024;
    }
};

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Memory from an address on, for accesses with 32-bit offsets: one at kNowhere reads zeros and writes nothing.  So the loops below hold no branches
// around their loads and stores, and the compiler can wait for a load without waiting for the stores that follow it.
constexpr uint32_t kNowhere = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t whole_memory(const void* from) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(from), 0, 0x7fffffff, 0x00020000);
}

// A tile of a chunk's rows on its way from memory to LDS.  Rows behind the segment's end and columns behind head_dim read as zeros
// (an address outside the buffer resource), so that nothing behind a sequence ever meets a product.
template <int D>
struct TileLoad {
    static constexpr int kThreadsHere = D / 32 * 64, kRowsPerPass = kThreadsHere / (D / 8), kPasses = kLinearChunk / kRowsPerPass;
    u32x4 r[kPasses];
    __device__ __forceinline__ void issue(const uint16_t* first_row, int64_t token_stride, int rows, int head_dim) {
        int stride = (int)token_stride;
        asm volatile("" : "+s"(stride));      // (its multiples are made here, and not kept in scalar registers across the loop)
        const int row = threadIdx.x / (D / 8), col = threadIdx.x % (D / 8) * 8, there = col < head_dim ? rows : 0;
        const uint32_t off = (uint32_t)(row * stride + col) * 2u;
        const __amdgpu_buffer_rsrc_t rsrc = whole_memory(first_row);
#pragma unroll
        for (int i = 0; i < kPasses; ++i)
            r[i] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, row + i * kRowsPerPass < there ? off : kNowhere, i * kRowsPerPass * stride * 2, 0);
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

// The wave's 32 columns of a chunk's outputs: lane's token in a block of 32 along the columns of the accumulators, columns of the head along the rows.
// row_stride: elements
template <bool F32>
__device__ __forceinline__ void store_rows(void* base, int64_t first, const f32x16 (&out)[2], int row_stride, int rows, int d, int wave, int lane) {
    const __amdgpu_buffer_rsrc_t rsrc = whole_memory(static_cast<char*>(base) + first * (F32 ? 4 : 2));
    const int row = lane & 31, col = wave * 32 + 4 * (lane >> 5);
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
        const uint32_t off = row + tb * 32 < rows ? (uint32_t)((row + tb * 32) * row_stride + col) * (F32 ? 4u : 2u) : kNowhere;
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
            const f32x4 x = {out[tb][4 * i4], out[tb][4 * i4 + 1], out[tb][4 * i4 + 2], out[tb][4 * i4 + 3]};
            const uint32_t at = wave * 32 + 8 * i4 < d ? off + 8 * i4 * (F32 ? 4 : 2) : kNowhere;
            if constexpr (F32) {
                union { f32x4 f; u32x4 u; } y;
                y.f = x;
                __builtin_amdgcn_raw_buffer_store_b128(y.u, rsrc, at, 0, 0);
            } else {
                __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])}, rsrc, at, 0, 0);
            }
        }
    }
}

// The wave's part of a state: columns 32 wave .. + 31 (of c) along the lanes, all 32 NB rows (of b) in registers; register i of
// block db holds row 32 db + 16 (i / 8) + 8 (lane / 32) + i % 8.
template <int NB>
struct State {
    f32x16 x[NB];
    __device__ __forceinline__ void clear(float value) {
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[db][i] = value;
    }
    // as `in memory`: [row][col], or [col][row]
    __device__ __forceinline__ void load(const float* m, int d, bool transposed, int wave, int lane) {
        const int col = wave * 32 + (lane & 31);
#pragma unroll
        for (int db = 0; db < NB; ++db)
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
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = db * 32 + h * 16 + (lane >> 5) * 8;
                if (row < d && col < d) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) m[(row + i) * d + col] = x[db][8 * h + i];
                }
            }
    }
    // 2^log2 times it as it lies in the registers, without the rows that nothing of head_dim is in
    __device__ __forceinline__ void keep(float* m, int d, float log2, int wave, int lane) const {
        const float by = fast_exp2(log2);
        const __amdgpu_buffer_rsrc_t rsrc = whole_memory(m + wave * ((d + 15) / 16 * 16 * 32));
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                union { f32x4 f; u32x4 u; } y;
                y.f = f32x4{x[db][i] * by, x[db][i + 1] * by, x[db][i + 2] * by, x[db][i + 3] * by};
                // (with its offset in a scalar register the store would read what the next instructions leave in y's registers: the compiler takes it to need no room)
                if (db * 32 + i / 8 * 16 < d) __builtin_amdgcn_raw_buffer_store_b128(y.u, rsrc, lane * 16 + (db * 16 + i) * 256, 0, 0);
                __builtin_amdgcn_sched_barrier(0);      // (one at a time: else the products take registers that are not there)
            }
    }
    // this lane's share of the sum over all elements of this state times the one in memory, which is its transpose
    __device__ __forceinline__ float dot_transposed(const float* m, int d, int wave, int lane) const {
        const __amdgpu_buffer_rsrc_t rsrc = whole_memory(m);
        const int col = wave * 32 + (lane & 31), row = (lane >> 5) * 8;
        float sum = 0.f;
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int at = row + db * 32 + i / 8 * 16 + i % 8;
                union { u32x4 u; f32x4 f; } y;
                y.u = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at < d && col < d ? (uint32_t)(col * d + at) * 4u : kNowhere, 0, 0);
                // (a state's columns behind head_dim may hold NaN, of weights that are)
                const float part = x[db][i] * y.f[0] + x[db][i + 1] * y.f[1] + x[db][i + 2] * y.f[2] + x[db][i + 3] * y.f[3];
                sum += at < d && col < d ? part : 0.f;
            }
        return sum;
    }
};

// A hidden pair has the weight 0, and 0 times an infinity or NaN is NaN: sources that hold one are left out of the products, element by element, and
// added for the targets that see them.
__device__ __forceinline__ bool all_finite(const bf16x8 (&x)[4], const PairOps& ops) {
    float zero[2] = {0.f, 0.f};              // 0 times an infinity or NaN is NaN
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        union { bf16x8 v; u32x4 u; } c;
        c.v = x[t];
#pragma unroll
        for (int i = 0; i < 4; ++i) zero[i % 2] = PairOps::dot(c.u[i], ops.none, zero[i % 2]);
    }
    return !__any(zero[0] + zero[1] != 0.f);
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

// What the sources of the own chunk give: parts FIRST .. LAST of the weights times c, (source block, target block) of 32 x 32 pairs by their number, see walk
template <int D, bool LATER, bool ONE, int WEIGHT_PARTS, int FIRST, int LAST>
__device__ __forceinline__ void add_own_chunk(const char* lds, const bf16x8 (&sources)[4], int lane, f32x16 (&out)[2]) {
    using L = Lds<D, WEIGHT_PARTS, ONE>;
#pragma unroll
    for (int part = FIRST; part <= LAST; ++part)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int blk = 0; blk < 3; ++blk) {
                const int sb = LATER ? (blk > 0) : blk >> 1, tb = LATER ? blk >> 1 : (blk > 0);
                out[tb] = mfma(sources[2 * sb + tt], *reinterpret_cast<const bf16x8*>(lds + L::weights(blk, tt, part) + lane * 16), out[tb]);
            }
}
template <int D, bool LATER, bool ONE, int WEIGHT_PARTS>
__device__ __forceinline__ void add_not_finite(const char* lds, int wave, int lane, f32x16 (&out)[2]) {
    using L = Lds<D, WEIGHT_PARTS, ONE>;
    const char* const tile = lds + L::kC;
    const int t32 = lane & 31, hh = lane >> 5;
#pragma unroll 1
    for (int s = 0; s < kLinearChunk; ++s) {
        const int sb = s / 32, r = s % 32;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            if (LATER ? sb < tb : sb > tb) continue;
            const bool sees = sb != tb || (LATER ? r >= t32 : r <= t32);
            // the weight of (s, t32) as it was laid out for the products: lane 32 (r / 4 % 2) + t32, element 4 (r / 8 % 2) + r % 4 of step r / 16
            const int at = (32 * (r / 4 % 2) + t32) * 16 + (4 * (r / 8 % 2) + r % 4) * 2;
            float weight = 0.f;
#pragma unroll
            for (int part = 0; part < WEIGHT_PARTS; ++part) weight += (float)*reinterpret_cast<const __bf16*>(lds + L::weights(sb + tb, r / 16, part) + at);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int col = wave * 32 + 8 * (i / 4) + 4 * hh + i % 4;
                const uint32_t raw = *reinterpret_cast<const uint16_t*>(tile + tile_offset<D>(s, col & ~3) + (col & 3) * 2);
                if (sees && (raw & 0x7f80) == 0x7f80) out[tb][i] += weight * __uint_as_float(raw << 16);
            }
        }
    }
}

// The state is held as 2^held times what the registers hold, and multiplied out when that leaves 2^-16 .. 2^16: decays near 1 cost no operation per element
// and chunk.  (false for NaN, which is multiplied out into the state)
__device__ __forceinline__ bool can_hold(float log2) { return __builtin_fabsf(log2) <= 16.f; }

// Walks a segment's chunks, forwards or (LATER) backwards, with the state that reaches it in `S`.
//   LATER   targets see the tokens from themselves on, and a KV head's sources are those of all its query heads (dk, dv); else they see the
//           tokens up to themselves, and a KV head's targets are those of all its query heads (o, dq)
//   OUT     outputs are wanted, not only the state
//   DOTS    the dot products of the output with the tensor it is the gradient of, the part from the own chunk (without the token's own) and
//           the part from the state apart
//   ONE     a KV head has one query head
//   NB      blocks of 32 columns that head_dim takes; steps, and waves, that would compute on columns behind them pass
//   PARTS, WEIGHT_PARTS   bf16 values that the state and its sources, and the weights of pairs, enter products as; three of the weights go with
//           fp32 outputs, two with bf16
// Returns the log2 of the segment's decay, to the last wave and without OUT.
template <int D, bool LATER, bool OUT, bool DOTS, bool ONE, int PARTS, int WEIGHT_PARTS, int NB>
__device__ __forceinline__ float walk(const LinearParams& p, const Routine& f, const Segment& seg, int kv_head, char* lds, State<NB>& S) {
    constexpr bool OUT_F32 = WEIGHT_PARTS == 3;
    using L = Lds<D, WEIGHT_PARTS, ONE>;
    constexpr int kWaves = L::kWaves;
    constexpr bool kEarly = !DOTS || ONE;      // when the next tiles are loaded: four of them, beside outputs kept over several heads, are too many
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int d = p.shape.head_dim, group = ONE ? 1 : p.shape.group;
    const bool mine = NB == kWaves || wave < NB;      // this wave has columns
    const int hh = lane >> 5, token = LATER ? 63 - lane : lane;      // whose decay the lane has
    TileReads<D> reads;
    reads.init(lane);
    PairOps ops;
    ops.init();
    char* const tile_a = lds + L::kA;
    char* const tile_b = lds + L::kB;
    char* const tile_c = lds + L::kC;
    char* const tile_e = lds + L::kE;
    float* const sums = reinterpret_cast<float*>(lds + L::kSums);
    float* const rests = sums + kLinearChunk;
    float* const in_weight = rests + kLinearChunk;
    float* const out_weight = in_weight + kLinearChunk;
    // What goes with the state from chunk to chunk, here so that it takes no registers in the loop.  0, 1: log2 of what the state is held as behind the chunk, in two parts;
    // 2: the same in front of it; 3: what the state's registers are multiplied by; 4: the sum of 0 and 1
    float* const passing = out_weight + kLinearChunk;
    float* const near = reinterpret_cast<float*>(lds + L::kNear);
    float* const far = reinterpret_cast<float*>(lds + L::kFar);

    const int chunks = (seg.rows + kLinearChunk - 1) / kLinearChunk;
    const int target_heads = LATER ? p.shape.kv_heads : p.shape.q_heads;
    float all_decay = 0.f, all_decay_rest = 0.f;

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
        next_g = 0.f;
        if (ONE || h == 0)
            next_g = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(whole_memory(base_g + first * p.decay_stride),
                                                                          token < rows ? (uint32_t)(token * (int)p.decay_stride * 4) : kNowhere, 0, 0));
    };
    auto issue_next = [&](int n, int h) {
        if (h + 1 < group) issue(n, h + 1);
        else issue(n + 1, 0);
    };
    if (chunks > 0) issue(0, 0);
    for (int n = 0; n < chunks; ++n) {
        const int chunk = LATER ? chunks - 1 - n : n;
        const int first = chunk * kLinearChunk;
        if (wave == kWaves - 1) {        // (of four waves the one without a block of pairs)
            // LATER: the sums are those of the tokens behind each, from the chunk's end on, so that a decay that is NaN reaches the tokens it decays alone
            const bool there = token < seg.rows - first;
            const DecayLog2 g = split_decay_log2(next_g);
            const float upto = sum_up_to(there ? g.whole : 0.f), upto_rest = sum_up_to(there ? g.rest : 0.f);
            const float all = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(upto), 63));
            const float all_rest = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(upto_rest), 63));
            const float sum = LATER ? -lane_before(upto) : upto, rest = LATER ? -lane_before(upto_rest) : upto_rest;
            const float held = n > 0 ? passing[0] : 0.f, held_rest = n > 0 ? passing[1] : 0.f;
            const bool holds = can_hold(held + all);
            const float left = holds ? held + all : 0.f, left_rest = holds ? held_rest + all_rest : 0.f;
            const float in = LATER ? (held - sum) + (held_rest - rest) : (held + sum) + (held_rest + rest);
            const float out = LATER ? (all + sum - left) + (all_rest + rest - left_rest) : (all - sum - left) + (all_rest - rest - left_rest);
            sums[token] = sum;
            rests[token] = rest;
            in_weight[token] = f.scale_in * fast_exp2(in);
            out_weight[token] = f.scale_state * fast_exp2(out);
            if (lane == 0) {
                passing[0] = left, passing[1] = left_rest, passing[2] = held + held_rest, passing[4] = left + left_rest;
                passing[3] = holds ? 1.f : fast_exp2((held + all) + (held_rest + all_rest));
            }
            if (!OUT) all_decay += all, all_decay_rest += all_rest;
        }
        // tiles of the chunk; those of a head follow in the loop over them
        if (LATER && OUT) {
            la.put(tile_a);
            if (DOTS) le.put(tile_e);
        }
        if (!LATER) {
            lb.put(tile_b);
            lc.put(tile_c);
        }
        f32x16 out_of_heads[2];            // LATER: summed over the heads
        for (int h = 0; h < group; ++h) {
            f32x16 out_of_head[2];
            f32x16 (&out)[2] = LATER ? out_of_heads : out_of_head;
            const bool first_head = h == 0, last_head = h == group - 1;
            int t32 = lane & 31;
            asm volatile("" : "+v"(t32));      // (as reads.fresh(): or the mask of every hidden pair is kept in registers)
            reads.fresh();
            if (!LATER && OUT) {
                la.put(tile_a);
                if (DOTS) le.put(tile_e);
            }
            if (LATER) {
                lb.put(tile_b);
                lc.put(tile_c);
            }
            __syncthreads();
            if constexpr (DOTS) {
                // the state in front of this chunk (LATER: behind it), for the gradients of the decays
                if (first_head && mine && linear_is_anchor(chunk, chunks))
                    S.keep(f.anchors + ((int64_t)linear_anchor(seg.start, chunk, chunks) * p.shape.kv_heads + kv_head) * linear_anchor_elements(d), d, passing[2], wave, lane);
            }
            if (!OUT) issue_next(n, h);
            if constexpr (OUT) {
                bf16x8 late[2];        // (kLate: a wave has one block at most)
                // pairs of sources (along the rows) and targets (along the lanes): of the four blocks of 32 x 32, the three that are not all hidden
#pragma unroll 1
                for (int blk = wave; blk < 3; blk += kWaves) {
                    const int sb = LATER ? (blk > 0) : blk >> 1, tb = LATER ? blk >> 1 : (blk > 0);
                    f32x16 w{};
#pragma unroll
                    for (int kk = 0; kk < 2 * NB; ++kk) w = mfma(reads.along(tile_b, sb, kk), reads.along(tile_a, tb, kk), w);
                    f32x16 y{};
                    if constexpr (DOTS) {
#pragma unroll
                        for (int kk = 0; kk < 2 * NB; ++kk) y = mfma(reads.along(tile_c, sb, kk), reads.along(tile_e, tb, kk), y);
                    }
                    const float target_sum = LATER ? sums[tb * 32 + t32] - p.scale_log2.whole : sums[tb * 32 + t32] + p.scale_log2.whole;
                    const float target_rest = LATER ? rests[tb * 32 + t32] - p.scale_log2.rest : rests[tb * 32 + t32] + p.scale_log2.rest;
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const f32x4 source_sum = *reinterpret_cast<const f32x4*>(sums + sb * 32 + 8 * i4 + 4 * hh);
                        const f32x4 source_rest = *reinterpret_cast<const f32x4*>(rests + sb * 32 + 8 * i4 + 4 * hh);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float between = LATER ? source_sum[j] - target_sum : target_sum - source_sum[j];
                            w[4 * i4 + j] *= fast_exp2(between + (LATER ? source_rest[j] - target_rest : target_rest - source_rest[j]));
                        }
                        if (!kEarly) __builtin_amdgcn_sched_barrier(0);     // (or the sums of all sources are read at once, into registers that are not there)
                    }
                    if (sb == tb) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int s = 8 * (i / 4) + 4 * hh + i % 4;
                            w[i] = (LATER ? s < t32 : s > t32) ? 0.f : w[i];
                            if constexpr (DOTS) y[i] = (LATER ? s <= t32 : s >= t32) ? 0.f : y[i];
                        }
                    }
                    if constexpr (DOTS) {
                        float dot = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) dot += w[i] * y[i];
                        dot += partner32(dot);
                        if (lane < 32) near[blk * 32 + lane] = LATER && !first_head ? near[blk * 32 + lane] + dot : dot;
                    }
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt) {
                        Parts<WEIGHT_PARTS> parts;
                        f32x8 x;
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = w[8 * tt + i];
                        parts.of(x, ops);
#pragma unroll
                        for (int part = 0; part < L::kAreaParts; ++part)
                            *reinterpret_cast<bf16x8*>(lds + L::weights(0, tt, part) + blk * (2 * L::kAreaParts * 1024) + lane * 16) = parts.part[part];
                        if constexpr (L::kLate) late[tt] = parts.part[2];
                    }
                }
                if (kEarly) issue_next(n, h);      // (in front of the pairs they would take registers that these need)
                // what the state gives to the targets
                if (!LATER || first_head) {
                    __builtin_amdgcn_s_setprio(1);     // (products before the other workgroup's vector operations)
                    out[0] = out[1] = f32x16{};
                    if (mine) {
#pragma unroll
                        for (int kk = 0; kk < 2 * NB; ++kk) {
                            Parts<PARTS> parts;
                            f32x8 x;
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[i] = S.x[kk / 2][8 * (kk % 2) + i];
                            parts.template of<true>(x, ops);       // (the state's last products are two barriers behind)
                            const bf16x8 a[2] = {reads.along(tile_a, 0, kk), reads.along(tile_a, 1, kk)};
#pragma unroll
                            for (int part = 0; part < PARTS; ++part)
#pragma unroll
                                for (int tb = 0; tb < 2; ++tb) out[tb] = mfma(parts.part[part], a[tb], out[tb]);
                        }
                    }
                    __builtin_amdgcn_s_setprio(0);
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
                if constexpr (L::kLate) {
                    if (wave < 3) {
#pragma unroll
                        for (int tt = 0; tt < 2; ++tt) *reinterpret_cast<bf16x8*>(lds + L::weights(0, tt, 2) + wave * 2048 + lane * 16) = late[tt];
                    }
                }
            }
            if constexpr (OUT) {
                bf16x8 sources[4];     // c, 16 sources at a time down the operand's k
                bool finite = true;
                if (mine) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) sources[t] = reads.down(tile_c, wave, t);
                    finite = all_finite(sources, ops);
                    if (!finite) {
#pragma unroll
                        for (int t = 0; t < 4; ++t) sources[t] = finite_part(sources[t]);
                    }
                    add_own_chunk<D, LATER, ONE, WEIGHT_PARTS, 0, L::kAreaParts - 1>(lds, sources, lane, out);
                }
                if constexpr (L::kLate) {
                    __syncthreads();
                    if (mine) add_own_chunk<D, LATER, ONE, WEIGHT_PARTS, 2, 2>(lds, sources, lane, out);
                }
                if (!finite) add_not_finite<D, LATER, ONE, WEIGHT_PARTS>(lds, wave, lane, out);
                if (!LATER || last_head) {
                    const int64_t at = (int64_t)(seg.start + first) * target_heads + (LATER ? kv_head : kv_head * group + h);
                    store_rows<OUT_F32>(f.out, at * d, out, target_heads * d, seg.rows - first, d, wave, lane);
                }
                if constexpr (DOTS) {
                    if (!LATER || last_head) {
                        const int64_t at = (int64_t)(LATER ? kv_head : kv_head * group + h) * p.shape.total_rows + seg.start + first;
                        // blocks 0 | 1, 2 of the pairs have targets 0 .. 31 | 32 .. 63, or (LATER) 0, 1 | 2
                        const float near_sum = LATER ? (lane < 32 ? near[lane] + near[32 + lane] : near[32 + lane])
                                                     : (lane < 32 ? near[lane] : near[lane] + near[32 + lane]);
                        float far_sum = 0.f;
#pragma unroll
                        for (int w = 0; w < kWaves; ++w) far_sum += far[w * kLinearChunk + lane];
                        const uint32_t off = wave == 0 && lane < seg.rows - first ? lane * 4 : kNowhere;
                        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(near_sum), whole_memory(f.near + at), off, 0, 0);
                        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(far_sum), whole_memory(f.far + at), off, 0, 0);
                    }
                }
            }
            if (OUT && !kEarly) issue_next(n, h);
            if (mine && (LATER || last_head)) {
                const float left = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(passing[3])));
                if ((!LATER || first_head) && left != 1.f) {
#pragma unroll
                    for (int db = 0; db < NB; ++db)
#pragma unroll
                        for (int i = 0; i < 16; ++i) S.x[db][i] *= left;
                }
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const f32x4 w0 = *reinterpret_cast<const f32x4*>(out_weight + 16 * t + 4 * hh);
                    const f32x4 w1 = *reinterpret_cast<const f32x4*>(out_weight + 16 * t + 8 + 4 * hh);
                    union { bf16x8 v; u32x4 u; } c;
                    c.v = reads.down(tile_c, wave, t);
                    f32x8 x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[2 * i] = __uint_as_float(c.u[i] << 16) * (i < 2 ? w0[2 * i] : w1[2 * i - 4]);
                        x[2 * i + 1] = __uint_as_float(c.u[i] & 0xffff0000u) * (i < 2 ? w0[2 * i + 1] : w1[2 * i - 3]);
                    }
                    Parts<PARTS> parts;
                    parts.of(x, ops);
                    bf16x8 rows[NB];
#pragma unroll
                    for (int db = 0; db < NB; ++db) rows[db] = reads.down_ordered(tile_b, db, t);
#pragma unroll
                    for (int part = 0; part < PARTS; ++part)
#pragma unroll
                        for (int db = 0; db < NB; ++db) S.x[db] = mfma(rows[db], parts.part[part], S.x[db]);
                }
                __builtin_amdgcn_s_setprio(0);
            }
            __syncthreads();
        }
    }
    if (chunks > 0 && passing[4] != 0.f) {
        const float left = fast_exp2(passing[4]);
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) S.x[db][i] *= left;
    }
    return all_decay + all_decay_rest;
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

template <int D, bool LATER, bool DOTS, bool ONE, int PARTS, int WEIGHT_PARTS, int NB>
__device__ __forceinline__ void outputs_of(const LinearParams& p, const Routine& f, const Segment& seg, int slot, int kv_head, char* lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), d = p.shape.head_dim;
    State<NB> S;
    bool bad;
    // <S, dS> behind the segment's last token, or (LATER) in front of the sequence's first: what the gradients of its decays start from.  Where the other state is and the
    // sum goes waits in LDS: in registers, it would cost the walk some
    uint64_t* const later = reinterpret_cast<uint64_t*>(lds + Lds<D, WEIGHT_PARTS, ONE>::kLater);
    if (DOTS && threadIdx.x == 0) {
        const float* other = nullptr;
        bad = false;
        if (!LATER || seg.index == 0) other = reaching_state<!LATER>(p, seg, kv_head, &bad);
        float* const to = p.across + ((LATER ? p.shape.slots : 0) + (int64_t)slot) * p.shape.kv_heads + kv_head;
        if (!other) *to = bad ? __builtin_nanf("") : 0.f;
        later[0] = reinterpret_cast<uint64_t>(other);
        later[1] = reinterpret_cast<uint64_t>(to);
    }
    const float* const from = reaching_state<LATER>(p, seg, kv_head, &bad);
    if (from) S.load(from, d, f.transposed, wave, lane);
    else S.clear(bad ? __builtin_nanf("") : 0.f);
    walk<D, LATER, true, DOTS, ONE, PARTS, WEIGHT_PARTS, NB>(p, f, seg, kv_head, lds, S);
    if (DOTS) {
        __syncthreads();
        const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)later[0]), high = __builtin_amdgcn_readfirstlane((uint32_t)(later[0] >> 32));
        const float* const other = reinterpret_cast<const float*>((uint64_t)high << 32 | low);
        if (other) {
            float* const parts = reinterpret_cast<float*>(lds);
            const float sum = wave_sum(S.dot_transposed(other, d, wave, lane));
            if (lane == 0) parts[wave] = sum;
            __syncthreads();
            if (threadIdx.x == 0) {
                float all = 0.f;
                for (int w = 0; w < D / 32; ++w) all += parts[w];
                *reinterpret_cast<float*>(later[1]) = all;
            }
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

// what a workgroup works on: item -> (role, KV head, slot), roles innermost.  LAST_FIRST: the last slots start first, whose keys and values the launch in
// front has read last
template <bool LAST_FIRST = false>
__device__ __forceinline__ bool item_of_block(const LinearShape& shape, int roles, int& role, int& kv_head, int& slot) {
    const int64_t items = (int64_t)shape.slots * shape.kv_heads * roles;
    int64_t item = linear_item(blockIdx.x, 4 * roles);
    if (item >= items) return false;
    if (LAST_FIRST) item = items - 1 - item;
    role = (int)(item % roles);
    kv_head = (int)(item / roles % shape.kv_heads);
    slot = (int)(item / roles / shape.kv_heads);
    return true;
}

__device__ __forceinline__ Routine forward_routine(const LinearParams& p) {
    return Routine{p.q, p.k, p.v, nullptr, p.q_stride, p.kv_stride, p.kv_stride, 0, p.scale, 1.f, p.o, false, nullptr, nullptr, nullptr};
}
__device__ __forceinline__ Routine dq_routine(const LinearParams& p) {
    return Routine{p.d_o, p.v, p.k, p.q, p.do_stride, p.kv_stride, p.kv_stride, p.q_stride, p.scale, 1.f, p.dq, true, p.q_near, p.q_far, p.anchors};
}
__device__ __forceinline__ Routine dk_routine(const LinearParams& p) {
    return Routine{p.v, p.d_o, p.q, p.k, p.kv_stride, p.do_stride, p.q_stride, p.kv_stride, 1.f, p.scale, p.dk, true, p.k_near, p.k_far, p.d_anchors};
}
__device__ __forceinline__ Routine dv_routine(const LinearParams& p) {
    return Routine{p.k, p.q, p.d_o, nullptr, p.kv_stride, p.q_stride, p.do_stride, 0, 1.f, p.scale, p.dv, false, nullptr, nullptr, nullptr};
}

// calls f(tile width, blocks of 32 columns, one query head per KV head) as constants
template <typename F>
void with_shape(const LinearShape& shape, F&& f) {
    using std::integral_constant;
    const auto heads = [&](auto d, auto blocks) { shape.group == 1 ? f(d, blocks, std::true_type{}) : f(d, blocks, std::false_type{}); };
    if (shape.head_dim <= 32) heads(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (shape.head_dim <= 64) heads(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (shape.head_dim <= 96) heads(integral_constant<int, 128>{}, integral_constant<int, 3>{});
    else heads(integral_constant<int, 128>{}, integral_constant<int, 4>{});
}

unsigned grid_of(const LinearParams& p, int roles) { return (unsigned)linear_grid((int64_t)p.shape.slots * p.shape.kv_heads * roles, 4 * roles); }

}  // namespace
}  // namespace hspmd
