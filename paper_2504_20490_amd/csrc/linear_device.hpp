// Device code shared by the kernels of the linear attention: where a workgroup's tokens are, decays along a chunk, two-part operands.
#pragma once
#include "attn_device.hpp"
#include "linear.hpp"

#include <type_traits>

namespace hspmd {

// A decay of 2^-160 or less leaves nothing of any fp32 number, and infinities would make differences of sums NaN.
constexpr float kForgetLog2 = -160.f;
__device__ __forceinline__ float decay_log2(float log_decay) {
    const float g = log_decay * kLog2e;
    return g < kForgetLog2 ? kForgetLog2 : g;      // (NaN stays)
}

// The same as a multiple of 2^-10 and the rest: sums of 64 of the former, at most 10240, are exact, those of the latter below 2^-5 and off by 2^-30, and so is what a
// difference of two sums is off by, however strong the decays between.  All that compute the weight of a pair, from either end of a chunk, then come to the same
// bits, but for a rounding here and there: the decays' gradients are differences between sums of such weights.  (One sum: decays of e^-5 in every row left errors of 6e-5
// in their gradients; whole numbers and rests: a fixed decay of e^-1 5e-5 in the gradient over 8192 rows.)
constexpr float kDecayStep = 0x1p-10f;
__device__ __forceinline__ DecayLog2 split_decay_log2(float log_decay) {
    constexpr float kLog2eRest = 1.9259629e-8f;       // log2(e) - kLog2e
    const float whole = __builtin_rintf(log_decay * (kLog2e / kDecayStep)) * kDecayStep;
    if (whole < kForgetLog2) return {kForgetLog2, 0.f};
    return {whole, __builtin_fmaf(log_decay, kLog2eRest, __builtin_fmaf(log_decay, kLog2e, -whole))};
}

// inclusive sum over the lanes 0 .. lane of a wave (all lanes active): rows of 16 lanes, then their last lanes to the rows behind
__device__ __forceinline__ float sum_up_to(float x) {
    const auto moved = [](float v, auto ctrl, auto rows) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, true));
    };
    using std::integral_constant;
    x += moved(x, integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});      // row_shr 1, 2, 4, 8
    x += moved(x, integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
    x += moved(x, integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
    x += moved(x, integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
    x += moved(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});      // row_bcast 15: lane 15 of rows 0, 2 to rows 1, 3
    x += moved(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});      // row_bcast 31: lane 31 to rows 2, 3
    return x;
}
// the value of the lane before, 0 in lane 0 (all lanes active): wave_shr 1
__device__ __forceinline__ float lane_before(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x138, 0xf, 0xf, true)); }
// over the lanes lane .. 63
__device__ __forceinline__ float sum_from(float x, int lane) {
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
        const float y = __shfl_down(x, step, 64);
        x += lane + step < 64 ? y : 0.f;
    }
    return x;
}
template <typename T>
__device__ __forceinline__ T wave_sum(T x) {
#pragma unroll
    for (int step = 1; step < 64; step *= 2) x += __shfl_xor(x, step, 64);
    return x;
}

// A segment of a sequence: what a workgroup computes for one KV head.
struct Segment {
    int seq, index, count;   // of the sequence's segments
    int start, rows;         // its first token in the packed tensors, tokens of it (0: an empty sequence)
    int entry;               // first entry of the sequence (count > 1)
};

// by a whole wave, the same slot in every lane; false: the slot is none
__device__ __forceinline__ bool find_segment(const LinearShape& p, int slot, Segment& out) {
    const int lane = threadIdx.x & 63;
    int seq = slot;
    if (p.seg_rows > 0) {
        // the last sequence whose first slot is not behind this one, 64 of them at a time
        int lo = 0, n = p.num_seqs;
        while (n > 1) {
            const int step = (n + 63) / 64, at = lane * step;
            bool before = false;
            if (at < n) before = linear_first_slot(linear_rows(p.cu_rows[lo + at], 0, p.total_rows).start, lo + at, p.seg_rows) <= slot;
            const uint64_t m = __ballot(before);
            const int found = m ? 63 - __builtin_clzll(m) : 0;
            lo += found * step;
            n = min(step, n - found * step);
        }
        seq = lo;
    }
    const LinearRows r = linear_rows(p.cu_rows[seq], p.cu_rows[seq + 1], p.total_rows);
    out.seq = seq;
    out.count = 1;
    out.index = 0;
    out.start = r.start;
    out.rows = r.n;
    out.entry = 0;
    if (p.seg_rows > 0) {
        out.count = linear_segments(r.n, p.seg_rows);
        out.index = slot - linear_first_slot(r.start, seq, p.seg_rows);
        if (out.index < 0 || out.index >= out.count) return false;
        out.entry = linear_first_entry(r.start, p.seg_rows);
        const int rows = linear_segment_rows(r.n, out.count);
        out.start = r.start + out.index * rows;
        out.rows = min(r.n - out.index * rows, rows);
    }
    return true;
}

// A state of a pool: *exists = false where there is none (no pool, a negative slot: a state of zeros), NULL with *exists where the
// slot is outside the pool (it is not followed)
__device__ __forceinline__ float* state_of(const LinearStates& s, int seq, int head, int head_dim, bool* exists) {
    *exists = false;
    if (s.data == nullptr) return nullptr;
    const int slot = s.slots ? s.slots[seq] : seq;
    if (slot < 0) return nullptr;
    *exists = true;
    return slot < s.num_slots ? s.data + slot * s.slot_stride + (int64_t)head * head_dim * head_dim : nullptr;
}

typedef __attribute__((ext_vector_type(8))) float f32x8;

// a - the low, or high, half of a pair of bf16 values, or 0 * both + a: one operation instead of unpacking and subtracting.  (The difference is exact where
// the pair is a rounding of a; a pair with an infinity or NaN gives NaN.)
struct PairOps {
    uint32_t low, high, none;     // (-1, 0), (0, -1), (0, 0): in scalar registers, of which an inline constant would mean something else
    __device__ __forceinline__ void init() {
        low = 0x0000bf80u, high = 0xbf800000u, none = 0u;
        asm("" : "+s"(low), "+s"(high), "+s"(none));
    }
    static __device__ __forceinline__ float dot(uint32_t pair, uint32_t by, float a) {
        union { uint32_t u; bf16x2 v; } x, y;
        x.u = pair, y.u = by;
        return __builtin_amdgcn_fdot2_f32_bf16(x.v, y.v, a, false);
    }
};

// What eight values leave of their roundings to bf16, x kept: as PairOps::dot, which overwrites its third operand.  The operations are written out because
// the compiler takes the overwriting form with a copy in front: one more for each value of a state.  A dot product's result may be read three operations
// later by one of another kind; and x must not come from a matrix product just in front, whose results an instruction here would not wait for.
__device__ __forceinline__ f32x8 rest_of_rounding(const f32x8& x, const u32x4& pairs, const PairOps& ops) {
    f32x8 r;
    float r0, r1, r2, r3, r4, r5, r6, r7;
    asm volatile("v_dot2_f32_bf16 %0, %8, %20, %12\n\tv_dot2_f32_bf16 %1, %8, %21, %13\n\t"
                 "v_dot2_f32_bf16 %2, %9, %20, %14\n\tv_dot2_f32_bf16 %3, %9, %21, %15\n\t"
                 "v_dot2_f32_bf16 %4, %10, %20, %16\n\tv_dot2_f32_bf16 %5, %10, %21, %17\n\t"
                 "v_dot2_f32_bf16 %6, %11, %20, %18\n\tv_dot2_f32_bf16 %7, %11, %21, %19\n\ts_nop 2"
                 : "=&v"(r0), "=&v"(r1), "=&v"(r2), "=&v"(r3), "=&v"(r4), "=&v"(r5), "=&v"(r6), "=&v"(r7)
                 : "v"(pairs[0]), "v"(pairs[1]), "v"(pairs[2]), "v"(pairs[3]), "v"(x[0]), "v"(x[1]), "v"(x[2]), "v"(x[3]), "v"(x[4]), "v"(x[5]), "v"(x[6]),
                   "v"(x[7]), "s"(ops.low), "s"(ops.high));
    r[0] = r0, r[1] = r1, r[2] = r2, r[3] = r3, r[4] = r4, r[5] = r5, r[6] = r6, r[7] = r7;
    return r;
}

// fp32 values as sums of bf16 values, each the rounding of what those before it leave: two hold 16 to 17 bits (error 2^-17.5 at most), three all 24
template <int PARTS>
struct Parts {
    bf16x8 part[PARTS];
    // KEEP: x lives on (see rest_of_rounding)
    template <bool KEEP = false>
    __device__ __forceinline__ void of(f32x8 x, const PairOps& ops) {
        if constexpr (KEEP) {
            union { u32x4 u; bf16x8 v; } p;
#pragma unroll
            for (int i = 0; i < 4; ++i) p.u[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
            part[0] = p.v;
            Parts<PARTS - 1> others;
            others.of(rest_of_rounding(x, p.u, ops), ops);
#pragma unroll
            for (int n = 1; n < PARTS; ++n) part[n] = others.part[n - 1];
            return;
        }
#pragma unroll
        for (int n = 0; n < PARTS; ++n) {
            union { u32x4 u; bf16x8 v; } p;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p.u[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
                asm("" : "+v"(p.u[i]));      // (one register from here on: else both halves are converted a second time for the differences)
                if (n + 1 < PARTS) {
                    x[2 * i] = PairOps::dot(p.u[i], ops.low, x[2 * i]);
                    x[2 * i + 1] = PairOps::dot(p.u[i], ops.high, x[2 * i + 1]);
                }
            }
            part[n] = p.v;
        }
    }
};

// Reads of a swizzled tile (see swizzle in attn_device.hpp).  Row and column take part in an address by different bits, and the swizzle is an exclusive
// or of the column's with some of the row's: so an address is a lane's own part, exclusive or the part of the column, plus 32-row steps.
// The lane's parts are values of their own in every round of a loop (`fresh`): derived addresses are then made where they are used, in one operation,
// and not kept in dozens of registers across the loop.
template <int D>
struct TileReads {
    uint32_t row_part;          // row lane % 32, chunk lane / 32
    uint32_t down_part;         // row 4 (lane / 32) + lane % 16 / 4, columns 16 (lane / 16 % 2) + 4 (lane % 4)
    uint32_t ordered_part;      // the same with columns 16 (lane / 16 % 2) + 4 * (0, 2, 1, 3)[lane % 4]
    __device__ __forceinline__ void init(int lane) {
        row_part = tile_offset<D>(lane & 31, (lane >> 5) * 8);
        const int row = ((lane >> 5) << 2) + ((lane & 15) >> 2), c = lane & 3, group = ((lane >> 4) & 1) << 4;
        down_part = tile_offset<D>(row, group + c * 4);
        ordered_part = tile_offset<D>(row, group + ((c & 1) << 1 | c >> 1) * 4);
    }
    __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(row_part), "+v"(down_part), "+v"(ordered_part)); }
    // an operand whose k runs along the rows: rows 32 rb .. + 31, columns 16 kk .. + 15
    __device__ __forceinline__ bf16x8 along(const char* tile, int rb, int kk) const {
        return *reinterpret_cast<const bf16x8*>(tile + (row_part ^ (kk << 5)) + rb * 32 * D * 2);
    }
    // an operand whose k runs down the rows: rows 16 t .. + 15 in the order of an accumulator (see read_transposed_frag), columns 32 cb .. + 31
    __device__ __forceinline__ bf16x8 down(const char* tile, int cb, int t) const { return down_from(tile, down_part ^ (cb << 6), t); }
    // the same with the columns in another order: result row (MFMA M index) 16 g + 8 hi + 4 mid + low is column 16 g + 8 mid + 4 hi + low.
    // An accumulator of a product with such an A operand then holds, in registers 8 t .. 8 t + 7 of lane half hh, the columns
    // 16 t + 8 hh + {0 .. 7}: the k order that an operand read along a row has.
    __device__ __forceinline__ bf16x8 down_ordered(const char* tile, int cb, int t) const { return down_from(tile, ordered_part ^ (cb << 6), t); }

private:
    __device__ __forceinline__ static bf16x8 down_from(const char* tile, uint32_t at, int t) {
        // eight rows further down: the row's bit 3 is bit 1 of the swizzle's (row / 4) % 4
        const s16x4 lo = lds_transpose_read(tile + at + t * 16 * D * 2);
        const s16x4 hi = lds_transpose_read(tile + (at ^ (2 << 4)) + t * 16 * D * 2 + 8 * D * 2);
        union { struct { s16x4 a, b; } s; bf16x8 v; } u;
        u.s.a = lo;
        u.s.b = hi;
        return u.v;
    }
};

}  // namespace hspmd
