// Device code shared by the kernels around the paged cache: where a row is, rotation by a token's own positions,
// 8-bit conversions.
#pragma once
#include "attn_device.hpp"
#include "paged.hpp"

namespace hspmd {

// A row's sequence and position, and its place in the pool.  All values come from device arrays that nobody has checked: every
// index that follows from them is bounded here.
struct RowPlace {
    int seq;        // -1: the row belongs to no sequence
    int pos;        // position in the sequence; negative: no place
    int page;       // page number, -1 where the table holds none that exists
    int slot;       // slot in the page
};

// by a whole wave, the same x in every lane: the i < n with ends[i] <= x < ends[i + 1], 64 ends at a time; -1: none.  n > 0; ends: n + 1 of them
template <typename T>
__device__ __forceinline__ int interval_of(const T* ends, int n, T x) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n;                                    // it is one of lo .. hi - 1, or none
    for (;;) {
        const int step = (hi - lo + 63) / 64, end = min(lo + (lane + 1) * step, hi);
        const uint64_t m = __ballot(ends[end] > x);
        if (m == 0) return -1;
        const int found = __builtin_ctzll(m);
        hi = min(lo + (found + 1) * step, hi);
        lo += found * step;
        if (step == 1) return ends[lo] <= x ? lo : -1;
    }
}

__device__ __forceinline__ int page_at(const PagedPool& pool, const PagedRows& b, int seq, int index) {
    const int page = b.page_table[(int64_t)seq * b.table_width + index];
    return (unsigned)page < (unsigned)pool.num_pages ? page : -1;
}

__device__ __forceinline__ RowPlace place_of(const PagedPool& pool, const PagedRows& b, int row) {
    RowPlace r{interval_of(b.cu_rows, b.num_seqs, row), -1, -1, 0};
    if (r.seq < 0) return r;
    const int kv = seq_rows(0, 0, b.kv_lens[r.seq], 0, b.table_width, pool.page_shift).kv;
    const int pos = kv - (min(b.cu_rows[r.seq + 1], b.total_rows) - row);   // (cu_rows[seq + 1] > row)
    if (pos < 0) return r;
    r.pos = pos;
    r.page = page_at(pool, b, r.seq, pos >> pool.page_shift);
    r.slot = pos & ((1 << pool.page_shift) - 1);
    return r;
}

// (cos, sin) of VEC consecutive pairs from pair `first` on; `pos`: a token's position on each axis
template <int VEC>
__device__ __forceinline__ void load_turn(const AxesParams& a, const int (&pos)[4], int first, int half, float (&c)[VEC], float (&s)[VEC]) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        const int i = first + j;
        const int axis = (int)(a.axis_of[i >> 5] >> ((i & 31) * 2)) & 3;
        const int at = axis == 0 ? pos[0] : axis == 1 ? pos[1] : axis == 2 ? pos[2] : pos[3];
        float2 cs = make_float2(__builtin_nanf(""), __builtin_nanf(""));
        if ((unsigned)at < (unsigned)a.table_positions) cs = *reinterpret_cast<const float2*>(a.table + ((int64_t)at * half + i) * 2);
        c[j] = cs.x;
        s[j] = cs.y;
    }
}

// One pair turned.  Products and sums are rounded one by one (no fused multiply-add): the result then does not depend on how a
// compiler contracts the expression, which matters where it is quantised next: a value at a rounding border, or a row maximum
// at a power of two, comes out the same from any fp32 evaluation of the formula.
__device__ __forceinline__ void turn_pair(float lo, float hi, float c, float s, float& out_lo, float& out_hi) {
#pragma clang fp contract(off)
    const float a = lo * c, b = hi * s, d = hi * c, e = lo * s;
    out_lo = a - b;
    out_hi = d + e;
}

// VEC consecutive elements, 2 or 4 bytes each, as floats and back
template <int VEC, bool F32>
__device__ __forceinline__ void load_floats(const void* base, int elem, float (&x)[VEC]) {
    if constexpr (F32) {
#pragma unroll
        for (int j = 0; j < VEC; j += 4) {
            const f32x4 t = *reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + elem + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j + e] = t[e];
        }
    } else {
        using Raw = typename std::conditional<VEC == 8, u32x4, u32x2>::type;
        const Raw t = *reinterpret_cast<const Raw*>(static_cast<const uint16_t*>(base) + elem);
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) {
            x[2 * j] = __uint_as_float(t[j] << 16);
            x[2 * j + 1] = __uint_as_float(t[j] & 0xffff0000u);
        }
    }
}
template <int VEC, bool F32>
__device__ __forceinline__ void store_floats(void* base, int elem, const float (&x)[VEC]) {
    if constexpr (F32) {
#pragma unroll
        for (int j = 0; j < VEC; j += 4)
            *reinterpret_cast<f32x4*>(static_cast<float*>(base) + elem + j) = f32x4{x[j], x[j + 1], x[j + 2], x[j + 3]};
    } else {
        using Raw = typename std::conditional<VEC == 8, u32x4, u32x2>::type;
        Raw t;
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) t[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
        *reinterpret_cast<Raw*>(static_cast<uint16_t*>(base) + elem) = t;
    }
}

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// the scale that a stored byte stands for (bytes that the library writes: 27 .. 247)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// smallest e >= -100 with amax <= 448 * 2^e (448 = 1.75 * 2^8, the largest e4m3 number); amax finite, >= 0
__device__ __forceinline__ int e4m3_exponent(float amax) {
    const uint32_t u = __float_as_uint(amax);
    return max((int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), -100);
}

__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// four floats, already in units of the scale, as e4m3 (round to nearest even)
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// four e4m3 numbers times `scale` (a power of two) as bf16, exactly
__device__ __forceinline__ u32x2 e4m3_to_bf16(uint32_t x, float scale) {
    union { bf16x2 v; uint32_t u; } a, b;
    a.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false);
    b.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true);
    return u32x2{a.u, b.u};
}

}  // namespace hspmd
