// One key tile of the forward: scores, online softmax and the product with V, written MFMA step by MFMA step (gfx950 only).
// Shared by the kernels that walk key tiles of packed sequences and of a paged cache; where the tiles' copies come from is
// the caller's (`Load`).
#pragma once
#include "attn_device.hpp"
#include "schedule.hpp"

namespace hspmd {

// KD: 16-column steps of head_dim that hold data (D / 16, or fewer when head_dim ends before the tile width: the steps
// beyond it would multiply the zero padding of the query fragments); the product whose output is head_dim wide takes
// (KD + 1) / 2 blocks of 32 columns.  8 x 2048, 32 heads, head_dim 96: 6 steps and 3 blocks instead of 7 and 4, 282 -> 256 us.
template <int D, int KD>
struct FwdGeom {
    static_assert(KD >= 1 && KD <= D / 16, "k-steps inside the tile width");
    static constexpr int KK = KD;       // k-steps of S^T = K Q^T
    static constexpr int DB = (KD + 1) / 2;   // 32-row blocks of O^T that hold data
    static constexpr int kTileBytes = kFwdKTile * D * 2;
};

// NB: 32-key blocks of every tile that the wave takes: both, or one when two waves share the tile (SPLIT)
template <int D, int KD, int NB>
struct FwdState {
    using G = FwdGeom<D, KD>;
    bf16x8 qf[G::KK];      // this lane's query row (B operand of S^T = K Q^T)
    f32x16 acc[G::DB];     // O^T accumulator
    f32x16 s[NB];          // S^T of the current tile, one fragment per 32-key block
    float m, l;            // running row max of the raw scores; this lane's share of the running row sum
    float tnext;           // this lane's maximum over s[] as it stands (all keys taken as visible)
    int rm[G::KK];         // per-lane LDS offsets of the K fragments (row-major read), block 0 of a tile
    int tr[G::DB][2];      // per-lane LDS offsets of the V^T fragments (transpose read), k-step 0 of a tile
};

// this wave's single copy instructions of one whole K tile and one whole V tile
template <int D>
struct FwdTileLoad {
    using Copy = TileCopy<D, kFwdKTile>;
    static constexpr int kPieces = Copy::kPerWave;
    const Copy* copy;
    const uint16_t* k_row;   // first row of the K tile, this kv head, column 0
    const uint16_t* v_row;
    uint32_t k_dst;          // LDS byte addresses
    uint32_t v_dst;
    int wave;
    __device__ __forceinline__ void k_piece(int i) const {
#pragma unroll
        for (int n = 0; n < Copy::kPerWave; ++n)
            if (n == i) copy->issue_full_one_at(n, k_dst, k_row, wave);
    }
    __device__ __forceinline__ void v_piece(int i) const {
#pragma unroll
        for (int n = 0; n < Copy::kPerWave; ++n)
            if (n == i) copy->issue_full_one_at(n, v_dst, v_row, wave);
    }
};

// this lane's maximum over its 16 NB scores of a tile (v_max3: two scores per instruction)
template <int NB>
__device__ __forceinline__ float lane_max(const f32x16 (&s)[NB]) {
    float t = fmaxf(s[0][0], s[0][1]);
#pragma unroll
    for (int e = 2; e < 16 * NB; ++e) t = fmaxf(t, s[e >> 4][e & 15]);   // a chain: pairs of steps become one v_max3
    return t;
}

__device__ __forceinline__ float pair_max(float x) {
    // v_permlane32_swap: first result = the value held by lane l % 32, second = the value of lane l % 32 + 32
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// One iteration on key tile kt, whose scores are already in st.s:
//   first  : VALU only: running max of tile kt; accumulator rescale if some lane's max moved
//   phase A: MFMA S^T(kt+1) = K(kt+1) Q^T   |  VALU: exp2, row sum, bf16 pack of tile kt's first key block
//   phase B: MFMA O^T += V(kt)^T P^T(kt)     |  VALU: the same for its second key block, under the first MFMAs
// kbuf: K tile kt+1; vbuf: V tile kt.  MASK: tile kt touches the diagonal (keys beyond a lane's own row get
// weight 0); LAST: there is no tile kt+1.
// SPREAD: the iteration also issues this wave's share of the copies of K(kt+2) and V(kt+1), both whole
// tiles, one instruction per MFMA step of phase A.  Issued back to back after the barrier, the copies of
// all waves queue up in front of the CU's one address unit.
// SOME (block variant, half items, teams): a lane's row may have no visible key so far, or, with a share of the keys, none with a finite score (its
// running max is still -inf): the maximum that the exponentials are taken against is then replaced by 0, which keeps every
// weight and the rescale factor at 0.
// Load: k_piece(i), v_piece(i) issue the wave's copies of the iteration.
// NB = 1: the wave's only 32-key block of the tile is part of the addresses; its eight score pairs all go under the
// MFMAs of phase A, the copies too (two per step where the phase has fewer steps than copies).
template <int D, int KD, int NB, bool MASK, bool LAST, bool SPREAD, bool SOME, typename Load>
__device__ __forceinline__ void fwd_iteration(FwdState<D, KD, NB>& st, const char* kbuf, const char* vbuf, float c,
                                              int dkey /* my_row - key0 - 4 * (lane / 32) */,
                                              const Load& load) {
    using G = FwdGeom<D, KD>;
    constexpr int KK = G::KK, DB = G::DB;
    constexpr int NP = Load::kPieces;   // copy instructions per wave and tile

    // ---------------- running max of tile kt and the (rare) accumulator rescale: a short VALU-only stretch
    if constexpr (MASK) {
        // element i of block jb is key 32 jb + 8 (i / 4) + i % 4 (+ 4 (lane / 32), folded into dkey)
#pragma unroll
        for (int jb = 0; jb < NB; ++jb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (32 * jb + 8 * (i >> 2) + (i & 3) > dkey) st.s[jb][i] = -INFINITY;
    }
    // An unmasked tile's maximum was taken while the scores were still warm: under the last MFMAs of the iteration
    // that produced them, which have no other VALU work to run beside them (st.tnext).
    float tmax = st.tnext;
    if constexpr (MASK) tmax = lane_max(st.s);
    tmax = pair_max(tmax);
    // st.m is the reference that the exponentials are taken against, not the exact running maximum: it moves only
    // when the maximum has risen by more than kMaxSlack in the exponent (base-2) domain.  Weights then lie in
    // (0, 2^kMaxSlack] instead of (0, 1] -- the same relative precision in bf16 and fp32, and O and LSE do not depend on
    // the reference -- while the accumulator rescale, which a moving maximum of ANY of the wave's 32 rows triggers,
    // becomes rare after the first tiles.  (-inf - -inf = NaN compares false: a row without a visible key keeps -inf.)
    constexpr float kMaxSlack = 8.f;
    const float m_new = (tmax - st.m) * c > kMaxSlack ? tmax : st.m;
    const float m_ref = (SOME && m_new == -INFINITY) ? 0.f : m_new;
    const float alpha = fast_exp2((st.m - m_ref) * c);
    const float mc = m_ref * c;
    if (__any(m_new > st.m)) {      // wave-uniform: skip the accumulator rescale when no lane's max moved
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) st.acc[db][i] *= alpha;
    }
    st.m = m_new;
    __builtin_amdgcn_sched_barrier(0);

    // The two waves of a SIMD (one of each resident workgroup) compete for its issue slots: the one that is in its
    // MFMA phases goes first, so that the matrix pipe does not wait behind the other's VALU-only stretch.
    __builtin_amdgcn_s_setprio(1);
    // ---------------- phase A: S^T(kt+1) on the MFMA, exp2 / row sum / bf16 pack of tile kt on the VALU.
    // Written out step by step with a scheduling barrier after each: step n issues the K fragment read of
    // MFMA n + kAheadK, MFMA n, and the softmax work on two scores.
    f32x16 sn[NB];
    float psum = 0.f;
    union { u32x4 u; bf16x8 v; } pw[2 * NB];
    auto softmax_pair = [&](int n) {   // scores 2n, 2n+1 of the tile's 32 per lane -> one packed bf16 pair
        const int jb = n >> 3, i = (n & 7) * 2;
        const float e0 = fast_exp2(fmaf(st.s[jb][i], c, -mc));
        const float e1 = fast_exp2(fmaf(st.s[jb][i + 1], c, -mc));
        psum += e0 + e1;
        // the sum is needed only at the end of the iteration, and left alone the compiler keeps all 32 weights in
        // registers and adds them up there, in one stretch of 32 VALU instructions with no MFMA to run under;
        // an (empty) statement that reads and writes the sum keeps each pair's two additions in this step
        asm volatile("" : "+v"(psum));
        pw[jb * 2 + (i >> 3)].u[(i >> 1) & 3] = pack_bf16(e0, e1);
    };
    if constexpr (!LAST) {
        constexpr int kAheadK = 4;
        constexpr int NM = NB * KK;              // MFMAs of the phase
        static_assert(NB == 1 || 2 * NP <= NM, "one copy instruction per MFMA step");
        // the tile's key blocks in turn: consecutive MFMAs take the same query fragment, and none continues its predecessor's chain
        // (one block after the other / in turn, interleaved: 8 x 2048, 32 heads, width 64 200.2 / 198.2 us; 6001 tokens, 32 heads on 8 96.5 /
        // 96.0; 8 x 2048, 32 heads 303.6 / 302.9; 8 x 4096, head_dim 104 522 / 521; short sequences of width 64 46.9 / 47.1)
        auto k_frag = [&](int n) {
            return *reinterpret_cast<const bf16x8*>(kbuf + st.rm[n / NB] + (n % NB) * 32 * D * 2);
        };
        bf16x8 kq[kAheadK + 1];
#pragma unroll
        for (int n = 0; n < kAheadK; ++n) kq[n] = k_frag(n);
#pragma unroll
        for (int jb = 0; jb < NB; ++jb)
#pragma unroll
            for (int i = 0; i < 16; ++i) sn[jb][i] = 0.f;
#pragma unroll
        for (int n = 0; n < NM; ++n) {
            if (n + kAheadK < NM) kq[(n + kAheadK) % (kAheadK + 1)] = k_frag(n + kAheadK);
            sn[n % NB] = mfma(kq[n % (kAheadK + 1)], st.qf[n / NB], sn[n % NB]);
            // the first 8 of the 16 score pairs (key block 0, P fragments 0 and 1) spread over the NM MFMAs; the
            // other 8 go under the first P V MFMAs of phase B, which only need fragments 0 and 1
            if constexpr (NB == 1) {
#pragma unroll
                for (int x = n * 8 / NM; x < (n + 1) * 8 / NM; ++x) softmax_pair(x);
            } else if constexpr (NM > 8) {
                // pairs 0 .. NM/2 - 1 at the even steps; with fewer than 16 steps the remaining ones at the last odd steps
                if (n % 2 == 0) softmax_pair(n / 2);
                else if (7 - (NM - 1 - n) / 2 >= NM / 2) softmax_pair(7 - (NM - 1 - n) / 2);
            } else {
                static_assert(NM == 8, "eight score pairs over the steps of the phase");
                softmax_pair(n);
            }
            if constexpr (SPREAD && NB == 1) {
#pragma unroll
                for (int x = n * 2 * NP / NM; x < (n + 1) * 2 * NP / NM; ++x) {
                    if (x < NP) load.k_piece(x);
                    else load.v_piece(x - NP);
                }
            } else if constexpr (SPREAD) {
                // all copies early in the iteration: both tiles are needed right after the next barrier
                if (n < NP) load.k_piece(n);
                else if (n < 2 * NP) load.v_piece(n - NP);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
#pragma unroll
        for (int n = 0; n < 8; ++n) softmax_pair(n);
    }
    __builtin_amdgcn_sched_barrier(0);

    // ---------------- phase B: O^T += V(kt)^T P^T(kt), transpose reads kAheadV MFMAs ahead
    {
        constexpr int kAheadV = 3;
        constexpr int NM = 2 * NB * DB;
        auto v_frag = [&](int n) {
            const int t = n / DB, db = n % DB;
            const int off = t * 16 * D * 2;
            union { struct { s16x4 a, b; } s; bf16x8 v; } u;
            u.s.a = lds_transpose_read(vbuf + st.tr[db][0] + off);
            u.s.b = lds_transpose_read(vbuf + st.tr[db][1] + off);
            return u.v;
        };
        bf16x8 vq[kAheadV + 1];
#pragma unroll
        for (int n = 0; n < kAheadV; ++n) vq[n] = v_frag(n);
        // the next tile's maximum, a share of its 32 scores per step (the scores are complete since phase A)
        float tnext = -INFINITY;
        auto max_share = [&](int e0, int count) {
#pragma unroll
            for (int e = e0; e < e0 + count; ++e) tnext = fmaxf(tnext, sn[e >> 4][e & 15]);   // a chain: v_max3 per pair
            // (an empty statement on the running value keeps the share in its step: nothing else needs the value
            // before the end of the iteration, and the compiler would collect all 32 there)
            asm volatile("" : "+v"(tnext));
        };
#pragma unroll
        for (int n = 0; n < NM; ++n) {
            if (n + kAheadV < NM) vq[(n + kAheadV) % (kAheadV + 1)] = v_frag(n + kAheadV);
            st.acc[n % DB] = mfma(vq[n % (kAheadV + 1)], pw[n / DB].v, st.acc[n % DB]);
            // score pairs 8 .. 15 (key block 1, P fragments 2 and 3) under the MFMAs of fragments 0 and 1
            if constexpr (NB == 1) {
                if (!LAST) max_share(n * 16 / NM, (n + 1) * 16 / NM - n * 16 / NM);
            } else if (n < NM / 2) {
#pragma unroll
                for (int x = n * 16 / NM; x < (n + 1) * 16 / NM; ++x) softmax_pair(8 + x);
            } else if (!LAST) {
                const int h = n - NM / 2;
                max_share(h * 64 / NM, (h + 1) * 64 / NM - h * 64 / NM);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (!LAST) st.tnext = tnext;
    }
    __builtin_amdgcn_s_setprio(0);
    st.l = st.l * alpha + psum;
    if constexpr (!LAST) {
#pragma unroll
        for (int jb = 0; jb < NB; ++jb) st.s[jb] = sn[jb];
    }
}

}  // namespace hspmd
