// Kernel parameter blocks and host-callable launchers of the linear attention (internal to the library).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/hspmd_attn.h"
#include "linear_index.hpp"

namespace hspmd {

// The rows of a call and what they are cut into
struct LinearShape {
    const int32_t* cu_rows;
    int32_t num_seqs, total_rows;
    int32_t q_heads, kv_heads, group, head_dim;
    int32_t seg_rows;              // 0: every sequence is one segment, slot = sequence
    int32_t slots, entries, windows;
};

// A pool of states, or one state per sequence
struct LinearStates {
    float* data;                   // NULL: none
    const int32_t* slots;          // NULL: sequence s has slot s
    int64_t slot_stride;
    int32_t num_slots;
};

// A log2 as a multiple of 2^-10 and the rest
struct DecayLog2 {
    float whole, rest;
};

struct LinearParams {
    LinearShape shape;
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const uint16_t* d_o;           // backward only
    const float* log_decay;
    int64_t q_stride, kv_stride, do_stride, decay_stride;
    float scale;
    DecayLog2 scale_log2;          // its log2
    LinearStates initial, final;   // backward: `final` is the gradient that comes in (read)
    void* o;                       // forward: bf16
    void* dq;
    void* dk;
    void* dv;
    int32_t grad_f32;
    float* d_initial;              // may be NULL
    float* d_log_decay;            // may be NULL
    // workspace
    float* states;                 // [entries][kv_heads][d][d]: the state at a segment's start
    float* d_states;               // its gradient at a segment's end
    float* seg_decay;              // [entries][kv_heads]: log2 of a segment's decay
    float* q_near;                 // [q_heads][total_rows]: <q, dq> from the own chunk's other tokens ...
    float* q_far;                  // ... and from before the chunk
    float* k_near;                 // [kv_heads][total_rows], likewise
    float* k_far;
    float* across;                 // [2][slots][kv_heads]: <S, dS> at a segment's end, and at a sequence's start (its first slot)
    double* decay_sums;            // [slots][kv_heads]: a segment's share of a fixed decay's gradient
    float* anchors;                // [linear_anchors][kv_heads][linear_anchor_elements]: S at an anchor's start, as the waves hold it ...
    float* d_anchors;              // ... and dS at its end
};

struct LinearSizes {
    int32_t seg_rows;              // as in LinearShape
    int64_t slots, entries, windows;
    size_t state_bytes, decay_bytes, q_row_bytes, k_row_bytes, slot_bytes, anchor_bytes;
    size_t total_bytes(bool backward) const {      // (without anchors where decay gradients are not wanted: anchor_bytes is 0 then)
        return backward ? 2 * state_bytes + decay_bytes + 2 * q_row_bytes + 2 * k_row_bytes + 2 * slot_bytes + 2 * anchor_bytes : state_bytes + decay_bytes;
    }
};
LinearSizes linear_sizes(int32_t total_rows, int32_t num_seqs, int32_t max_rows, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                         bool backward, bool decays);
// states of sequences that are cut into segments; parts: of a source's bf16 values, 2 or 3
void launch_linear_states(const LinearParams& p, bool backward, int parts, hipStream_t stream);
hipError_t launch_linear_fwd(const LinearParams& p, hipStream_t stream);
hipError_t launch_linear_bwd(const LinearParams& p, hipStream_t stream);

struct LinearStepParams {
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const float* log_decay;
    int64_t q_stride, kv_stride, decay_stride;
    float scale;
    LinearStates initial, final;
    uint16_t* o;
    int32_t num_seqs, q_heads, kv_heads, group, head_dim;
};
hipError_t launch_linear_step(const LinearStepParams& p, hipStream_t stream);

}  // namespace hspmd
