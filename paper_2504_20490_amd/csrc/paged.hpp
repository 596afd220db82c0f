// Kernel parameter blocks and host-callable launchers of the rotary embedding with several axes and of the paged
// key/value cache (internal to the library).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/hspmd_attn.h"
#include "paged_index.hpp"

namespace hspmd {

struct AxesParams {
    const float* table;            // (cos, sin) pairs [position][head_dim / 2]
    const int32_t* positions;      // [axis][token], axis stride positions_stride; cache write only: NULL = the row's own position
    int64_t positions_stride;
    uint64_t axis_of[2];           // two bits per pair: pair i in word i / 32
    int32_t table_positions, num_axes;
};

struct RopeAxesParams {
    AxesParams rope;
    const void* q;
    const void* k;
    void* q_out;
    void* k_out;
    int64_t q_stride, kv_stride, q_out_stride, kv_out_stride;   // token strides in elements
    int32_t tokens, q_heads, kv_heads, head_dim;
    int32_t shares;                // waves that share a token's heads
    float sin_sign;                // +1: rotate, -1: rotate back
};
hipError_t launch_rope_axes(RopeAxesParams p, bool f32, hipStream_t stream);

// The pool and the rows of a call (hspmd_kv_cache, hspmd_kv_batch)
struct PagedPool {
    uint8_t* k;
    uint8_t* v;
    uint8_t* k_scale;              // e4m3 only
    uint8_t* v_scale;
    int64_t page_bytes, scale_page_bytes;
    int32_t num_pages, page_shift; // page_size = 1 << page_shift
    int32_t kv_heads, head_dim;
    int32_t row_bytes;             // of a token and head in k or v
};
struct PagedRows {
    const int32_t* cu_rows;
    const int32_t* kv_lens;
    const int32_t* page_table;
    int32_t num_seqs, table_width, total_rows;
};

struct CacheWriteParams {
    PagedPool pool;
    PagedRows rows;
    AxesParams rope;               // table NULL: k is not turned, q not looked at
    const uint16_t* k;
    const uint16_t* v;
    const uint16_t* q;             // may be NULL
    uint16_t* q_out;
    int64_t kv_stride, q_stride, q_out_stride;
    int32_t q_heads;               // 0 without q
    int32_t shares;                // waves that share a row's heads
};
hipError_t launch_cache_write(CacheWriteParams p, bool e4m3, hipStream_t stream);

struct CacheReadParams {
    PagedPool pool;
    PagedRows rows;
    uint16_t* k;
    uint16_t* v;
    int64_t kv_stride;
};
hipError_t launch_cache_read(const CacheReadParams& p, bool e4m3, hipStream_t stream);

// ---- attention over the cache --------------------------------------------------------------------------------------
// The rows of a sequence that share a KV head (n new tokens x group query heads, token by token) are cut into tiles; a row tile and a KV head
// are an item, and the keys of an item are shared out over several workgroups ("chunks") where there are few items.  The launch does not know
// the lengths: the workgroups work their shares out (find_item), the host launches as many as there can be (grid_bounds).
struct PagedAttnParams {
    PagedPool pool;
    PagedRows rows;
    const uint16_t* q;
    uint16_t* o;
    float* lse;                    // may be NULL
    int64_t q_stride;
    int32_t q_heads, group;
    int32_t few_limit;             // sequences with more rows per KV head are for paged_many_kernel
    float scale_log2;              // softmax_scale * log2(e)
    // workspace: results of chunks, row by row (fp32 sums of P V over the head's tile width, and (maximum, sum of weights)), those of
    // paged_few_kernel first; and for every row of the call where its chunks' results are
    float* part_o;
    float2* part_stats;
    const uint32_t* plan;          // NULL: every workgroup sums over the sequences for itself; see plan_words
    int2* where;                   // [total_rows][q_heads], see where_entry
    int32_t few_part_rows, part_rows;
};

// sizes that follow from what the host knows
struct PagedSizes {
    bool few, many, join;          // which kernels run
    int32_t few_limit;
    int64_t few_grid, many_grid;
    int64_t few_part_rows, part_rows;
    size_t where_bytes, stats_bytes, part_bytes, plan_bytes;
    size_t total_bytes() const { return where_bytes + stats_bytes + part_bytes + plan_bytes; }
};
PagedSizes paged_sizes(const PagedRows& rows, int max_rows, int page_shift, int q_heads, int kv_heads, int head_dim);
hipError_t launch_paged_attn(const PagedAttnParams& p, const PagedSizes& sizes, bool e4m3, hipStream_t stream);
hipError_t launch_paged_many(const PagedAttnParams& p, int64_t grid, bool e4m3, hipStream_t stream);

}  // namespace hspmd
