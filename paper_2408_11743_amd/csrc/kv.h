// Internal declarations of the paged key-value cache operators: rotating and
// appending new tokens (append.hip), attention of one token per sequence
// (attend.hip), the choice of pages to attend to (select.hip).  Argument
// checks are in kv_api.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "marlin.h"

namespace marlin {

constexpr int kKvMaxCus = 256;        // compute units a workspace is sized for
constexpr int kKvMaxBatch = 1 << 16;  // sequences of a call
constexpr int kTileKeys = 16;         // keys of a tile
constexpr int kHeadTile = 16;         // query heads of one kv head that share a pass over its keys
constexpr int kAttendWaves = 8;       // waves per work-group
constexpr int kAttendGroupsPerCu = 1; // work-groups per compute unit

// Floats of one partial result: fp32 sums of up to kHeadTile heads, then each
// head's maximum and sum.
inline int attend_slot_floats(int head_dim) { return kHeadTile * head_dim + 2 * kHeadTile; }

struct AttendProblem {
    const void *q;  // [B][heads][D], strides below (elements)
    int64_t q_row, q_head;
    const void *k, *v;  // [pages][kv_heads][page size][D]
    const int32_t *table;  // [B][kv_heads or 1][width]
    int64_t table_row, table_head;
    const int32_t *lengths;  // [B]
    void *out;               // [B][heads][D]
    float *lse;              // [B][heads] or NULL
    float *partials;
    uint32_t *counters;
    int B, heads, kv_heads, group, head_tiles;
    int page_shift, width, pages;
    float scale_log2;  // scale * log2(e)
    uint32_t grid_reciprocal;  // floor(2^32 / ranges)
};

hipError_t launch_attend(const AttendProblem &p, int head_dim, marlin_dtype_t dtype, int cus, hipStream_t stream);

struct AppendProblem {
    const void *q, *k, *v;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;
    void *q_out, *k_cache, *v_cache, *bounds;
    const float *cos_sin;
    int positions, rot, interleaved;
    const int32_t *table;
    int64_t table_row;
    const int32_t *lengths, *starts;
    int tokens, B, heads, kv_heads;
    int page_shift, width, pages;
};

hipError_t launch_append(const AppendProblem &p, int head_dim, marlin_dtype_t dtype, hipStream_t stream);

struct SelectProblem {
    const void *q;
    int64_t q_row, q_head;
    const void *bounds;
    const int32_t *table;
    int64_t table_row;
    const int32_t *lengths;
    int32_t *chosen, *chosen_lengths;
    uint32_t *scores;  // [B][kv_heads][width]
    int B, heads, kv_heads, group;
    int page_shift, width, pages, select;
};

hipError_t launch_select(const SelectProblem &p, int head_dim, marlin_dtype_t dtype, hipStream_t stream);

}  // namespace marlin
