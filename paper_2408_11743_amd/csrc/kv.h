// Internal declarations of the paged key-value cache operators: rotating and
// appending new tokens (append.hip, append8.hip), attention of one token per sequence
// (attend.hip) and of several (prompt.hip), the choice of pages to attend to
// (select.hip), pages for new tokens (pages.hip).  Argument checks are in kv_api.cpp.
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
    const float *scales;       // [pages][kv_heads][2][page size / 16] of an 8-bit cache, or NULL
    int window, sinks;         // 0: no window
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

// The same into an 8-bit cache with scales.
struct Append8Problem : AppendProblem {
    float *scales;  // [pages][kv_heads][2][page size / 16]
};

hipError_t launch_append8(const Append8Problem &p, int head_dim, marlin_dtype_t dtype, hipStream_t stream);

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

constexpr int kBlockSlots = 16;  // slots of an 8-bit cache that share a scale
static_assert(kBlockSlots == kTileKeys, "a tile of keys has one scale");
constexpr float kLeastScale = 0x1p-40f, kMostScale = 0x1p40f;

// Attention of several tokens per sequence.
struct PromptProblem {
    const void *q;  // [tokens][heads][D], strides below (elements)
    int64_t q_row, q_head;
    const void *k, *v;
    const float *scales;
    const int32_t *table;  // [B][width]
    int64_t table_row;
    const int32_t *lengths, *starts;
    void *out;
    float *lse;
    float *partials;
    void *records;
    int tokens, B, heads, kv_heads, group;
    int page_shift, width, pages;
    int window, sinks;
    float scale_log2;           // |scale| * log2(e), above zero
    uint32_t q_and, q_xor;      // of two elements of q: the scale's sign, or nothing left where it is zero
    int target;     // work-groups to split the keys for; 0: a tile is one's
    int64_t groups; // of all launches
    int base;       // the launch's first work-group
};

// How a call of these sizes is split: rows of a tile, work-groups to split the keys for (or 0) and at the most, workspace floats of one.
struct PromptPlan {
    bool few;  // the kernel for few rows a sequence
    bool two;  // weights in two parts
    int rows, target, slot_floats;
    int64_t groups;
};
// positions: of a table's row, at most.  A plan for more compute units, up to kKvMaxCus, needs no less of the workspace.
PromptPlan plan_prompt(int64_t tokens, int64_t B, int64_t heads, int64_t kv_heads, int head_dim, bool eight, int64_t positions, int cus);
size_t prompt_workspace(const PromptPlan &plan);  // bytes behind the counters

hipError_t launch_prompt(const PromptProblem &p, const PromptPlan &plan, int head_dim, marlin_dtype_t dtype, hipStream_t stream);

struct PagesProblem {
    int32_t *table;
    int64_t table_row;
    int32_t *lengths;
    const int32_t *new_tokens;
    int32_t *free_pages, *free_count, *starts;
    int64_t *slots;
    int32_t *before;  // workspace: [B] pages taken before the sequence, then the free ones' count
    int B, width, pages, page_shift, tokens, window, sinks;
    const int32_t *back;  // [B] tokens taken back first, or NULL
};

hipError_t launch_pages(const PagesProblem &p, hipStream_t stream);

}  // namespace marlin
