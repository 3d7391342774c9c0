// Host side of the paged key-value cache entry points (include/marlin.h):
// argument checks, all before any HIP call, and launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "internal.h"
#include "kv.h"
#include "marlin.h"

using namespace marlin;

namespace {

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool aligned16(const void *p) { return aligned(p, 16); }

int shift_of(int64_t pow2)
{
    int s = 0;
    while (((int64_t)1 << s) < pow2) ++s;
    return s;
}

bool dtype_ok(int64_t d) { return d == MARLIN_F16 || d == MARLIN_BF16; }

bool shape_ok(int64_t B, int64_t heads, int64_t kv_heads, int64_t head_dim, int64_t pages, int64_t page_size,
              int64_t width)
{
    if (B < 0 || B > kKvMaxBatch) return false;
    if (kv_heads < 1 || heads < kv_heads || heads > 1024 || heads % kv_heads != 0) return false;
    if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 256) return false;
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0) return false;
    if (pages < 1 || pages > INT32_MAX || width < 1 || width > (1 << 30) / page_size) return false;
    return true;
}

// Strides (elements) of 16-bit rows that 16-byte loads can follow.
bool strides_ok(int64_t row, int64_t head) { return row >= 0 && head >= 0 && row % 8 == 0 && head % 8 == 0; }

// Scores of one call: at most 2^29, whole 64-page blocks counted.
bool scores_ok(int64_t B, int64_t kv_heads, int64_t width)
{
    return width <= (1 << 29) && (width + 63) / 64 * B * kv_heads <= (1 << 23);
}

constexpr int64_t kMaxTokens = 1 << 24;     // of a call
constexpr int64_t kMaxPositions = 1 << 30;  // of a table's row

// Rows of a kv head: new tokens by the heads that share it.
bool rows_of_tokens_ok(int64_t tokens, int64_t heads, int64_t kv_heads)
{
    return tokens >= 0 && tokens <= kMaxTokens && tokens * (heads / kv_heads) <= (1 << 30);
}

bool visible_ok(int64_t window, int64_t sinks) { return window >= 0 && window <= (1 << 30) && sinks >= 0 && sinks <= (1 << 30); }

}  // namespace

extern "C" {

marlin_status_t marlin_kv_append(const marlin_kv_append_args *a, hipStream_t stream)
{
    if (!a) return MARLIN_ERR_NULL_POINTER;
    if (!shape_ok(a->B, a->heads, a->kv_heads, a->head_dim, a->pages, a->page_size, a->width)) return MARLIN_ERR_INVALID_SHAPE;
    if (a->tokens < 0 || a->tokens > (1 << 24) || (!a->starts && a->tokens != a->B)) return MARLIN_ERR_INVALID_SHAPE;
    if (!strides_ok(a->q_row, a->q_head) || !strides_ok(a->k_row, a->k_head) || !strides_ok(a->v_row, a->v_head) ||
        a->table_row < 0)
        return MARLIN_ERR_INVALID_SHAPE;
    if (!dtype_ok(a->dtype) || a->rot < 0 || a->rot > a->head_dim || a->rot % 16 != 0 || a->interleaved < 0 ||
        a->interleaved > 1)
        return MARLIN_ERR_INVALID_ARGUMENT;
    if (a->rot > 0 && (a->positions < 1 || a->positions > (1 << 30))) return MARLIN_ERR_INVALID_SHAPE;
    if (a->B == 0 || a->tokens == 0) return MARLIN_OK;
    if (!a->q || !a->k || !a->v || !a->q_out || !a->k_cache || !a->v_cache || !a->table || !a->lengths ||
        (a->rot > 0 && !a->cos_sin))
        return MARLIN_ERR_NULL_POINTER;
    if (!aligned16(a->q) || !aligned16(a->k) || !aligned16(a->v) || !aligned16(a->q_out) || !aligned16(a->k_cache) ||
        !aligned16(a->v_cache) || !aligned16(a->bounds) || !aligned16(a->cos_sin) || !aligned(a->table, 4) ||
        !aligned(a->lengths, 4) || !aligned(a->starts, 4))
        return MARLIN_ERR_MISALIGNED;

    AppendProblem p;
    p.q = a->q;
    p.k = a->k;
    p.v = a->v;
    p.q_row = a->q_row;
    p.q_head = a->q_head;
    p.k_row = a->k_row;
    p.k_head = a->k_head;
    p.v_row = a->v_row;
    p.v_head = a->v_head;
    p.q_out = a->q_out;
    p.k_cache = a->k_cache;
    p.v_cache = a->v_cache;
    p.bounds = a->bounds;
    p.cos_sin = a->cos_sin;
    p.positions = (int)(a->rot > 0 ? a->positions : 0);
    p.rot = (int)a->rot;
    p.interleaved = (int)a->interleaved;
    p.table = a->table;
    p.table_row = a->table_row;
    p.lengths = a->lengths;
    p.starts = a->starts;
    p.tokens = (int)a->tokens;
    p.B = (int)a->B;
    p.heads = (int)a->heads;
    p.kv_heads = (int)a->kv_heads;
    p.page_shift = shift_of(a->page_size);
    p.width = (int)a->width;
    p.pages = (int)a->pages;
    return launch_append(p, (int)a->head_dim, (marlin_dtype_t)a->dtype, stream) == hipSuccess ? MARLIN_OK : MARLIN_ERR_HIP;
}

size_t marlin_paged_attention_workspace_bytes(int64_t head_dim)
{
    if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 256) return 0;
    return kCounterRegionBytes + (size_t)2 * kKvMaxCus * kAttendGroupsPerCu * attend_slot_floats((int)head_dim) * sizeof(float);
}

marlin_status_t marlin_paged_attention(const marlin_paged_attention_args *a, hipStream_t stream)
{
    if (!a) return MARLIN_ERR_NULL_POINTER;
    if (!shape_ok(a->B, a->heads, a->kv_heads, a->head_dim, a->pages, a->page_size, a->width)) return MARLIN_ERR_INVALID_SHAPE;
    if (!strides_ok(a->q_row, a->q_head) || a->table_row < 0 || a->table_head < 0) return MARLIN_ERR_INVALID_SHAPE;
    const int64_t group = a->heads / a->kv_heads, head_tiles = (group + kHeadTile - 1) / kHeadTile;
    const int64_t tiles = a->width * a->page_size / kTileKeys;
    if (a->B > 0 && tiles + 2 > INT32_MAX / (a->B * a->kv_heads * head_tiles)) return MARLIN_ERR_INVALID_SHAPE;
    if (!dtype_ok(a->dtype) || !std::isfinite(a->scale) || !std::isfinite((float)(a->scale * 1.4426950408889634)))
        return MARLIN_ERR_INVALID_ARGUMENT;
    if (a->B == 0) return MARLIN_OK;
    if (!a->q || !a->k_cache || !a->v_cache || !a->table || !a->lengths || !a->out || !a->workspace)
        return MARLIN_ERR_NULL_POINTER;
    if (!aligned16(a->q) || !aligned16(a->k_cache) || !aligned16(a->v_cache) || !aligned16(a->out) ||
        !aligned16(a->workspace) || !aligned(a->table, 4) || !aligned(a->lengths, 4) || !aligned(a->lse, 4))
        return MARLIN_ERR_MISALIGNED;
    if (a->workspace_bytes < marlin_paged_attention_workspace_bytes(a->head_dim)) return MARLIN_ERR_WORKSPACE_TOO_SMALL;

    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return MARLIN_ERR_HIP;
    const int cus = device_cu_count(device);
    if (cus <= 0) return MARLIN_ERR_HIP;
    AttendProblem p;
    p.q = a->q;
    p.q_row = a->q_row;
    p.q_head = a->q_head;
    p.k = a->k_cache;
    p.v = a->v_cache;
    p.table = a->table;
    p.table_row = a->table_row;
    p.table_head = a->table_head;
    p.lengths = a->lengths;
    p.out = a->out;
    p.lse = a->lse;
    p.counters = (uint32_t *)a->workspace;
    p.partials = (float *)((char *)a->workspace + kCounterRegionBytes);
    p.B = (int)a->B;
    p.heads = (int)a->heads;
    p.kv_heads = (int)a->kv_heads;
    p.group = (int)group;
    p.head_tiles = (int)head_tiles;
    p.page_shift = shift_of(a->page_size);
    p.width = (int)a->width;
    p.pages = (int)a->pages;
    p.scale_log2 = (float)(a->scale * 1.4426950408889634);
    p.scales = nullptr;
    p.window = p.sinks = 0;
    return launch_attend(p, (int)a->head_dim, (marlin_dtype_t)a->dtype, cus, stream) == hipSuccess ? MARLIN_OK : MARLIN_ERR_HIP;
}

size_t marlin_select_pages_workspace_bytes(int64_t B, int64_t kv_heads, int64_t width)
{
    if (B < 0 || B > kKvMaxBatch || kv_heads < 1 || kv_heads > 1024 || width < 1 || !scores_ok(B, kv_heads, width)) return 0;
    return kCounterRegionBytes + (size_t)B * (size_t)kv_heads * (size_t)width * sizeof(uint32_t);
}

marlin_status_t marlin_select_pages(const marlin_select_pages_args *a, hipStream_t stream)
{
    if (!a) return MARLIN_ERR_NULL_POINTER;
    if (!shape_ok(a->B, a->heads, a->kv_heads, a->head_dim, a->pages, a->page_size, a->width)) return MARLIN_ERR_INVALID_SHAPE;
    if (!strides_ok(a->q_row, a->q_head) || a->table_row < 0) return MARLIN_ERR_INVALID_SHAPE;
    if (!scores_ok(a->B, a->kv_heads, a->width)) return MARLIN_ERR_INVALID_SHAPE;
    if (!dtype_ok(a->dtype) || a->select < 1 || a->select > (1 << 20)) return MARLIN_ERR_INVALID_ARGUMENT;
    if (a->B == 0) return MARLIN_OK;
    if (!a->q || !a->bounds || !a->table || !a->lengths || !a->chosen || !a->chosen_lengths || !a->workspace)
        return MARLIN_ERR_NULL_POINTER;
    if (!aligned16(a->q) || !aligned16(a->bounds) || !aligned16(a->workspace) || !aligned(a->table, 4) ||
        !aligned(a->lengths, 4) || !aligned(a->chosen, 4) || !aligned(a->chosen_lengths, 4))
        return MARLIN_ERR_MISALIGNED;
    if (a->workspace_bytes < marlin_select_pages_workspace_bytes(a->B, a->kv_heads, a->width))
        return MARLIN_ERR_WORKSPACE_TOO_SMALL;

    SelectProblem p;
    p.q = a->q;
    p.q_row = a->q_row;
    p.q_head = a->q_head;
    p.bounds = a->bounds;
    p.table = a->table;
    p.table_row = a->table_row;
    p.lengths = a->lengths;
    p.chosen = a->chosen;
    p.chosen_lengths = a->chosen_lengths;
    p.scores = (uint32_t *)((char *)a->workspace + kCounterRegionBytes);
    p.B = (int)a->B;
    p.heads = (int)a->heads;
    p.kv_heads = (int)a->kv_heads;
    p.group = (int)(a->heads / a->kv_heads);
    p.page_shift = shift_of(a->page_size);
    p.width = (int)a->width;
    p.pages = (int)a->pages;
    p.select = (int)a->select;
    return launch_select(p, (int)a->head_dim, (marlin_dtype_t)a->dtype, stream) == hipSuccess ? MARLIN_OK : MARLIN_ERR_HIP;
}

marlin_status_t marlin_kv_append8(const marlin_kv_append8_args *a, hipStream_t stream)
{
    if (!a) return MARLIN_ERR_NULL_POINTER;
    if (!shape_ok(a->B, a->heads, a->kv_heads, a->head_dim, a->pages, a->page_size, a->width)) return MARLIN_ERR_INVALID_SHAPE;
    if (a->tokens < 0 || a->tokens > kMaxTokens || (!a->starts && a->tokens != a->B)) return MARLIN_ERR_INVALID_SHAPE;
    if (!strides_ok(a->q_row, a->q_head) || !strides_ok(a->k_row, a->k_head) || !strides_ok(a->v_row, a->v_head) ||
        a->table_row < 0)
        return MARLIN_ERR_INVALID_SHAPE;
    if (!dtype_ok(a->dtype) || a->rot < 0 || a->rot > a->head_dim || a->rot % 16 != 0 || a->interleaved < 0 ||
        a->interleaved > 1)
        return MARLIN_ERR_INVALID_ARGUMENT;
    if (a->rot > 0 && (a->positions < 1 || a->positions > (1 << 30))) return MARLIN_ERR_INVALID_SHAPE;
    if (a->B == 0 || a->tokens == 0) return MARLIN_OK;
    if (!a->q || !a->k || !a->v || !a->q_out || !a->k_cache || !a->v_cache || !a->scales || !a->table || !a->lengths ||
        (a->rot > 0 && !a->cos_sin))
        return MARLIN_ERR_NULL_POINTER;
    if (!aligned16(a->q) || !aligned16(a->k) || !aligned16(a->v) || !aligned16(a->q_out) || !aligned16(a->k_cache) ||
        !aligned16(a->v_cache) || !aligned16(a->cos_sin) || !aligned(a->scales, 4) || !aligned(a->table, 4) ||
        !aligned(a->lengths, 4) || !aligned(a->starts, 4))
        return MARLIN_ERR_MISALIGNED;

    Append8Problem p;
    p.q = a->q;
    p.k = a->k;
    p.v = a->v;
    p.q_row = a->q_row;
    p.q_head = a->q_head;
    p.k_row = a->k_row;
    p.k_head = a->k_head;
    p.v_row = a->v_row;
    p.v_head = a->v_head;
    p.q_out = a->q_out;
    p.k_cache = a->k_cache;
    p.v_cache = a->v_cache;
    p.bounds = nullptr;
    p.scales = a->scales;
    p.cos_sin = a->cos_sin;
    p.positions = (int)(a->rot > 0 ? a->positions : 0);
    p.rot = (int)a->rot;
    p.interleaved = (int)a->interleaved;
    p.table = a->table;
    p.table_row = a->table_row;
    p.lengths = a->lengths;
    p.starts = a->starts;
    p.tokens = (int)a->tokens;
    p.B = (int)a->B;
    p.heads = (int)a->heads;
    p.kv_heads = (int)a->kv_heads;
    p.page_shift = shift_of(a->page_size);
    p.width = (int)a->width;
    p.pages = (int)a->pages;
    return launch_append8(p, (int)a->head_dim, (marlin_dtype_t)a->dtype, stream) == hipSuccess ? MARLIN_OK : MARLIN_ERR_HIP;
}

size_t marlin_cache_attention_workspace_bytes(int64_t starts, int64_t tokens, int64_t B, int64_t heads, int64_t kv_heads,
                                              int64_t head_dim)
{
    if (!shape_ok(B, heads, kv_heads, head_dim, 1, 16, 1) || !rows_of_tokens_ok(tokens, heads, kv_heads)) return 0;
    if (!starts) return marlin_paged_attention_workspace_bytes(head_dim);
    size_t most = 0;
    for (const bool eight : {false, true}) {
        const size_t x = prompt_workspace(plan_prompt(tokens, B, heads, kv_heads, (int)head_dim, eight, kMaxPositions, kKvMaxCus));
        if (x > most) most = x;
    }
    return kCounterRegionBytes + most;
}

marlin_status_t marlin_cache_attention(const marlin_cache_attention_args *a, hipStream_t stream)
{
    if (!a) return MARLIN_ERR_NULL_POINTER;
    if (!shape_ok(a->B, a->heads, a->kv_heads, a->head_dim, a->pages, a->page_size, a->width)) return MARLIN_ERR_INVALID_SHAPE;
    if (!strides_ok(a->q_row, a->q_head) || a->table_row < 0 || a->table_head < 0) return MARLIN_ERR_INVALID_SHAPE;
    if (!rows_of_tokens_ok(a->tokens, a->heads, a->kv_heads)) return MARLIN_ERR_INVALID_SHAPE;
    if (a->starts ? a->table_head != 0 : a->tokens != a->B) return MARLIN_ERR_INVALID_SHAPE;
    const int64_t group = a->heads / a->kv_heads, head_tiles = (group + kHeadTile - 1) / kHeadTile;
    const int64_t tiles = a->width * a->page_size / kTileKeys;
    if (!a->starts && a->B > 0 && tiles + 2 > INT32_MAX / (a->B * a->kv_heads * head_tiles)) return MARLIN_ERR_INVALID_SHAPE;
    if (!dtype_ok(a->dtype) || !std::isfinite(a->scale) || !std::isfinite((float)(a->scale * 1.4426950408889634)) ||
        !visible_ok(a->window, a->sinks))
        return MARLIN_ERR_INVALID_ARGUMENT;
    if (a->B == 0 || a->tokens == 0) return MARLIN_OK;
    if (!a->q || !a->k_cache || !a->v_cache || !a->table || !a->lengths || !a->out || !a->workspace)
        return MARLIN_ERR_NULL_POINTER;
    if (!aligned16(a->q) || !aligned16(a->k_cache) || !aligned16(a->v_cache) || !aligned16(a->out) ||
        !aligned16(a->workspace) || !aligned(a->scales, 4) || !aligned(a->table, 4) || !aligned(a->lengths, 4) ||
        !aligned(a->starts, 4) || !aligned(a->lse, 4))
        return MARLIN_ERR_MISALIGNED;
    if (a->workspace_bytes <
        marlin_cache_attention_workspace_bytes(a->starts != nullptr, a->tokens, a->B, a->heads, a->kv_heads, a->head_dim))
        return MARLIN_ERR_WORKSPACE_TOO_SMALL;

    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return MARLIN_ERR_HIP;
    const int cus = device_cu_count(device);
    if (cus <= 0) return MARLIN_ERR_HIP;
    if (a->starts) {
        PromptProblem p;
        p.q = a->q;
        p.q_row = a->q_row;
        p.q_head = a->q_head;
        p.k = a->k_cache;
        p.v = a->v_cache;
        p.scales = a->scales;
        p.table = a->table;
        p.table_row = a->table_row;
        p.lengths = a->lengths;
        p.starts = a->starts;
        p.out = a->out;
        p.lse = a->lse;
        p.partials = (float *)((char *)a->workspace + kCounterRegionBytes);
        p.tokens = (int)a->tokens;
        p.B = (int)a->B;
        p.heads = (int)a->heads;
        p.kv_heads = (int)a->kv_heads;
        p.group = (int)group;
        p.page_shift = shift_of(a->page_size);
        p.width = (int)a->width;
        p.pages = (int)a->pages;
        p.window = (int)a->window;
        p.sinks = (int)a->sinks;
        // the maximum is taken of the products before they are scaled, by a factor above zero
        const float scale = (float)(a->scale * 1.4426950408889634), least = 0x1p-126f;
        p.scale_log2 = std::fabs(scale) > least ? std::fabs(scale) : least;
        p.q_and = std::fabs(scale) > 0 ? 0xFFFFFFFFu : 0u;
        p.q_xor = scale < 0 ? 0x80008000u : 0u;
        const PromptPlan plan = plan_prompt(a->tokens, a->B, a->heads, a->kv_heads, (int)a->head_dim, a->scales != nullptr,
                                            a->width * a->page_size, cus);
        return launch_prompt(p, plan, (int)a->head_dim, (marlin_dtype_t)a->dtype, stream) == hipSuccess ? MARLIN_OK : MARLIN_ERR_HIP;
    }
    AttendProblem p;
    p.q = a->q;
    p.q_row = a->q_row;
    p.q_head = a->q_head;
    p.k = a->k_cache;
    p.v = a->v_cache;
    p.scales = a->scales;
    p.table = a->table;
    p.table_row = a->table_row;
    p.table_head = a->table_head;
    p.lengths = a->lengths;
    p.out = a->out;
    p.lse = a->lse;
    p.counters = (uint32_t *)a->workspace;
    p.partials = (float *)((char *)a->workspace + kCounterRegionBytes);
    p.B = (int)a->B;
    p.heads = (int)a->heads;
    p.kv_heads = (int)a->kv_heads;
    p.group = (int)group;
    p.head_tiles = (int)head_tiles;
    p.page_shift = shift_of(a->page_size);
    p.width = (int)a->width;
    p.pages = (int)a->pages;
    p.window = (int)a->window;
    p.sinks = (int)a->sinks;
    p.scale_log2 = (float)(a->scale * 1.4426950408889634);
    return launch_attend(p, (int)a->head_dim, (marlin_dtype_t)a->dtype, cus, stream) == hipSuccess ? MARLIN_OK : MARLIN_ERR_HIP;
}

size_t marlin_assign_pages_workspace_bytes(int64_t B)
{
    return B < 0 || B > kKvMaxBatch ? 0 : kCounterRegionBytes + ((size_t)B + 1) * sizeof(int32_t);
}

marlin_status_t marlin_assign_pages(const marlin_assign_pages_args *a, hipStream_t stream)
{
    if (!a) return MARLIN_ERR_NULL_POINTER;
    if (!shape_ok(a->B, 1, 1, 64, a->pages, a->page_size, a->width) || a->table_row < 0 || a->tokens < 0 || a->tokens > kMaxTokens)
        return MARLIN_ERR_INVALID_SHAPE;
    if (a->B > 1 && a->table_row < a->width) return MARLIN_ERR_INVALID_SHAPE;  // rows that are written must not overlap
    if (!visible_ok(a->window, a->sinks)) return MARLIN_ERR_INVALID_ARGUMENT;
    if ((a->B > 0 && (!a->table || !a->lengths || !a->new_tokens)) || !a->free_pages || !a->free_count || !a->starts ||
        (a->tokens > 0 && !a->slots) || !a->workspace)
        return MARLIN_ERR_NULL_POINTER;
    if (!aligned(a->table, 4) || !aligned(a->lengths, 4) || !aligned(a->new_tokens, 4) || !aligned(a->free_pages, 4) ||
        !aligned(a->free_count, 4) || !aligned(a->starts, 4) || !aligned(a->slots, 8) || !aligned16(a->workspace) ||
        !aligned(a->back, 4))
        return MARLIN_ERR_MISALIGNED;
    if (a->workspace_bytes < marlin_assign_pages_workspace_bytes(a->B)) return MARLIN_ERR_WORKSPACE_TOO_SMALL;
    PagesProblem p;
    p.table = a->table;
    p.table_row = a->table_row;
    p.lengths = a->lengths;
    p.new_tokens = a->new_tokens;
    p.free_pages = a->free_pages;
    p.free_count = a->free_count;
    p.starts = a->starts;
    p.slots = a->slots;
    p.back = a->back;
    p.before = (int32_t *)((char *)a->workspace + kCounterRegionBytes);
    p.B = (int)a->B;
    p.width = (int)a->width;
    p.pages = (int)a->pages;
    p.page_shift = shift_of(a->page_size);
    p.tokens = (int)a->tokens;
    p.window = (int)a->window;
    p.sinks = (int)a->sinks;
    return launch_pages(p, stream) == hipSuccess ? MARLIN_OK : MARLIN_ERR_HIP;
}

}  // extern "C"
