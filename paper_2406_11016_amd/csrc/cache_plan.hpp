// Host planning of the key/value cache's operators: argument checks, the
// attention's split into tasks and its workspace.  No GPU needed.
#pragma once

#include <limits.h>
#include <stddef.h>
#include <stdint.h>

#include <initializer_list>

#include "spec_cache.h"

namespace sv {

// batch * max_new up to which the plan's one workgroup writes the slots itself.
// (On the GPU 5.3, 6.0, 7.6, 11.4 and 34 us for 64 sequences of 32, 64, 128, 256 and
// 1,000 tokens, and 7.0, 6.9, 7.0, 7.2 and 10.8 with a second kernel; a call that is
// not replayed in a graph pays 2 us more for the second launch.)
constexpr int64_t kPlanOwnSlots = 8192;

// Workgroups of the append at most.  (65,536 tokens of 8 heads of 128: 70 us, and 78
// with 8,192; 16,384 tokens and fewer take the same with either.)
constexpr uint32_t kAppendBlocks = 32768;

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

inline bool strides_ok(const int64_t (&s)[3]) {
    for (int64_t x : s)
        if (x < 0 || x % 8 != 0) return false;
    return true;
}

// A tensor that is written: no two of its rows begin at the same place.
inline bool rows_apart(const int64_t (&s)[3], int32_t batch, int32_t tokens, int32_t heads) {
    return (batch == 1 || s[0] != 0) && (tokens == 1 || s[1] != 0) && (heads == 1 || s[2] != 0);
}

inline bool page_size_ok(int32_t p) { return p >= 16 && p <= 1024 && (p & (p - 1)) == 0; }

inline int32_t page_shift(int32_t p) { return __builtin_ctz((unsigned)p); }

// Slots, table places and a sequence's tokens all fit an int32.
inline bool cache_table_sizes_ok(int32_t batch, int32_t max_pages, int32_t num_pages, int32_t page_size) {
    return batch >= 1 && batch <= SV_CACHE_MAX_BATCH && max_pages >= 1 && num_pages >= 1 && page_size_ok(page_size) &&
           (int64_t)num_pages * page_size <= INT_MAX && (int64_t)max_pages * page_size <= INT_MAX &&
           (int64_t)batch * max_pages <= INT_MAX;
}

inline sv_status_t check_cache(sv_dtype_t dtype, int32_t batch, int32_t max_new, int32_t kv_heads, int32_t head_dim,
                               int32_t num_pages, int32_t page_size, int64_t page_stride) {
    if (dtype != SV_F16 && dtype != SV_BF16) return SV_ERR_DTYPE;
    if (batch < 1 || batch > SV_CACHE_MAX_BATCH || max_new < 1 || (int64_t)batch * max_new > INT_MAX || kv_heads < 1 ||
        kv_heads > 65536 || head_dim < 8 || head_dim > 4096 || head_dim % 8 != 0 || num_pages < 1 ||
        !page_size_ok(page_size) || (int64_t)num_pages * page_size > INT_MAX)
        return SV_ERR_SHAPE;
    if (page_stride < (int64_t)kv_heads * page_size * head_dim || page_stride % 8 != 0) return SV_ERR_PARAM;
    return SV_OK;
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------

// Keys of a unit of work: what a workgroup holds of K and V twice, the unit it
// computes and the one on its way.
constexpr int kAttendKeys = 64;

// What a workgroup's start and end with a task cost it, in units: tasks count that
// many units more where work is dealt out.  (2 to 8 differ by 2 % without a prefix; behind
// a long one 5, 6 and 8 take 5 to 8 % longer.)
constexpr uint32_t kTaskUnits = 3;

// How a call's work is cut (see cache_attend.hpp).
struct AttendPlan {
    // joined: a task runs over the prefix and then over its sequence's keys, and
    // only tasks cut by a workgroup's border have parts.  Otherwise the prefix
    // has tasks of its own, for the rows of the whole batch.
    bool joined;
    int32_t own_rows, own_tiles;  // rows of a sequence's own task (32, 64 or 128); tasks a key/value head
    int32_t prefix_rows;          // rows of a prefix task
    int32_t own_shift, prefix_shift;  // their logarithms
    int32_t groups;               // workgroups
    int64_t own_parts, rows;      // row places of the parts: of the first own one, of all
    size_t cum_bytes;             // one array of sums over the batch
};

constexpr size_t kTotalsBytes = 256;  // room in the workspace for the split's totals, see cache_split.hpp

inline bool head_dim_ok(int32_t d) { return d == 64 || d == 80 || d == 96 || d == 128 || d == 256; }

// Rows of a task: 32 for each wave that has rows of its own.  At head_dim 256 two
// waves of the four: four would need more registers than there are.  (64 sequences of
// 2,000 keys at head_dim 128: 4 to 32 rows take 99 to 102 us, 102 to 104 in tasks of 64
// and 108 to 114 of 128; 48 or 64 rows 106, and 115 of 128 or 189 of 32; at head_dim 256
// 8 to 32 rows 37 to 43, and 45 to 51 of 64.)
inline int32_t task_rows(int64_t rows, int32_t head_dim) {
    return rows <= 32 ? 32 : rows <= 64 || head_dim > 128 ? 64 : 128;
}

// Whether the sequences' own tasks run over the prefix themselves: their row tiles
// are of the largest size and nearly full, so that sharing would save no products,
// and there are enough of them, so that few have to be cut and have parts.  (Time so
// to time with the prefix's rows pooled, prefixes of 2,000 to 16,384: tiles full, a
// task for two workgroups, 0.83 to 0.93 at head_dim 128, 0.93 at 256; tiles full, one
// for four, 1.10 and 1.07; tiles 7/8 full, a task or more a workgroup, 0.74 to 0.91;
// tiles 3/4 full, 0.79 to 1.08; 9/16 full, 0.94 to 1.44.)
constexpr bool joined_pays(int64_t tasks, int64_t groups, int64_t rows, int64_t tile_rows) {
    return 2 * tasks >= groups && 8 * rows >= 7 * ((rows + tile_rows - 1) / tile_rows * tile_rows);
}

inline AttendPlan attend_plan(int32_t batch, int32_t max_new, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                              bool prefix) {
    AttendPlan p{};
    const int64_t group = q_heads / kv_heads, rows = max_new * group;
    p.own_rows = task_rows(rows, head_dim);
    p.own_tiles = (int32_t)((rows + p.own_rows - 1) / p.own_rows);
    p.prefix_rows = task_rows(batch * rows, head_dim);
    p.own_shift = __builtin_ctz((unsigned)p.own_rows);
    p.prefix_shift = __builtin_ctz((unsigned)p.prefix_rows);
    p.groups = head_dim > 128 ? 256 : 512;  // what the 256 CUs hold at a time: one of 128 KiB LDS each, or two of 64
    p.joined = !prefix || joined_pays((int64_t)batch * kv_heads * p.own_tiles, p.groups, rows, task_rows(1 << 20, head_dim));
    if (p.joined) {
        p.own_parts = 0;
        p.rows = 2 * (int64_t)p.groups * p.own_rows;
    } else {
        const int64_t prefix_tasks = kv_heads * ((batch * rows + p.prefix_rows - 1) / p.prefix_rows);
        // (chunks of the prefix have at least a workgroup's share of its units, see Totals: at most `groups` tasks more)
        p.own_parts = (prefix_tasks + 3 * p.groups + 1) * p.prefix_rows;
        p.rows = p.own_parts + ((int64_t)batch * kv_heads * p.own_tiles + p.groups) * p.own_rows;
    }
    p.cum_bytes = (sizeof(int32_t) * ((size_t)batch + 1) + 255) / 256 * 256;
    return p;
}

inline bool attend_sizes_ok(int32_t batch, int32_t max_new, int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
    return batch >= 1 && batch <= SV_CACHE_MAX_BATCH && max_new >= 1 && kv_heads >= 1 && q_heads >= kv_heads &&
           q_heads <= 65536 && q_heads % kv_heads == 0 && head_dim_ok(head_dim) &&
           (head_dim <= 128 || batch <= SV_CACHE_MAX_BATCH_D256) &&
           (int64_t)batch * max_new <= INT_MAX && (int64_t)batch * max_new * q_heads <= INT_MAX;
}

// The numbers of units (with what the tasks cost) fit 31 bits at the longest sequences that the table can name.
inline bool attend_units_ok(const sv_cache_attend_desc_t& d, const AttendPlan& p) {
    const int64_t pre = ((int64_t)d.prefix_len + kAttendKeys - 1) / kAttendKeys;
    const int64_t own = ((int64_t)d.max_pages * d.page_size + kAttendKeys - 1) / kAttendKeys;
    const double tiles = (double)d.batch * d.kv_heads * p.own_tiles;
    const double rows = (double)d.batch * d.max_new * (d.q_heads / d.kv_heads);
    // (a chunk of the prefix has a unit at least)
    const double pooled = p.joined ? 0.0 : d.kv_heads * (double)pre * (1 + kTaskUnits) * (rows / p.prefix_rows + 1.0);
    return tiles * (double)(own + kTaskUnits + (p.joined ? pre : 0)) + pooled < 2147483647.0;
}

inline size_t attend_workspace_bytes(int32_t batch, int32_t max_new, int32_t q_heads, int32_t kv_heads,
                                     int32_t head_dim) {
    if (!attend_sizes_ok(batch, max_new, q_heads, kv_heads, head_dim)) return 0;
    size_t most = 0;
    for (const bool prefix : {false, true}) {
        const AttendPlan p = attend_plan(batch, max_new, q_heads, kv_heads, head_dim, prefix);
        const size_t n = 2 * p.cum_bytes + kTotalsBytes + (size_t)p.rows * ((size_t)head_dim + 2) * sizeof(float);
        if (n > most) most = n;
    }
    return (most + 255) / 256 * 256;
}

inline sv_status_t check_attend(const sv_cache_attend_desc_t& d) {
    if (d.q == nullptr || d.out == nullptr || d.k_cache == nullptr || d.v_cache == nullptr || d.block_table == nullptr ||
        d.lengths == nullptr || d.workspace == nullptr || (d.prefix_len != 0 && d.prefix_table == nullptr))
        return SV_ERR_NULL;
    const sv_status_t st = check_cache(d.dtype, d.batch, d.max_new, d.kv_heads, d.head_dim, d.num_pages, d.page_size,
                                       d.page_stride);
    if (st != SV_OK) return st;
    if (!attend_sizes_ok(d.batch, d.max_new, d.q_heads, d.kv_heads, d.head_dim) || d.max_pages < 1 ||
        (int64_t)d.batch * d.max_pages > INT_MAX || (int64_t)d.max_pages * d.page_size > INT_MAX || d.prefix_len < 0 ||
        (int64_t)d.prefix_len + (int64_t)d.max_pages * d.page_size > INT_MAX)
        return SV_ERR_SHAPE;
    if (!attend_units_ok(d, attend_plan(d.batch, d.max_new, d.q_heads, d.kv_heads, d.head_dim, d.prefix_len > 0)))
        return SV_ERR_SHAPE;
    // (scale * log2(e) and its inverse have to be finite)
    if (!(d.scale > 1e-30f && d.scale < 1e30f)) return SV_ERR_PARAM;
    if (!aligned16(d.q) || !aligned16(d.out) || !aligned16(d.k_cache) || !aligned16(d.v_cache) ||
        !strides_ok(d.q_stride) || !strides_ok(d.out_stride) ||
        !rows_apart(d.out_stride, d.batch, d.max_new, d.q_heads))
        return SV_ERR_PARAM;
    if (!aligned16(d.workspace) ||
        d.workspace_bytes < attend_workspace_bytes(d.batch, d.max_new, d.q_heads, d.kv_heads, d.head_dim))
        return SV_ERR_WORKSPACE;
    return SV_OK;
}

}  // namespace sv
