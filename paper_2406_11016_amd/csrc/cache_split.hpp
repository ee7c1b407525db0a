// How the cache attention's work is cut, in the terms of cache_attend.hip: rows
// and row tiles, units of keys, the workgroups' runs of units, and the places of
// the parts.  Plain constexpr C++17: the kernels call it, and so does a checker
// on the CPU (tests/native/cache_check.cpp).
#pragma once

#include <stdint.h>

#include "cache_plan.hpp"

namespace sv {

constexpr int32_t smaller(int32_t x, int32_t y) { return x < y ? x : y; }
constexpr uint32_t smaller(uint32_t x, uint32_t y) { return x < y ? x : y; }

// What a call is about, apart from its tensors.
struct Split {
    const int32_t* lengths;
    const int32_t* counts;
    int32_t batch, max_new, kv_heads, group;
    int32_t max_pages, page_shift;
    int32_t prefix_units;  // of kAttendKeys keys
    AttendPlan plan;
};

inline Split make_split(const sv_cache_attend_desc_t& d, const AttendPlan& plan) {
    return Split{d.lengths,
                 d.counts,
                 d.batch,
                 d.max_new,
                 d.kv_heads,
                 d.q_heads / d.kv_heads,
                 d.max_pages,
                 page_shift(d.page_size),
                 (d.prefix_len + kAttendKeys - 1) / kAttendKeys,
                 plan};
}

// The tokens of sequence b that take part, and its cached ones.  Data that
// cannot be right (`bad`) stands for rows without cached tokens, so that they can
// be written.
struct Sequence {
    int32_t count, length;
    bool bad;
};
constexpr Sequence sequence(const Split& a, int32_t b) {
    Sequence s{(a.counts != nullptr) ? a.counts[b] : a.max_new, a.lengths[b], false};
    s.bad = s.count > 0 && (s.count > a.max_new || s.length < 0 ||
                            (uint32_t)s.length + (uint32_t)s.count > (uint32_t)a.max_pages << a.page_shift);
    if (s.bad) s.length = 0;
    s.count = smaller(s.count, a.max_new);
    if (s.count < 0) s.count = 0;
    return s;
}

// Units of row tile rt of a sequence's own tasks (of each key/value head).
constexpr uint32_t tile_units(const Split& a, const Sequence& s, int32_t rt) {
    const int32_t first = rt * a.plan.own_rows;
    if (first >= s.count * a.group) return 0;
    const int32_t last = smaller(s.count - 1, (first + a.plan.own_rows - 1) / a.group);
    const uint32_t own = ((uint32_t)s.length + (uint32_t)last + kAttendKeys) / kAttendKeys;
    return own + (a.plan.joined ? (uint32_t)a.prefix_units : 0u);
}
constexpr uint32_t sequence_units(const Split& a, const Sequence& s) {
    uint32_t n = 0;
    for (int32_t rt = 0; rt < a.plan.own_tiles; ++rt) n += tile_units(a, s, rt);
    return n;
}

// The tasks in order: the shared prefix's (key/value head, then row tile), then
// each sequence's own (sequence, head, row tile).
struct Totals {
    int32_t tokens, prefix_tiles;  // prefix tiles of one key/value head
    uint32_t prefix_units, units;  // units of all prefix tasks; of all tasks
    uint32_t groups;               // workgroups that take part: each has a unit
};
constexpr Totals totals(const Split& a, int32_t tokens, uint32_t own_units) {
    Totals t{};
    t.tokens = tokens;
    t.prefix_tiles =
        a.plan.joined ? 0 : (int32_t)(((int64_t)tokens * a.group + a.plan.prefix_rows - 1) / a.plan.prefix_rows);
    t.prefix_units = (uint32_t)t.prefix_tiles * (uint32_t)a.prefix_units * (uint32_t)a.kv_heads;
    t.units = t.prefix_units + own_units;
    t.groups = smaller((uint32_t)a.plan.groups, t.units);
    return t;
}

// Workgroup w's run of units begins at group_start(w); group_of is its inverse.
constexpr uint32_t group_start(const Totals& t, uint32_t w) { return (uint32_t)((uint64_t)w * t.units / t.groups); }
constexpr uint32_t group_of(const Totals& t, uint32_t u) {
    return (uint32_t)((((uint64_t)u + 1) * t.groups - 1) / t.units);
}

// The last b of n with cum[b] <= x (cum[0] <= x < cum[n]).
template <class I>
constexpr int32_t find(const I* cum, int32_t n, I x) {
    int32_t lo = 0, hi = n - 1;
    while (lo < hi) {
        const int32_t mid = (lo + hi + 1) >> 1;
        if (cum[mid] <= x)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// A run of units of one task.
struct Segment {
    uint32_t task;               // number among the prefix's, or among the sequences' own tasks
    uint32_t task_start, units;  // the task's first unit (of all), and its units
    uint32_t first, end;         // this run, within the task
    uint32_t prefix_units;       // units of the prefix that the task begins with
    int32_t kv_head, b, row0;    // b < 0: the prefix, for rows of the whole batch
    int32_t count, length;       // of sequence b
    bool bad;
};

// The task of unit u.  `find_tile(sequence, at, start)` gives the row tile that
// holds unit `at` of a sequence and head, and the unit at which it starts.
template <class FindTile>
constexpr Segment locate(const Split& a, const Totals& t, const uint32_t* cum_units, uint32_t u, FindTile find_tile) {
    Segment g{};
    if (u < t.prefix_units) {
        g.task = u / (uint32_t)a.prefix_units;
        g.task_start = g.task * (uint32_t)a.prefix_units;
        g.units = g.prefix_units = (uint32_t)a.prefix_units;
        g.kv_head = (int32_t)(g.task / (uint32_t)t.prefix_tiles);
        g.row0 = (int32_t)(g.task - (uint32_t)g.kv_head * (uint32_t)t.prefix_tiles) * a.plan.prefix_rows;
        g.b = -1;
        return g;
    }
    const uint32_t v = u - t.prefix_units;
    g.b = find(cum_units, a.batch, v);
    const Sequence s = sequence(a, g.b);
    const uint32_t base = cum_units[g.b], own = (cum_units[g.b + 1] - base) / (uint32_t)a.kv_heads;
    g.kv_head = (int32_t)((v - base) / own);
    uint32_t start = 0;
    const int32_t rt = find_tile(s, v - base - (uint32_t)g.kv_head * own, start);
    g.task = (uint32_t)(g.b * a.kv_heads + g.kv_head) * (uint32_t)a.plan.own_tiles + (uint32_t)rt;
    g.task_start = t.prefix_units + base + (uint32_t)g.kv_head * own + start;
    g.units = tile_units(a, s, rt);
    g.prefix_units = a.plan.joined ? (uint32_t)a.prefix_units : 0u;
    g.row0 = rt * a.plan.own_rows;
    g.count = s.count;
    g.length = s.length;
    g.bad = s.bad;
    return g;
}

// The keys of a unit that a wave stages are two runs of 16, each within a page.
// Run r (0 .. kAttendKeys / 16 - 1) of a unit that begins at key `base`: its
// first key; behind the last key there is, the run that holds it.
constexpr int32_t run_start(int32_t base, int32_t r, int32_t last_key) {
    return smaller(base + 16 * r, last_key & ~15);
}
// Keys that every row of a sequence's task sees of it, and that some row sees.
constexpr int32_t own_common(const Split& a, const Segment& g) { return g.length + g.row0 / a.group + 1; }
constexpr int32_t own_end(const Split& a, const Segment& g) {
    return g.length + smaller(g.count - 1, (g.row0 + a.plan.own_rows - 1) / a.group) + 1;
}

// Row place of a segment's part.  With a shared prefix every task's every
// segment has one: segments in order differ in their task or in their workgroup,
// and so in the sum of the two.  Else only a cut task's have: a workgroup cuts at
// most the one that it begins in and the one that it ends in.
constexpr bool whole_task(const Split& a, const Segment& g) {
    return a.plan.joined && g.first == 0 && g.end == g.units;
}
constexpr int64_t part_place(const Split& a, const Segment& g, uint32_t w) {
    if (a.plan.joined) return (int64_t)(2 * w + (g.first == 0 ? 1u : 0u)) * a.plan.own_rows;
    return g.b < 0 ? (int64_t)(g.task + w) * a.plan.prefix_rows
                   : a.plan.own_parts + (int64_t)(g.task + w) * a.plan.own_rows;
}

// The parts of one row: n of them, from place `first` on in steps.
struct Parts {
    int64_t first, step;
    int32_t n;
};

// With a shared prefix: the row's parts of the prefix's task and of its sequence's own.
constexpr Parts prefix_parts(const Split& a, const Totals& t, int32_t tokens_before, int32_t token, int32_t kv_head,
                             int32_t g) {
    const int32_t r = (tokens_before + token) * a.group + g, tile = r / a.plan.prefix_rows;
    const uint32_t task = (uint32_t)kv_head * (uint32_t)t.prefix_tiles + (uint32_t)tile;
    const uint32_t start = task * (uint32_t)a.prefix_units;
    const uint32_t w0 = group_of(t, start), w1 = group_of(t, start + (uint32_t)a.prefix_units - 1);
    return Parts{(int64_t)(task + w0) * a.plan.prefix_rows + (r - tile * a.plan.prefix_rows), a.plan.prefix_rows,
                 (int32_t)(w1 - w0) + 1};
}
constexpr Parts own_parts(const Split& a, const Totals& t, const Sequence& s, uint32_t units_before, uint32_t units,
                          int32_t b, int32_t token, int32_t kv_head, int32_t g) {
    const int32_t r = token * a.group + g, tile = r / a.plan.own_rows;
    uint32_t start = t.prefix_units + units_before + (uint32_t)kv_head * (units / (uint32_t)a.kv_heads);
    for (int32_t rt = 0; rt < tile; ++rt) start += tile_units(a, s, rt);
    const uint32_t task = (uint32_t)(b * a.kv_heads + kv_head) * (uint32_t)a.plan.own_tiles + (uint32_t)tile;
    const uint32_t w0 = group_of(t, start), w1 = group_of(t, start + tile_units(a, s, tile) - 1);
    return Parts{a.plan.own_parts + (int64_t)(task + w0) * a.plan.own_rows + (r - tile * a.plan.own_rows),
                 a.plan.own_rows, (int32_t)(w1 - w0) + 1};
}

// Without one: row r of a task cut by the borders of workgroups w0 .. w1; the
// first one's part is its last segment's, the others' are their first ones'.
constexpr Parts first_cut_part(const Split& a, uint32_t w0, int32_t r) {
    return Parts{(int64_t)(2 * w0 + 1) * a.plan.own_rows + r, 0, 1};
}
constexpr Parts later_cut_parts(const Split& a, uint32_t w0, uint32_t w1, int32_t r) {
    return Parts{(int64_t)(2 * (w0 + 1)) * a.plan.own_rows + r, 2 * (int64_t)a.plan.own_rows, (int32_t)(w1 - w0)};
}

}  // namespace sv
