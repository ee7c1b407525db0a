// How the cache attention's work is cut, in the terms of cache_attend.hpp: rows
// and row tiles, units of keys, the workgroups' runs of units, and the places of
// the parts.  Plain constexpr C++17: the kernels call it, and so does a test
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
    const int32_t first = rt << a.plan.own_shift;
    if (first >= s.count * a.group) return 0;
    const int32_t last =
        smaller(s.count - 1, (int32_t)((uint32_t)(first + a.plan.own_rows - 1) / (uint32_t)a.group));
    const uint32_t own = ((uint32_t)s.length + (uint32_t)last + kAttendKeys) / kAttendKeys;
    return own + (a.plan.joined ? (uint32_t)a.prefix_units : 0u);
}
constexpr uint32_t tile_cost(const Split& a, const Sequence& s, int32_t rt) {
    const uint32_t n = tile_units(a, s, rt);
    return n == 0 ? 0 : n + a.plan.own_task_units;
}

// A cost dealt to workgroups in equal runs; the first `longer` have one more.
struct Deal {
    uint32_t cost, groups, each, longer;
};
constexpr Deal deal(uint32_t cost, uint32_t groups) {
    Deal d{cost, smaller(groups, cost), 0, 0};
    if (d.groups == 0) return d;
    d.each = cost / d.groups;
    d.longer = cost - d.each * d.groups;
    return d;
}
// Workgroup w's run begins at group_start(w); group_of is its inverse.
constexpr uint32_t group_start(const Deal& d, uint32_t w) { return w * d.each + smaller(w, d.longer); }
constexpr uint32_t group_of(const Deal& d, uint32_t u) {
    const uint32_t border = d.longer * (d.each + 1);
    return u < border ? u / (d.each + 1) : d.longer + (u - border) / d.each;
}

// The tasks: the shared prefix's, and each sequence's own in the order of sequence,
// head, row tile.  Each kind has workgroups of its own, by its cost, in every XCD: the
// prefix's wait for the matrix units and the others for memory, so a CU has some of
// both.
//
// The prefix is cut into chunks of a workgroup's share of its units, and its tasks are
// ordered by chunk, key/value head, row tile: workgroups next to each other then run
// over the same keys at the same time, for other rows, and find them in their XCD's
// L2.  Where chunks that are longer by no more than a task's cost make at most a task a
// workgroup, they are, and there are as many workgroups as tasks.  Their runs are equal
// all the same, so where the last chunk is a shorter one borders do cut tasks: 15 of
// 104 for 32 sequences of 4 rows a head behind 8,192, 279 of 432 for 64 of 36 behind 16,384.
// (With tasks over the whole prefix every workgroup was somewhere else in it:
// 18,432 rows and 16,384 keys read 1.07 GB from behind the L2s, and 0.40 GB so.)
struct Totals {
    int32_t tokens, prefix_tiles;  // prefix tiles of one key/value head
    uint32_t chunk, chunks;        // units of a chunk of the prefix; chunks
    Deal prefix, own;              // (the grid's first workgroups are the prefix's)
};
constexpr Totals totals(const Split& a, int32_t tokens, uint32_t own_cost) {
    Totals t{};
    t.tokens = tokens;
    const uint32_t groups = (uint32_t)a.plan.groups;
    if (!a.plan.joined && tokens > 0) {
        t.prefix_tiles =
            (int32_t)(((uint32_t)tokens * (uint32_t)a.group + (uint32_t)a.plan.prefix_rows - 1) >> a.plan.prefix_shift);
        const uint32_t tasks = (uint32_t)t.prefix_tiles * (uint32_t)a.kv_heads, units = (uint32_t)a.prefix_units;
        const uint32_t cost = tasks * (units + a.plan.prefix_task_units);
        // (as many in each of the 8 XCDs: 64 sequences of 64 to 144 rows at head_dim 256
        // behind 16,384 took 117, 140, 180 and 280 us so, 156, 170, 212 and 309 to the nearest number)
        const uint64_t weight = (uint64_t)cost * a.plan.prefix_weight;
        const uint32_t eighths = (uint32_t)((uint64_t)(groups / 8) * weight / (weight + own_cost));
        const uint32_t places = 8 * (eighths < 1 ? 1u : smaller(eighths, groups / 8 - 1));
        const uint32_t fair = smaller(units, (tasks * units + places - 1) / places), most = places / tasks;
        const uint32_t whole = most == 0 ? units : (units + most - 1) / most;
        const bool by_tasks = most != 0 && whole <= fair + a.plan.prefix_task_units;
        t.chunk = by_tasks ? whole : fair;
        t.chunks = (units + t.chunk - 1) / t.chunk;
        t.prefix = deal(tasks * (units + t.chunks * a.plan.prefix_task_units), by_tasks ? tasks * t.chunks : places);
    }
    t.own = deal(own_cost, groups - t.prefix.groups);
    return t;
}

// Tasks of the prefix, one chunk of it all, if every sequence has max_new tokens.
constexpr int64_t pooled_tasks(const Split& a) {
    return (int64_t)a.kv_heads * (((int64_t)a.batch * a.max_new * a.group + a.plan.prefix_rows - 1) >> a.plan.prefix_shift);
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
    uint32_t task_start, units;  // where its units begin in its kind's cost (behind what the task costs); its units
    uint32_t first, end;         // this run, within the task
    uint32_t offset;             // units of the prefix before the task's chunk
    uint32_t prefix_units;       // units of the prefix that the task begins with
    int32_t kv_head, b, row0;    // b < 0: the prefix, for rows of the whole batch
    int32_t count, length;       // of sequence b
    int32_t bad;                 // (a word, which stays in a scalar register)
};

// The prefix's task at place u of its cost.
constexpr Segment prefix_task(const Split& a, const Totals& t, uint32_t u) {
    Segment g{};
    const uint32_t tiles = (uint32_t)t.prefix_tiles, units = (uint32_t)a.prefix_units;
    const uint32_t tasks = tiles * (uint32_t)a.kv_heads, chunk_cost = (t.chunk + a.plan.prefix_task_units) * tasks;
    const uint32_t chunk = u / chunk_cost, in_chunk = u - chunk * chunk_cost;
    g.offset = chunk * t.chunk;
    g.units = smaller(t.chunk, units - g.offset);
    const uint32_t task = in_chunk / (g.units + a.plan.prefix_task_units);
    g.kv_head = (int32_t)(task / tiles);
    const uint32_t tile = task - (uint32_t)g.kv_head * tiles;
    g.task = chunk * tasks + task;
    g.task_start = u - (in_chunk - task * (g.units + a.plan.prefix_task_units)) + a.plan.prefix_task_units;
    g.prefix_units = units;
    g.row0 = (int32_t)tile << a.plan.prefix_shift;
    g.b = -1;
    return g;
}
// The sequences' own task at place u of their cost.  `sequence_of(b)` gives sequence
// b; `find_tile(sequence, at, start)` the row tile that holds place `at` of a sequence
// and head, and the place at which that tile's task begins.
template <class SequenceOf, class FindTile>
constexpr Segment own_task_of(const Split& a, const uint32_t* cum_cost, int32_t b, uint32_t u, SequenceOf sequence_of,
                              FindTile find_tile) {
    Segment g{};
    g.b = b;
    const Sequence s = sequence_of(g.b);
    const uint32_t base = cum_cost[g.b], head = (cum_cost[g.b + 1] - base) / (uint32_t)a.kv_heads;
    g.kv_head = (int32_t)((u - base) / head);
    uint32_t start = 0;
    const int32_t rt = find_tile(s, u - base - (uint32_t)g.kv_head * head, start);
    g.task = (uint32_t)(g.b * a.kv_heads + g.kv_head) * (uint32_t)a.plan.own_tiles + (uint32_t)rt;
    g.task_start = base + (uint32_t)g.kv_head * head + start + a.plan.own_task_units;
    g.units = tile_units(a, s, rt);
    g.prefix_units = a.plan.joined ? (uint32_t)a.prefix_units : 0u;
    g.row0 = rt << a.plan.own_shift;
    g.count = s.count;
    g.length = s.length;
    g.bad = s.bad ? 1 : 0;
    return g;
}
template <class SequenceOf, class FindTile>
constexpr Segment own_task(const Split& a, const uint32_t* cum_cost, uint32_t u, SequenceOf sequence_of,
                           FindTile find_tile) {
    return own_task_of(a, cum_cost, find(cum_cost, a.batch, u), u, sequence_of, find_tile);
}
// A workgroup's run of the task that it finds at place u of the cost, its run of the
// cost ending before place `end`; empty (first == end) if it ends before the task's units.
constexpr void cut(Segment& g, uint32_t u, uint32_t end) {
    g.first = u > g.task_start ? u - g.task_start : 0u;
    g.end = end > g.task_start ? smaller(g.units, end - g.task_start) : 0u;
}

// Where a call's tasks are left whole (AttendPlan::whole_tasks), a workgroup has those that begin in
// its run of the cost.  `g` is the task at place `at` of it: one that began before `at` was
// another's, and then `g` and `at` move to the next one (`task_at` gives the task at a place); false
// if there is none before `end`.
template <class TaskAt>
constexpr bool to_whole_task(const Split& a, Segment& g, uint32_t& at, uint32_t end, TaskAt task_at) {
    if (at + a.plan.own_task_units <= g.task_start) return true;
    at = g.task_start + g.units;
    if (at >= end) return false;
    g = task_at(at);
    return true;
}

// The keys of a unit that a wave stages are a run of 16, which lies within a page.
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

// Row place of a segment's part.  With a shared prefix every segment of every task
// has one: segments of a kind in order differ in their task or in their workgroup,
// and so in the sum of the two.  Without one only cut tasks have parts: a workgroup cuts at
// most the one that it begins in and the one that it ends in.
constexpr bool whole_task(const Split& a, const Segment& g) {
    return a.plan.joined && g.first == 0 && g.end == g.units;
}
constexpr int64_t part_place(const Split& a, const Segment& g, uint32_t w) {
    if (a.plan.joined) return (int64_t)(2 * w + (g.first == 0 ? 1u : 0u)) * a.plan.own_rows;
    return g.b < 0 ? (int64_t)(g.task + w) * a.plan.prefix_rows
                   : a.plan.own_parts + (int64_t)(g.task + w) * a.plan.own_rows;
}

// With a shared prefix: part k (0 .. kChunkParts chunks - 1) of row r of a key/value
// head's prefix rows, or -1 where its task has fewer.  (A chunk has no
// more units than a workgroup is dealt, so at most one border cuts its tasks.)
constexpr uint32_t kChunkParts = 2;
constexpr int64_t prefix_part(const Split& a, const Totals& t, int32_t kv_head, int32_t r, uint32_t k) {
    const uint32_t tiles = (uint32_t)t.prefix_tiles, tile = (uint32_t)r >> a.plan.prefix_shift;
    const uint32_t chunk = k / kChunkParts, offset = chunk * t.chunk;
    const uint32_t units = smaller(t.chunk, (uint32_t)a.prefix_units - offset);
    const uint32_t tasks = tiles * (uint32_t)a.kv_heads, in_chunk = (uint32_t)kv_head * tiles + tile;
    const uint32_t start = chunk * (t.chunk + a.plan.prefix_task_units) * tasks +
                           in_chunk * (units + a.plan.prefix_task_units) + a.plan.prefix_task_units;
    const uint32_t task = chunk * tasks + in_chunk;
    const uint32_t w = group_of(t.prefix, start) + (k - chunk * kChunkParts);
    if (w > group_of(t.prefix, start + units - 1)) return -1;
    return (int64_t)(task + w) * a.plan.prefix_rows + (r & (a.plan.prefix_rows - 1));
}

// The parts of one row: n of them, from place `first` on in steps.
struct Parts {
    int64_t first, step;
    int32_t n;
};
// With a shared prefix: a row's parts of its sequence's own task.
constexpr Parts own_parts(const Split& a, const Totals& t, const Sequence& s, uint32_t cost_before, uint32_t cost,
                          int32_t b, int32_t token, int32_t kv_head, int32_t g) {
    const int32_t r = token * a.group + g, tile = r >> a.plan.own_shift;
    uint32_t start = cost_before + (uint32_t)kv_head * (cost / (uint32_t)a.kv_heads) + a.plan.own_task_units;
    for (int32_t rt = 0; rt < tile; ++rt) start += tile_cost(a, s, rt);
    const uint32_t task = (uint32_t)(b * a.kv_heads + kv_head) * (uint32_t)a.plan.own_tiles + (uint32_t)tile;
    const uint32_t w0 = group_of(t.own, start), w1 = group_of(t.own, start + tile_units(a, s, tile) - 1);
    return Parts{a.plan.own_parts + (int64_t)(task + w0) * a.plan.own_rows + (r - (tile << a.plan.own_shift)),
                 a.plan.own_rows, (int32_t)(w1 - w0) + 1};
}

// Without one: whether the border before workgroup w (w > 0) cuts a task's units, and
// then the first and last of the workgroups that have parts of it (w0 < w <= w1).
constexpr bool cuts_task(const Totals& t, const Segment& g, uint32_t w, uint32_t& w0, uint32_t& w1) {
    w0 = group_of(t.own, g.task_start);
    w1 = group_of(t.own, g.task_start + g.units - 1);
    return group_start(t.own, w) > g.task_start;
}
// Row r of a task cut by the borders of workgroups w0 .. w1; the
// first one's part is its last segment's, the others' are their first ones'.
constexpr Parts first_cut_part(const Split& a, uint32_t w0, int32_t r) {
    return Parts{(int64_t)(2 * w0 + 1) * a.plan.own_rows + r, 0, 1};
}
constexpr Parts later_cut_parts(const Split& a, uint32_t w0, uint32_t w1, int32_t r) {
    return Parts{(int64_t)(2 * (w0 + 1)) * a.plan.own_rows + r, 2 * (int64_t)a.plan.own_rows, (int32_t)(w1 - w0)};
}

}  // namespace sv
