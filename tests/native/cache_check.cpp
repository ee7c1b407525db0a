// Host-side checks of the key/value cache's operators (cache_plan.hpp,
// cache_split.hpp), built on the CPU with -fsanitize=address,undefined
// (tests/test_cache_native.py builds and runs it).
//
//   1. The attention's split, simulated workgroup by workgroup over random
//      batches: every unit of every task is computed once, every part lies in
//      the workspace and overlaps no other, every row finds exactly the parts
//      that hold its keys, and every key that is staged has its page inside the
//      tables.
//   2. Argument validation: the error contract of spec_cache.h.
//
// Prints one line per section and exits nonzero on the first failure.
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <map>
#include <random>
#include <vector>

#include "cache_split.hpp"

using namespace sv;

static long long g_checks = 0;

#define CHECK(cond, ...)                                                       \
    do {                                                                       \
        ++g_checks;                                                            \
        if (!(cond)) {                                                         \
            fprintf(stderr, "FAILED %s:%d: %s: ", __FILE__, __LINE__, #cond);  \
            fprintf(stderr, __VA_ARGS__);                                      \
            fprintf(stderr, "\n");                                             \
            exit(1);                                                           \
        }                                                                      \
    } while (0)

struct Case {
    int32_t batch, max_new, q_heads, kv_heads, head_dim, page_size, max_pages, prefix_len;
    std::vector<int32_t> lengths, counts;
};

static int32_t find_tile_host(const Split& a, const Sequence& s, uint32_t at, uint32_t& start) {
    start = 0;
    for (int32_t rt = 0; rt < a.plan.own_tiles; ++rt) {
        const uint32_t n = tile_cost(a, s, rt);
        if (at < start + n) return rt;
        start += n;
    }
    CHECK(false, "unit %u behind the last tile", at);
    return -1;
}

struct Got {
    uint32_t first, end;
    int64_t place;
};

static void simulate(const Case& c, int id) {
    sv_cache_attend_desc_t d{};
    d.lengths = c.lengths.data();
    d.counts = c.counts.empty() ? nullptr : c.counts.data();
    d.batch = c.batch;
    d.max_new = c.max_new;
    d.q_heads = c.q_heads;
    d.kv_heads = c.kv_heads;
    d.head_dim = c.head_dim;
    d.max_pages = c.max_pages;
    d.page_size = c.page_size;
    d.prefix_len = c.prefix_len;
    const AttendPlan plan = attend_plan(c.batch, c.max_new, c.q_heads, c.kv_heads, c.head_dim, c.prefix_len > 0);
    CHECK(attend_units_ok(d, plan), "case %d", id);
    const size_t bytes = attend_workspace_bytes(c.batch, c.max_new, c.q_heads, c.kv_heads, c.head_dim);
    CHECK(sizeof(Totals) <= kTotalsBytes && 2 * plan.cum_bytes + kTotalsBytes + (size_t)plan.rows * (c.head_dim + 2) * 4 <= bytes, "case %d", id);
    CHECK(plan.cum_bytes % 16 == 0 && plan.rows % 4 == 0, "case %d", id);  // the parts lie on 16 bytes
    const Split a = make_split(d, plan);
    std::vector<int32_t> cum_tokens(c.batch + 1, 0);
    std::vector<uint32_t> cum_cost(c.batch + 1, 0);
    for (int32_t b = 0; b < c.batch; ++b) {
        const Sequence s = sequence(a, b);
        cum_tokens[b + 1] = cum_tokens[b] + s.count;
        uint32_t cost = 0;
        for (int32_t rt = 0; rt < plan.own_tiles; ++rt) cost += tile_cost(a, s, rt);
        cum_cost[b + 1] = cum_cost[b] + cost * (uint32_t)c.kv_heads;
    }
    const Totals t = totals(a, cum_tokens[c.batch], cum_cost[c.batch]);
    // the segments of each task, in order: by (prefix's?, task)
    std::map<std::pair<bool, uint32_t>, std::vector<Got>> got;
    std::map<std::pair<bool, uint32_t>, Segment> tasks;
    std::vector<std::pair<int64_t, int64_t>> places;
    std::map<std::pair<bool, uint32_t>, uint32_t> done;  // units of each task
    CHECK(t.prefix.groups + t.own.groups <= (uint32_t)plan.groups, "case %d", id);
    CHECK(t.chunk <= (uint32_t)a.prefix_units || t.prefix.cost == 0, "case %d", id);
    CHECK((t.prefix.cost == 0) == (plan.joined || t.tokens == 0), "case %d", id);
    for (const bool shared : {true, false}) {
    const Deal& d = shared ? t.prefix : t.own;
    uint32_t covered = 0;
    for (uint32_t w = 0; w < d.groups; ++w) {
        const uint32_t end = group_start(d, w + 1);
        uint32_t u = group_start(d, w);
        CHECK(u == covered && u < end, "case %d: group %u", id, w);
        covered = end;
        while (u < end) {
            CHECK(group_of(d, u) == w, "case %d: unit %u", id, u);
            Segment g = shared ? prefix_task(a, t, u)
                               : own_task(
                                     a, cum_cost.data(), u, [&](int32_t b) { return sequence(a, b); },
                                     [&](const Sequence& s, uint32_t at, uint32_t& start) {
                                         return find_tile_host(a, s, at, start);
                                     });
            CHECK((g.b < 0) == shared, "case %d", id);
            CHECK(u + kTaskUnits >= g.task_start && u < g.task_start + g.units && g.units > 0, "case %d: unit %u", id, u);
            cut(g, u, end);
            if (g.first == g.end) break;
            CHECK(g.first < g.end && g.end <= g.units && g.first == done[std::make_pair(g.b < 0, g.task)], "case %d", id);
            done[std::make_pair(g.b < 0, g.task)] = g.end;
            const int32_t rows = g.b < 0 ? plan.prefix_rows : plan.own_rows;
            if (!whole_task(a, g)) {
                const int64_t place = part_place(a, g, w);
                CHECK(place >= 0 && place + rows <= plan.rows, "case %d: place %lld", id, (long long)place);
                places.push_back({place, place + rows});
                got[{g.b < 0, g.task}].push_back({g.first, g.end, place});
            }
            tasks[{g.b < 0, g.task}] = g;
            for (uint32_t k = g.offset + g.first; k < g.offset + g.end; ++k) {
                const bool pre = k < g.prefix_units;
                const int32_t base = (int32_t)(pre ? k : k - g.prefix_units) * kAttendKeys;
                const int32_t last = pre ? c.prefix_len - 1 : own_end(a, g) - 1;
                CHECK(base <= last, "case %d: an empty unit", id);
                for (int32_t r = 0; r < kAttendKeys / 16; ++r) {
                    const int32_t first = run_start(base, r, last);
                    CHECK(first >= 0 && first <= last && first % 16 == 0, "case %d", id);
                    CHECK(first == base + 16 * r || base + 16 * r > last, "case %d", id);
                    if (pre)
                        CHECK((first >> a.page_shift) < (c.prefix_len + c.page_size - 1) / c.page_size, "case %d", id);
                    else if (!g.bad)
                        CHECK((first >> a.page_shift) < c.max_pages, "case %d: key %d", id, first);
                }
            }
            u = g.task_start + g.end;
        }
    }
    CHECK(covered == d.cost, "case %d", id);
    }
    for (const auto& x : tasks) CHECK(done[x.first] == x.second.units, "case %d: a task not done", id);
    std::sort(places.begin(), places.end());
    for (size_t i = 1; i < places.size(); ++i) CHECK(places[i - 1].second <= places[i].first, "case %d", id);

    // what the joining kernels look up, row by row
    auto same = [&](const Parts& p, const std::vector<Got>& have, size_t from, int32_t in_tile) {
        for (int32_t k = 0; k < p.n; ++k) {
            CHECK(from + k < have.size(), "case %d", id);
            CHECK(p.first + k * p.step == have[from + k].place + in_tile, "case %d: part %d", id, k);
        }
    };
    for (int32_t b = 0; b < c.batch; ++b) {
        const Sequence s = sequence(a, b);
        for (int32_t token = 0; token < s.count; ++token)
            for (int32_t kv = 0; kv < c.kv_heads; ++kv)
                for (int32_t h = 0; h < a.group; ++h) {
                    const int32_t r = token * a.group + h, tile = r / plan.own_rows;
                    const uint32_t task = (uint32_t)(b * c.kv_heads + kv) * plan.own_tiles + tile;
                    const auto it = tasks.find({false, task});
                    CHECK(it != tasks.end(), "case %d: a row without a task", id);
                    const Segment& g = it->second;
                    CHECK(g.b == b && g.kv_head == kv && g.row0 <= r && r < g.row0 + plan.own_rows, "case %d", id);
                    // its keys: all of them, and none of a later unit
                    const uint32_t need = (uint32_t)(s.length + token) / kAttendKeys + 1;
                    CHECK(g.units - g.prefix_units >= need, "case %d", id);
                    CHECK(own_common(a, g) <= s.length + token + 1 && s.length + token < own_end(a, g), "case %d", id);
                    if (!plan.joined) {
                        const int32_t flat = (cum_tokens[b] + token) * a.group + h;
                        uint32_t keys = 0;  // units of the prefix that its parts hold
                        for (uint32_t chunk = 0; chunk < t.chunks; ++chunk) {
                            const uint32_t ptask =
                                (chunk * (uint32_t)c.kv_heads + kv) * t.prefix_tiles + flat / plan.prefix_rows;
                            const auto& have = got[std::make_pair(true, ptask)];
                            CHECK(have.size() == 1 || have.size() == 2, "case %d", id);
                            CHECK(tasks.at({true, ptask}).offset == keys, "case %d", id);
                            for (uint32_t k = 0; k < 2; ++k) {
                                const int64_t place = prefix_part(a, t, kv, flat, 2 * chunk + k);
                                CHECK((place >= 0) == (k < have.size()), "case %d", id);
                                if (place < 0) continue;
                                CHECK(place == have[k].place + flat % plan.prefix_rows, "case %d", id);
                                keys += have[k].end - have[k].first;
                            }
                        }
                        CHECK(keys == (uint32_t)a.prefix_units, "case %d", id);
                        const Parts op =
                            own_parts(a, t, s, cum_cost[b], cum_cost[b + 1] - cum_cost[b], b, token, kv, h);
                        CHECK((size_t)op.n == got[std::make_pair(false, task)].size(), "case %d", id);
                        same(op, got[std::make_pair(false, task)], 0, r % plan.own_rows);
                    } else if (got.count({false, task})) {
                        const auto& have = got[std::make_pair(false, task)];
                        uint32_t w0 = 0, w1 = 0;
                        CHECK(cuts_task(t, g, group_of(t.own, g.task_start) + 1, w0, w1), "case %d", id);
                        CHECK(w1 > w0 && have.size() == w1 - w0 + 1, "case %d", id);
                        same(first_cut_part(a, w0, r % plan.own_rows), have, 0, r % plan.own_rows);
                        same(later_cut_parts(a, w0, w1, r % plan.own_rows), have, 1, r % plan.own_rows);
                        // the workgroups of the joining kernel that take it, and no other
                        uint32_t borders = 0;
                        for (uint32_t w = 1; w < t.own.groups && r % plan.own_rows == 0; ++w) {
                            const uint32_t u = group_start(t.own, w);
                            if (u + kTaskUnits < g.task_start || u >= g.task_start + g.units) continue;
                            uint32_t x0, x1;
                            CHECK(cuts_task(t, g, w, x0, x1) == (w > w0 && w <= w1), "case %d", id);
                            if (cuts_task(t, g, w, x0, x1)) {
                                CHECK(x0 == w0 && x1 == w1, "case %d", id);
                                ++borders;
                            }
                        }
                        CHECK(r % plan.own_rows != 0 || borders == w1 - w0, "case %d", id);
                    } else {
                        CHECK(group_of(t.own, g.task_start) == group_of(t.own, g.task_start + g.units - 1), "case %d", id);
                    }
                }
    }
}

static void section_split() {
    std::mt19937 rng(7);
    auto pick = [&](int lo, int hi) { return (int32_t)(lo + (int)(rng() % (unsigned)(hi - lo + 1))); };
    const int32_t dims[] = {64, 80, 96, 128, 256};
    int cases = 0;
    for (int i = 0; i < 1500; ++i) {
        Case c{};
        c.batch = pick(0, 9) == 0 ? pick(200, 400) : pick(1, 40);
        c.kv_heads = pick(1, 8);
        c.q_heads = c.kv_heads * pick(1, 9);
        c.head_dim = dims[pick(0, 4)];
        c.page_size = 16 << pick(0, 6);
        c.max_new = pick(0, 3) == 0 ? pick(1, 300) : pick(1, 21);
        if ((int64_t)c.batch * c.max_new * c.q_heads > 20000) c.batch = std::max(1, 20000 / (c.max_new * c.q_heads));
        const int32_t longest = pick(0, 3) == 0 ? pick(1, 60000) : pick(1, 2000);
        c.max_pages = (longest + c.max_new + c.page_size - 1) / c.page_size;
        c.prefix_len = pick(0, 2) == 0 ? 0 : pick(0, 1) ? pick(1, 300) : pick(1, 20000);
        const bool with_counts = pick(0, 2) != 0;
        for (int32_t b = 0; b < c.batch; ++b) {
            c.lengths.push_back(pick(0, 3) == 0 ? 0 : pick(0, longest));
            if (with_counts) c.counts.push_back(pick(0, 5) == 0 ? pick(-1, 0) : pick(1, c.max_new));
            if (pick(0, 60) == 0) c.lengths.back() = pick(0, 1) ? -5 : c.max_pages * c.page_size;      // bad
            if (with_counts && pick(0, 60) == 0) c.counts.back() = c.max_new + 1;                      // bad
        }
        simulate(c, i);
        ++cases;
    }
    // tasks that run over the prefix themselves: many, of nearly full row tiles
    for (int i = 0; i < 40; ++i) {
        Case c{};
        c.head_dim = dims[pick(0, 4)];
        c.kv_heads = pick(1, 8);
        c.q_heads = c.kv_heads * pick(1, 4);
        c.page_size = 64;
        c.max_new = 128 / (c.q_heads / c.kv_heads) * pick(1, 3);
        c.batch = 256 / c.kv_heads + pick(1, 9);
        c.max_pages = 20;
        c.prefix_len = pick(1, 2000);
        for (int32_t b = 0; b < c.batch; ++b) {
            c.lengths.push_back(pick(0, 500));
            c.counts.push_back(pick(0, 5) == 0 ? pick(-1, 3) : pick(c.max_new - 5, c.max_new));
        }
        CHECK(attend_plan(c.batch, c.max_new, c.q_heads, c.kv_heads, c.head_dim, true).joined, "joined case %d", i);
        simulate(c, 10000 + i);
        ++cases;
    }
    // nothing to do at all
    Case c{3, 4, 8, 2, 64, 16, 8, 100, {1, 2, 3}, {0, -1, 0}};
    simulate(c, -1);
    printf("split: %d batches\n", cases);
}

static sv_cache_attend_desc_t good() {
    sv_cache_attend_desc_t d{};
    d.q = (const void*)0x1000;
    d.out = (void*)0x2000;
    for (int i = 0; i < 3; ++i) d.q_stride[i] = d.out_stride[i] = 1024;
    d.k_cache = (const void*)0x3000;
    d.v_cache = (const void*)0x4000;
    d.page_stride = 2 * 16 * 128;
    d.block_table = (const int32_t*)0x5000;
    d.lengths = (const int32_t*)0x6000;
    d.prefix_table = (const int32_t*)0x7000;
    d.prefix_len = 5;
    d.dtype = SV_BF16;
    d.batch = 2;
    d.max_new = 3;
    d.q_heads = 8;
    d.kv_heads = 2;
    d.head_dim = 128;
    d.max_pages = 4;
    d.num_pages = 10;
    d.page_size = 16;
    d.scale = 0.1f;
    d.workspace = (void*)0x8000;
    d.workspace_bytes = attend_workspace_bytes(2, 3, 8, 2, 128);
    return d;
}

static void section_arguments() {
    CHECK(check_attend(good()) == SV_OK, "good");
    auto bad = [&](sv_status_t want, auto&& edit, const char* what) {
        sv_cache_attend_desc_t d = good();
        edit(d);
        CHECK(check_attend(d) == want, "%s: %d", what, (int)check_attend(d));
    };
#define BAD(want, edit) bad(want, [](sv_cache_attend_desc_t& d) { edit; }, #edit)
    BAD(SV_ERR_NULL, d.q = nullptr);
    BAD(SV_ERR_NULL, d.out = nullptr);
    BAD(SV_ERR_NULL, d.k_cache = nullptr);
    BAD(SV_ERR_NULL, d.v_cache = nullptr);
    BAD(SV_ERR_NULL, d.block_table = nullptr);
    BAD(SV_ERR_NULL, d.lengths = nullptr);
    BAD(SV_ERR_NULL, d.prefix_table = nullptr);
    BAD(SV_ERR_NULL, d.workspace = nullptr);
    BAD(SV_OK, d.prefix_table = nullptr; d.prefix_len = 0);
    BAD(SV_ERR_DTYPE, d.dtype = SV_F32);
    BAD(SV_ERR_DTYPE, d.dtype = (sv_dtype_t)9);
    BAD(SV_ERR_SHAPE, d.batch = 0);
    BAD(SV_ERR_SHAPE, d.batch = SV_CACHE_MAX_BATCH + 1);
    BAD(SV_ERR_SHAPE, d.head_dim = 256; d.page_stride = 2 * 16 * 256; d.batch = SV_CACHE_MAX_BATCH_D256 + 1);
    BAD(SV_ERR_WORKSPACE, d.head_dim = 256; d.page_stride = 2 * 16 * 256; d.batch = SV_CACHE_MAX_BATCH_D256);
    BAD(SV_ERR_SHAPE, d.max_new = 0);
    BAD(SV_ERR_SHAPE, d.max_new = 1 << 30);
    BAD(SV_ERR_SHAPE, d.kv_heads = 0);
    BAD(SV_ERR_SHAPE, d.q_heads = 7);
    BAD(SV_ERR_SHAPE, d.q_heads = 0);
    BAD(SV_ERR_SHAPE, d.head_dim = 72);
    BAD(SV_ERR_SHAPE, d.head_dim = 112);
    BAD(SV_ERR_SHAPE, d.page_size = 24; d.page_stride = 1 << 20);
    BAD(SV_ERR_SHAPE, d.page_size = 8);
    BAD(SV_ERR_SHAPE, d.page_size = 2048; d.page_stride = 1 << 20);
    BAD(SV_ERR_SHAPE, d.num_pages = 0);
    BAD(SV_ERR_SHAPE, d.num_pages = 1 << 28);
    BAD(SV_ERR_SHAPE, d.max_pages = 0);
    BAD(SV_ERR_SHAPE, d.max_pages = 1 << 28);
    BAD(SV_ERR_SHAPE, d.prefix_len = -1);
    BAD(SV_ERR_SHAPE, d.prefix_len = INT_MAX);
    BAD(SV_ERR_PARAM, d.page_stride = 2 * 16 * 128 - 8);
    BAD(SV_ERR_PARAM, d.page_stride = 2 * 16 * 128 + 4);
    BAD(SV_ERR_PARAM, d.scale = 0.0f);
    BAD(SV_ERR_PARAM, d.scale = -1.0f);
    BAD(SV_ERR_PARAM, d.scale = __builtin_nanf(""));
    BAD(SV_ERR_PARAM, d.scale = __builtin_inff());
    BAD(SV_ERR_PARAM, d.q = (const void*)0x1008);
    BAD(SV_ERR_PARAM, d.out = (void*)0x2002);
    BAD(SV_ERR_PARAM, d.k_cache = (const void*)0x3004);
    BAD(SV_ERR_PARAM, d.v_cache = (const void*)0x4004);
    BAD(SV_ERR_PARAM, d.q_stride[1] = 129);
    BAD(SV_ERR_PARAM, d.out_stride[0] = -8);
    BAD(SV_ERR_WORKSPACE, d.workspace = (void*)0x8008);
    BAD(SV_ERR_WORKSPACE, d.workspace_bytes -= 1);
#undef BAD
    CHECK(attend_workspace_bytes(0, 1, 1, 1, 64) == 0 && attend_workspace_bytes(1, 0, 1, 1, 64) == 0 &&
              attend_workspace_bytes(1, 1, 3, 2, 64) == 0 && attend_workspace_bytes(1, 1, 1, 1, 65) == 0 &&
              attend_workspace_bytes(1, 1, 1, 0, 64) == 0 &&
              attend_workspace_bytes(SV_CACHE_MAX_BATCH_D256 + 1, 1, 1, 1, 256) == 0 &&
              attend_workspace_bytes(SV_CACHE_MAX_BATCH, 1, 1, 1, 128) != 0,
          "sizes");
    // the counts of units stay below 2^31, or the call is refused
    sv_cache_attend_desc_t d = good();
    d.batch = 4096;
    d.max_new = 512;
    d.q_heads = d.kv_heads = 1024;
    d.max_pages = 1 << 20;
    CHECK(!attend_units_ok(d, attend_plan(d.batch, d.max_new, d.q_heads, d.kv_heads, d.head_dim, true)), "units");
    CHECK(cache_table_sizes_ok(1, 1, 1, 16) && cache_table_sizes_ok(4096, 1000, 1 << 20, 1024), "tables");
    CHECK(!cache_table_sizes_ok(0, 1, 1, 16) && !cache_table_sizes_ok(4097, 1, 1, 16) &&
              !cache_table_sizes_ok(1, 0, 1, 16) && !cache_table_sizes_ok(1, 1, 0, 16) &&
              !cache_table_sizes_ok(1, 1, 1, 17) && !cache_table_sizes_ok(1, 1, 1 << 27, 16) &&
              !cache_table_sizes_ok(1, 1 << 27, 1, 16) && !cache_table_sizes_ok(4096, 1 << 20, 1, 16),
          "tables");
    printf("arguments\n");
}

int main() {
    section_split();
    section_arguments();
    printf("all checks passed (%lld)\n", g_checks);
    return 0;
}
