// The split of the attention over a cache in 4 bits (tests/test_cache4_tasks_native.py builds
// and runs it):
//
//   1. cache_check.cpp's simulation with what each kind's tasks cost in such a call's plan,
//      at the bounds themselves.
//   2. Tasks left whole: every task of every sequence and head is taken once, by the
//      workgroup in whose run it begins, with all of its units.
#include "cache_split.hpp"

#define attend_plan attend4_plan
#define attend_workspace_bytes attend4_workspace_bytes
#define kTaskUnits (g.b < 0 ? plan.prefix_task_units : plan.own_task_units)
#define main all_checks
#include "cache_check.cpp"
#undef main
#undef kTaskUnits
#undef attend_workspace_bytes
#undef attend_plan

static Case few_rows(std::mt19937& rng, int32_t longest, bool prefix) {
    auto pick = [&](int lo, int hi) { return (int32_t)(lo + (int)(rng() % (unsigned)(hi - lo + 1))); };
    const int32_t dims[] = {64, 80, 96, 128, 256};
    Case c{};
    c.head_dim = dims[pick(0, 4)];
    c.batch = pick(0, 2) == 0 ? pick(1, 4) : pick(0, 9) == 0 ? pick(300, 1000) : pick(1, 200);
    c.kv_heads = pick(1, 8);
    const int32_t most = (int32_t)direct_rows(c.head_dim), group = pick(1, 8);
    c.q_heads = c.kv_heads * group;
    c.max_new = pick(1, most / group);
    c.page_size = 16 << pick(0, 6);
    const int32_t tokens = pick(1, longest);
    c.max_pages = std::max(1, tokens / c.page_size);
    c.prefix_len = prefix ? pick(1, 9000) : 0;
    const bool with_counts = pick(0, 2) != 0;
    const int32_t room = std::max(0, c.max_pages * c.page_size - c.max_new);
    for (int32_t b = 0; b < c.batch; ++b) {
        c.lengths.push_back(pick(0, 3) == 0 ? 0 : pick(0, room));
        if (with_counts) c.counts.push_back(pick(0, 4) == 0 ? pick(-1, 0) : pick(1, c.max_new));
        if (pick(0, 60) == 0) c.lengths.back() = pick(0, 1) ? -5 : c.max_pages * c.page_size;  // bad
        if (with_counts && pick(0, 60) == 0) c.counts.back() = c.max_new + 1;                  // bad
    }
    return c;
}

static void section_costs() {
    std::mt19937 rng(21);
    for (int i = 0; i < 600; ++i) {
        Case c = few_rows(rng, i % 2 == 0 ? 20000 : 1500, i % 3 != 0);
        if ((int64_t)c.batch * c.max_new * c.q_heads > 20000) {
            c.batch = std::max(1, 20000 / (c.max_new * c.q_heads));
            c.lengths.resize(c.batch);
            if (!c.counts.empty()) c.counts.resize(c.batch);
        }
        simulate(c, i);
    }
    printf("costs\n");
}

// As the kernel takes them.
static void whole(const Case& c, int id) {
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
    AttendPlan plan = attend4_plan(c.batch, c.max_new, c.q_heads, c.kv_heads, c.head_dim, false);
    CHECK(whole_pays(plan, d), "case %d", id);
    plan.whole_tasks = true;
    const Split a = make_split(d, plan);
    std::vector<uint32_t> cum_cost(c.batch + 1, 0);
    int32_t tokens = 0;
    uint32_t tasks = 0;
    for (int32_t b = 0; b < c.batch; ++b) {
        const Sequence s = sequence(a, b);
        CHECK(plan.own_tiles == 1, "case %d", id);
        cum_cost[b + 1] = cum_cost[b] + tile_cost(a, s, 0) * (uint32_t)c.kv_heads;
        tokens += s.count;
        if (s.count > 0) tasks += (uint32_t)c.kv_heads;
    }
    const Totals t = totals(a, tokens, cum_cost[c.batch]);
    std::map<std::pair<int32_t, int32_t>, uint32_t> by;  // the workgroup of each sequence and head
    for (uint32_t w = 0; w < t.own.groups; ++w) {
        const uint32_t start = group_start(t.own, w), end = group_start(t.own, w + 1);
        for (uint32_t at = start; at < end;) {
            auto task_at = [&](uint32_t u) {
                CHECK(u < t.own.cost, "case %d: place %u", id, u);
                return own_task(
                    a, cum_cost.data(), u, [&](int32_t b) { return sequence(a, b); },
                    [&](const Sequence& s, uint32_t in, uint32_t& first) { return find_tile_host(a, s, in, first); });
            };
            Segment g = task_at(at);
            if (!to_whole_task(a, g, at, end, task_at)) break;
            const uint32_t begins = g.task_start - plan.own_task_units, to = g.task_start + g.units;
            CHECK(at == begins && start <= begins && begins < end, "case %d: group %u", id, w);
            cut(g, at, to);
            CHECK(g.first == 0 && g.end == g.units && g.units > 0 && whole_task(a, g), "case %d: group %u", id, w);
            CHECK(by.emplace(std::make_pair(g.b, g.kv_head), w).second, "case %d: a task taken twice", id);
            at = to;
        }
    }
    CHECK(by.size() == tasks, "case %d: %zu of %u tasks", id, by.size(), tasks);
    for (int32_t b = 0; b < c.batch; ++b)
        if (sequence(a, b).count > 0)
            for (int32_t h = 0; h < c.kv_heads; ++h) CHECK(by.count({b, h}) == 1, "case %d: %d, %d", id, b, h);
}

static void section_whole() {
    std::mt19937 rng(22);
    int several = 0;
    for (int i = 0; i < 3000; ++i) {
        const Case c = few_rows(rng, 1024, false);
        whole(c, i);
        several += (int64_t)c.batch * c.kv_heads > 512;
    }
    whole(Case{3, 4, 8, 2, 64, 16, 8, 0, {1, 2, 3}, {0, -1, 0}}, -1);
    CHECK(several > 300, "%d", several);
    printf("whole tasks: %d batches with more tasks than workgroups\n", several);
}

int main() {
    section_split();
    section_costs();
    section_whole();
    printf("all checks passed (%lld)\n", g_checks);
    (void)all_checks;
    return 0;
}
