// The split of the attention over a cache in 4 bits: the checks of cache_check.cpp on the
// plan of such calls (tests/test_cache4_native.py builds and runs it).
#include "cache_split.hpp"

#define attend_plan attend4_plan
#define attend_workspace_bytes attend4_workspace_bytes
#define kTaskUnits 64  // (of any plan here)
#define main all_checks
#include "cache_check.cpp"
#undef main
#undef kTaskUnits
#undef attend_workspace_bytes
#undef attend_plan

// Single tokens and a few drafts, of one sequence to many: what the tasks of few rows are for.
static void section_few_rows() {
    std::mt19937 rng(11);
    auto pick = [&](int lo, int hi) { return (int32_t)(lo + (int)(rng() % (unsigned)(hi - lo + 1))); };
    const int32_t dims[] = {64, 80, 96, 128, 256};
    int direct = 0, pooled = 0;
    for (int i = 0; i < 800; ++i) {
        Case c{};
        c.batch = pick(0, 2) == 0 ? pick(1, 4) : pick(1, 90);
        c.kv_heads = pick(1, 8);
        c.q_heads = c.kv_heads * pick(1, 8);
        c.head_dim = dims[pick(0, 4)];
        c.page_size = 16 << pick(0, 6);
        c.max_new = pick(1, 12);
        const int32_t longest = pick(1, 20000);
        c.max_pages = (longest + c.max_new + c.page_size - 1) / c.page_size;
        c.prefix_len = pick(0, 1) == 0 ? 0 : pick(1, 9000);
        for (int32_t b = 0; b < c.batch; ++b) {
            c.lengths.push_back(pick(0, 3) == 0 ? pick(0, 20) : pick(0, longest));
            c.counts.push_back(pick(0, 9) == 0 ? pick(-1, 0) : pick(1, c.max_new));
        }
        simulate(c, i);
        const AttendPlan p = attend4_plan(c.batch, c.max_new, c.q_heads, c.kv_heads, c.head_dim, c.prefix_len > 0);
        const int64_t rows = (int64_t)c.max_new * (c.q_heads / c.kv_heads);
        CHECK(p.own_direct == (rows <= direct_rows(c.head_dim)) && (!p.own_direct || (p.own_tiles == 1 && p.own_rows >= rows)),
              "case %d", i);
        CHECK(!p.prefix_direct || (!p.joined && p.own_direct && p.prefix_rows >= c.batch * rows && p.prefix_rows >= p.own_rows),
              "case %d", i);
        CHECK(p.joined || p.prefix_rows >= p.own_rows, "case %d", i);
        direct += p.own_direct;
        pooled += p.prefix_direct;
    }
    CHECK(direct > 100 && pooled > 20, "%d %d", direct, pooled);
    printf("few rows: %d direct, %d with a direct prefix\n", direct, pooled);
}

// The refusals that are its own.
static void section_refusals() {
    int32_t word[4] = {};
    sv_cache_attend_desc_t d{};
    alignas(16) static char some[64];
    d.q = d.k_cache = d.v_cache = some;
    d.out = d.workspace = some;
    d.block_table = d.lengths = word;
    for (int i = 0; i < 3; ++i) d.q_stride[i] = d.out_stride[i] = 256;
    d.batch = 1024;
    d.max_new = 1;
    d.q_heads = d.kv_heads = 1;
    d.head_dim = 256;
    d.max_pages = d.num_pages = 1;
    d.page_size = 16;
    d.page_stride = 16 * packed_row(256);
    d.scale = 1.0f;
    d.dtype = SV_BF16;
    d.workspace_bytes = attend4_workspace_bytes(1024, 1, 1, 1, 256);
    CHECK(d.workspace_bytes > 0 && check_attend4(d) == SV_OK, " ");
    d.workspace_bytes -= 1;
    CHECK(check_attend4(d) == SV_ERR_WORKSPACE, " ");
    d.workspace_bytes = (size_t)1 << 40;
    d.page_stride -= 16;
    CHECK(check_attend4(d) == SV_ERR_PARAM, " ");
    d.page_stride += 24;
    CHECK(check_attend4(d) == SV_ERR_PARAM, " ");
    d.page_stride -= 8;
    d.batch = 1025;
    CHECK(check_attend4(d) == SV_ERR_SHAPE && attend4_workspace_bytes(1025, 1, 1, 1, 256) == 0, " ");
    CHECK(check_cache4(SV_F16, 1, 1, 1, 80, 1, 16, 16 * 43) == SV_OK, " ");
    CHECK(check_cache4(SV_F16, 1, 1, 1, 80, 1, 16, 16 * 42) == SV_ERR_PARAM, " ");
    CHECK(check_cache4(SV_F32, 1, 1, 1, 80, 1, 16, 16 * 43) == SV_ERR_DTYPE, " ");
    CHECK(check_cache4(SV_F16, 1, 1, 1, 84, 1, 16, 16 * 43) == SV_ERR_SHAPE, " ");
}

int main() {
    section_split();
    section_few_rows();
    section_refusals();
    printf("all checks passed (%lld)\n", g_checks);
    (void)all_checks;
    return 0;
}
