// spec_cache_attend: C ABI, and the kernels for bfloat16.
#include "cache_attend.hpp"
#include "cache_plan.hpp"

namespace sv {

sv_status_t attend_bf16(const AttendArgs& a, int32_t head_dim, hipStream_t stream) {
    return launch_dim<AttBF16>(a, head_dim, stream);
}

}  // namespace sv

extern "C" {

size_t spec_cache_attend_workspace_bytes(int32_t batch, int32_t max_new, int32_t q_heads, int32_t kv_heads,
                                         int32_t head_dim) {
    return sv::attend_workspace_bytes(batch, max_new, q_heads, kv_heads, head_dim);
}

sv_status_t spec_cache_attend(const sv_cache_attend_desc_t* desc, hipStream_t stream) {
    if (desc == nullptr) return SV_ERR_NULL;
    const sv_cache_attend_desc_t& d = *desc;
    const sv_status_t st = sv::check_attend(d);
    if (st != SV_OK) return st;
    sv::AttendArgs a{};
    const sv::AttendPlan plan =
        sv::attend_plan(d.batch, d.max_new, d.q_heads, d.kv_heads, d.head_dim, d.prefix_len > 0);
    a.split = sv::make_split(d, plan);
    a.q = static_cast<const uint16_t*>(d.q);
    a.out = static_cast<uint16_t*>(d.out);
    for (int i = 0; i < 3; ++i) {
        a.q_stride[i] = d.q_stride[i];
        a.out_stride[i] = d.out_stride[i];
    }
    a.k_cache = static_cast<const uint16_t*>(d.k_cache);
    a.v_cache = static_cast<const uint16_t*>(d.v_cache);
    a.page_stride = d.page_stride;
    a.block_table = d.block_table;
    a.prefix_table = d.prefix_table;
    a.prefix_len = d.prefix_len;
    a.num_pages = d.num_pages;
    a.q_heads = d.q_heads;
    a.scale_log2 = (float)((double)d.scale * 1.4426950408889634);
    a.lazy = 8.0f / a.scale_log2;
    char* ws = static_cast<char*>(d.workspace);
    a.cum_tokens = reinterpret_cast<int32_t*>(ws);
    a.cum_cost = reinterpret_cast<uint32_t*>(ws + plan.cum_bytes);
    a.totals = reinterpret_cast<sv::Totals*>(ws + 2 * plan.cum_bytes);
    a.part_max = reinterpret_cast<float*>(ws + 2 * plan.cum_bytes + sv::kTotalsBytes);
    a.part_sum = a.part_max + plan.rows;
    a.part_out = a.part_sum + plan.rows;
    return d.dtype == SV_F16 ? sv::attend_f16(a, d.head_dim, stream) : sv::attend_bf16(a, d.head_dim, stream);
}

}  // extern "C"
