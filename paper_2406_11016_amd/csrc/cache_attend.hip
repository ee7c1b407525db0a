// spec_cache_attend: C ABI, and the kernels for bfloat16.
#include "cache_attend.hpp"
#include "cache_attend_args.hpp"
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
    const sv::AttendArgs a =
        sv::attend_args(d, sv::attend_plan(d.batch, d.max_new, d.q_heads, d.kv_heads, d.head_dim, d.prefix_len > 0));
    return d.dtype == SV_F16 ? sv::attend_f16(a, d.head_dim, stream) : sv::attend_bf16(a, d.head_dim, stream);
}

}  // extern "C"
