// The kernels of spec_cache_attend4 for bfloat16.
#include "cache_attend.hpp"

namespace sv {

sv_status_t attend4_bf16(const AttendArgs& a, int32_t head_dim, hipStream_t stream) {
    return launch_dim<AttBF16, In4>(a, head_dim, stream);
}

}  // namespace sv
