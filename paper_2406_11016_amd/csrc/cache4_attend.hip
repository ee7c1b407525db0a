// The kernels of spec_cache_attend4 for bfloat16.
#include "cache4_attend.hpp"

namespace sv {

sv_status_t attend4_bf16(const AttendArgs& a, int32_t head_dim, hipStream_t stream) {
    return launch4_dim<AttBF16>(a, head_dim, stream);
}

}  // namespace sv
