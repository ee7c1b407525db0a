// The kernels of spec_cache_attend for float16.
#include "cache_attend.hpp"

namespace sv {

sv_status_t attend_f16(const AttendArgs& a, int32_t head_dim, hipStream_t stream) {
    return launch_dim<AttF16>(a, head_dim, stream);
}

}  // namespace sv
