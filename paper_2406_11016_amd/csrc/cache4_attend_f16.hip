// The kernels of spec_cache_attend4 for float16.
#include "cache4_attend.hpp"

namespace sv {

sv_status_t attend4_f16(const AttendArgs& a, int32_t head_dim, hipStream_t stream) {
    return launch4_dim<AttF16>(a, head_dim, stream);
}

}  // namespace sv
