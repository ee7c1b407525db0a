// The layout of a cache in 4 bits (spec_cache.h).  Plain constexpr C++17, for the
// host and the kernels.
#pragma once

#include <stdint.h>

namespace sv {

// Values of a scale.  The last block of a row may have fewer.
constexpr int kPackedBlock = 32;

constexpr int packed_blocks(int head_dim) { return (head_dim + kPackedBlock - 1) / kPackedBlock; }

// Bytes of a token and head: its codes, two a byte, and its scales.
constexpr int packed_row(int head_dim) { return head_dim / 2 + packed_blocks(head_dim); }

// The smallest scales' bytes (exponent + 127): half of such a scale is the smallest number
// of fp16, the smallest normal one of bf16.  So whatever is held is a number of the type
// (with the greatest scales, what is written is 3 times the scale at most: see quantise()).
constexpr uint32_t kPackedLeastF16 = 127 - 23;
constexpr uint32_t kPackedLeastBF16 = 127 - 125;
constexpr uint32_t kPackedNaN = 255;

}  // namespace sv
