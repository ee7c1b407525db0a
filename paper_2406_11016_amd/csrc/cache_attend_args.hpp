// What the cache attention's kernels are given, and how a call's descriptor
// becomes that.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_plan.hpp"
#include "cache_split.hpp"
#include "spec_cache.h"

namespace sv {

struct AttendArgs {
    const uint16_t* q;
    uint16_t* out;
    int64_t q_stride[3], out_stride[3];
    const uint16_t* k_cache;
    const uint16_t* v_cache;
    int64_t page_stride;
    const int32_t* block_table;
    const int32_t* prefix_table;
    int32_t prefix_len, num_pages, q_heads;
    float scale_log2, lazy;  // scale * log2(e); the rise of a maximum, in scores, that is let pass
    Split split;
    // workspace
    int32_t* cum_tokens;  // [batch + 1] tokens before each sequence
    uint32_t* cum_cost;   // [batch + 1] cost of the own tasks before each sequence's
    float* part_out;      // parts: rows x head_dim, fp32
    Totals* totals;       // of the split
    float* part_max;      // maximum (scores as they come from the product)
    float* part_sum;
};

// The kernels of each storage type are compiled by themselves.
sv_status_t attend_f16(const AttendArgs& a, int32_t head_dim, hipStream_t stream);
sv_status_t attend_bf16(const AttendArgs& a, int32_t head_dim, hipStream_t stream);

sv_status_t attend4_f16(const AttendArgs& a, int32_t head_dim, hipStream_t stream);  // caches in 4 bits
sv_status_t attend4_bf16(const AttendArgs& a, int32_t head_dim, hipStream_t stream);

// Of a call that has been checked.
inline AttendArgs attend_args(const sv_cache_attend_desc_t& d, const AttendPlan& plan) {
    AttendArgs a{};
    a.split = make_split(d, plan);
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
    a.totals = reinterpret_cast<Totals*>(ws + 2 * plan.cum_bytes);
    a.part_max = reinterpret_cast<float*>(ws + 2 * plan.cum_bytes + kTotalsBytes);
    a.part_sum = a.part_max + plan.rows;
    a.part_out = a.part_sum + plan.rows;
    return a;
}

}  // namespace sv
