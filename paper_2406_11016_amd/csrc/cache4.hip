// The cache in 4 bits for gfx950 (MI355X): the kernels of spec_cache_append4 and
// spec_cache_read4, and the C ABI of those and of spec_cache_attend4 (spec_cache.h).
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "cache4.hpp"
#include "cache_attend_args.hpp"
#include "cache_plan.hpp"
#include "spec_cache.h"

namespace sv {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The storage types: a magnitude as fp32, and two values to and from 4 bits each (byte
// `kByte` of the codes) with a scale, whose exponent counts.  kLast (twice): the last number
// before 3.5 times the greatest scale.
struct Half {
    static constexpr uint32_t kNotFinite = 0x7c00, kLeast = kPackedLeastF16, kLast = 0x7aff7affu;
    static __device__ __forceinline__ float value(uint32_t bits) {
        return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    }
    template <int kByte>
    static __device__ __forceinline__ uint32_t pack(uint32_t codes, uint32_t two, float scale) {
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(f16x2, two), scale, kByte);
    }
    template <int kByte>
    static __device__ __forceinline__ uint32_t unpack(uint32_t codes, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, kByte));
    }
};
struct BFloat {
    static constexpr uint32_t kNotFinite = 0x7f80, kLeast = kPackedLeastBF16, kLast = 0x7f5f7f5fu;
    static __device__ __forceinline__ float value(uint32_t bits) { return __uint_as_float(bits << 16); }
    template <int kByte>
    static __device__ __forceinline__ uint32_t pack(uint32_t codes, uint32_t two, float scale) {
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, two), scale, kByte);
    }
    template <int kByte>
    static __device__ __forceinline__ uint32_t unpack(uint32_t codes, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte));
    }
};

__device__ __forceinline__ uint32_t max_pair(uint32_t x, uint32_t y) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y)));
}
// Two values whose magnitudes are `last` at most.
__device__ __forceinline__ uint32_t within(uint32_t two, uint32_t last) {
    const uint32_t m = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, two & 0x7fff7fffu),
                                                                              __builtin_bit_cast(u16x2, last)));
    return m | (two & 0x80008000u);
}
// The largest magnitude (its bits) of 8 values, and of the 32 that four neighbouring lanes
// have: magnitudes are ordered as their bits, with infinity and NaN on top.
__device__ __forceinline__ uint32_t largest(const u32x4& x) {
    uint32_t m = x[0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 4; ++i) m = max_pair(m, x[i] & 0x7fff7fffu);
    return max(m & 0xffffu, m >> 16);
}
__device__ __forceinline__ uint32_t largest_of_four(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, true));  // lane ^ 1
    return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, true));  // lane ^ 2
}

// 8 values of a block whose largest magnitude is known: its scale's byte, and their codes.
// The scale is the power of two that brings the magnitude into 3.5 .. 7: adding a
// quarter of the mantissa's range carries into the exponent from 1.75 on.  The types have
// no number of 4 times the greatest scale (fp16 2^14, bf16 2^126), so what would round to it, from
// 3.5 on, goes to 3 times it; with smaller scales all numbers are below kLast.
template <class T>
__device__ __forceinline__ uint32_t quantise(const u32x4& x, uint32_t magnitude, uint32_t& byte) {
    const int exponent = (int)((__float_as_uint(T::value(magnitude)) + 0x200000u) >> 23) - 2;
    byte = (uint32_t)max(exponent, (int)T::kLeast);
    if (magnitude >= T::kNotFinite) byte = kPackedNaN;
    const float scale = __uint_as_float(byte << 23);
    uint32_t codes = T::template pack<0>(0u, within(x[0], T::kLast), scale);
    codes = T::template pack<1>(codes, within(x[1], T::kLast), scale);
    codes = T::template pack<2>(codes, within(x[2], T::kLast), scale);
    codes = T::template pack<3>(codes, within(x[3], T::kLast), scale);
    return byte == kPackedNaN ? 0u : codes;
}

// Where token `slot`'s codes of a head begin in a cache, and how far behind them its scales.
struct Place {
    int64_t codes;
    int32_t scales;
};
__device__ __forceinline__ Place place_of(uint32_t slot, uint32_t head, int64_t page_stride, int32_t page_shift,
                                          int32_t head_dim) {
    const int32_t in_page = (int32_t)(slot & ((1u << page_shift) - 1)), row = head_dim / 2, blocks = packed_blocks(head_dim);
    return Place{(int64_t)(slot >> page_shift) * page_stride + ((int64_t)head << page_shift) * (row + blocks) +
                     (int64_t)in_page * row,
                 (row << page_shift) - in_page * (row - blocks)};
}

// A thread has 8 values of K and of V, and four threads a block of 32 (head_dim is filled up
// to whole blocks by threads without values).  Bound by memory: 9,032 tokens of 8 heads of 128,
// 37 MB in and 10 out, 13.1 us, 3.6 TB/s; 447 tokens 3.4 us, the latency of a launch and two loads.
template <class T>
__global__ void __launch_bounds__(256) cache_append4_kernel(sv_cache_append_desc_t d, uint32_t chunks_head,
                                                            uint32_t chunks_token, int32_t page_shift, uint32_t total) {
    const uint32_t stride = gridDim.x * 256;
    const uint32_t slots_end = (uint32_t)d.num_pages << page_shift;
    for (uint64_t at = blockIdx.x * 256 + threadIdx.x; at < total; at += stride) {
        const uint32_t token = (uint32_t)at / chunks_token, rest = (uint32_t)at - token * chunks_token;
        const uint32_t head = rest / chunks_head, chunk = rest - head * chunks_head;
        const uint32_t slot = (uint32_t)d.slots[token];
        if (slot >= slots_end) continue;
        const uint32_t b = token / (uint32_t)d.max_new, i = token - b * (uint32_t)d.max_new;
        const bool there = chunk * 8 < (uint32_t)d.head_dim;
        u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
        if (there) {
            k = *(const u32x4*)((const uint16_t*)d.k + b * d.k_stride[0] + i * d.k_stride[1] + head * d.k_stride[2] +
                                chunk * 8);
            v = *(const u32x4*)((const uint16_t*)d.v + b * d.v_stride[0] + i * d.v_stride[1] + head * d.v_stride[2] +
                                chunk * 8);
        }
        uint32_t k_byte, v_byte;
        const uint32_t k_codes = quantise<T>(k, largest_of_four(largest(k)), k_byte);
        const uint32_t v_codes = quantise<T>(v, largest_of_four(largest(v)), v_byte);
        if (!there) continue;
        const Place to = place_of(slot, head, d.page_stride, page_shift, d.head_dim);
        uint8_t* const k_to = (uint8_t*)d.k_cache + to.codes;
        uint8_t* const v_to = (uint8_t*)d.v_cache + to.codes;
        *(uint32_t*)(k_to + chunk * 4) = k_codes;
        *(uint32_t*)(v_to + chunk * 4) = v_codes;
        if (chunk % 4 == 0) {
            k_to[to.scales + (int)(chunk / 4)] = (uint8_t)k_byte;
            v_to[to.scales + (int)(chunk / 4)] = (uint8_t)v_byte;
        }
    }
}

// A thread has 8 values of K and of V.  Bound by memory, most of it writes: 16,196 tokens of 8 heads of
// 128, 18 MB in and 66 out, 18.2 us, 4.6 TB/s.  (Two to eight tokens a thread, tokens in the order of the pages
// and no divisions took 19.5 to 22.6 us, and this 20.4, called from Python.)
template <class T>
__global__ void __launch_bounds__(256) cache_read4_kernel(sv_cache_read_desc_t d, uint32_t chunks_head, uint32_t chunks_token,
                                                          int32_t page_shift, uint32_t total) {
    const uint32_t stride = gridDim.x * 256;
    const uint32_t slots_end = (uint32_t)d.num_pages << page_shift;
    for (uint64_t at = blockIdx.x * 256 + threadIdx.x; at < total; at += stride) {
        const uint32_t token = (uint32_t)at / chunks_token, rest = (uint32_t)at - token * chunks_token;
        const uint32_t head = rest / chunks_head, chunk = rest - head * chunks_head;
        const uint32_t slot = (uint32_t)d.slots[token];
        if (slot >= slots_end) continue;
        const uint32_t b = token / (uint32_t)d.max_new, i = token - b * (uint32_t)d.max_new;
        const Place from = place_of(slot, head, d.page_stride, page_shift, d.head_dim);
        const uint8_t* const k_from = (const uint8_t*)d.k_cache + from.codes;
        const uint8_t* const v_from = (const uint8_t*)d.v_cache + from.codes;
        const uint32_t k = *(const uint32_t*)(k_from + chunk * 4), v = *(const uint32_t*)(v_from + chunk * 4);
        const float ks = __uint_as_float((uint32_t)k_from[from.scales + (int)(chunk / 4)] << 23);
        const float vs = __uint_as_float((uint32_t)v_from[from.scales + (int)(chunk / 4)] << 23);
        *(u32x4*)((uint16_t*)d.k + b * d.k_stride[0] + i * d.k_stride[1] + head * d.k_stride[2] + chunk * 8) =
            u32x4{T::template unpack<0>(k, ks), T::template unpack<1>(k, ks), T::template unpack<2>(k, ks),
                  T::template unpack<3>(k, ks)};
        *(u32x4*)((uint16_t*)d.v + b * d.v_stride[0] + i * d.v_stride[1] + head * d.v_stride[2] + chunk * 8) =
            u32x4{T::template unpack<0>(v, vs), T::template unpack<1>(v, vs), T::template unpack<2>(v, vs),
                  T::template unpack<3>(v, vs)};
    }
}

uint32_t blocks_for(uint32_t total) {
    const uint32_t blocks = (total + 255) / 256;
    return blocks < kAppendBlocks ? blocks : kAppendBlocks;
}

sv_status_t launched() { return hipGetLastError() == hipSuccess ? SV_OK : SV_ERR_HIP; }

}  // namespace
}  // namespace sv

extern "C" {

sv_status_t spec_cache_append4(const sv_cache_append_desc_t* desc, hipStream_t stream) {
    if (desc == nullptr) return SV_ERR_NULL;
    const sv_cache_append_desc_t& d = *desc;
    if (d.k == nullptr || d.v == nullptr || d.k_cache == nullptr || d.v_cache == nullptr || d.slots == nullptr)
        return SV_ERR_NULL;
    const sv_status_t st = sv::check_cache4(d.dtype, d.batch, d.max_new, d.kv_heads, d.head_dim, d.num_pages, d.page_size,
                                            d.page_stride);
    if (st != SV_OK) return st;
    const int64_t chunks_head = 4 * sv::packed_blocks(d.head_dim), chunks_token = d.kv_heads * chunks_head;
    if (chunks_token > INT_MAX || (int64_t)d.batch * d.max_new * chunks_token > INT_MAX) return SV_ERR_SHAPE;
    if (!sv::aligned16(d.k) || !sv::aligned16(d.v) || !sv::aligned16(d.k_cache) || !sv::aligned16(d.v_cache) ||
        !sv::strides_ok(d.k_stride) || !sv::strides_ok(d.v_stride))
        return SV_ERR_PARAM;
    const uint32_t total = (uint32_t)((int64_t)d.batch * d.max_new * chunks_token);
    const auto kernel = d.dtype == SV_F16 ? sv::cache_append4_kernel<sv::Half> : sv::cache_append4_kernel<sv::BFloat>;
    hipLaunchKernelGGL(kernel, dim3(sv::blocks_for(total)), dim3(256), 0, stream, d, (uint32_t)chunks_head,
                       (uint32_t)chunks_token, sv::page_shift(d.page_size), total);
    return sv::launched();
}

sv_status_t spec_cache_read4(const sv_cache_read_desc_t* desc, hipStream_t stream) {
    if (desc == nullptr) return SV_ERR_NULL;
    const sv_cache_read_desc_t& d = *desc;
    if (d.k == nullptr || d.v == nullptr || d.k_cache == nullptr || d.v_cache == nullptr || d.slots == nullptr)
        return SV_ERR_NULL;
    const sv_status_t st = sv::check_cache4(d.dtype, d.batch, d.max_new, d.kv_heads, d.head_dim, d.num_pages, d.page_size,
                                            d.page_stride);
    if (st != SV_OK) return st;
    const int64_t chunks_head = d.head_dim / 8, chunks_token = d.kv_heads * chunks_head;
    if (chunks_token > INT_MAX || (int64_t)d.batch * d.max_new * chunks_token > INT_MAX) return SV_ERR_SHAPE;
    if (!sv::aligned16(d.k) || !sv::aligned16(d.v) || !sv::aligned16(d.k_cache) || !sv::aligned16(d.v_cache) ||
        !sv::strides_ok(d.k_stride) || !sv::strides_ok(d.v_stride) ||
        !sv::rows_apart(d.k_stride, d.batch, d.max_new, d.kv_heads) ||
        !sv::rows_apart(d.v_stride, d.batch, d.max_new, d.kv_heads))
        return SV_ERR_PARAM;
    const uint32_t total = (uint32_t)((int64_t)d.batch * d.max_new * chunks_token);
    const auto kernel = d.dtype == SV_F16 ? sv::cache_read4_kernel<sv::Half> : sv::cache_read4_kernel<sv::BFloat>;
    hipLaunchKernelGGL(kernel, dim3(sv::blocks_for(total)), dim3(256), 0, stream, d, (uint32_t)chunks_head,
                       (uint32_t)chunks_token, sv::page_shift(d.page_size), total);
    return sv::launched();
}

size_t spec_cache_attend4_workspace_bytes(int32_t batch, int32_t max_new, int32_t q_heads, int32_t kv_heads,
                                          int32_t head_dim) {
    return sv::attend4_workspace_bytes(batch, max_new, q_heads, kv_heads, head_dim);
}

sv_status_t spec_cache_attend4(const sv_cache_attend_desc_t* desc, hipStream_t stream) {
    if (desc == nullptr) return SV_ERR_NULL;
    const sv_cache_attend_desc_t& d = *desc;
    const sv_status_t st = sv::check_attend4(d);
    if (st != SV_OK) return st;
    sv::AttendPlan plan = sv::attend4_plan(d.batch, d.max_new, d.q_heads, d.kv_heads, d.head_dim, d.prefix_len > 0);
    plan.whole_tasks = sv::whole_pays(plan, d);
    const sv::AttendArgs a = sv::attend_args(d, plan);
    return d.dtype == SV_F16 ? sv::attend4_f16(a, d.head_dim, stream) : sv::attend4_bf16(a, d.head_dim, stream);
}

}  // extern "C"
