// The paged key/value cache's tables and its writes for gfx950 (MI355X): the
// kernels and the C ABI of spec_cache_init, spec_cache_plan and
// spec_cache_append (spec_cache.h).
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "cache_plan.hpp"
#include "spec_cache.h"

namespace sv {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// empty tables
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(256) cache_init_kernel(sv_cache_tables_t t, int32_t first_page) {
    const int64_t stride = (int64_t)gridDim.x * 256;
    const int64_t rows = (int64_t)t.batch * t.max_pages;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t i = at; i < rows; i += stride) t.block_table[i] = -1;
    const int32_t spare = t.num_pages - first_page;
    for (int64_t i = at; i < t.num_pages; i += stride)
        t.free_pages[i] = (i < spare) ? t.num_pages - 1 - (int32_t)i : -1;
    for (int64_t i = at; i < t.batch; i += stride) t.lengths[i] = t.counts[i] = t.held[i] = 0;
    if (at == 0) t.free_count[0] = spare;
}

// ---------------------------------------------------------------------------
// plan
// ---------------------------------------------------------------------------
struct PlanArgs {
    sv_cache_tables_t t;
    const int32_t* accepted;
    const int32_t* new_tokens;
    const int32_t* release;
    int32_t* slots;
    int32_t* positions;
    int32_t max_new, position_base, page_shift;
    int32_t own_slots;  // nonzero: this kernel writes slots and positions too
};

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

// The first b whose inclusive sum end[b] exceeds p (p < end[n - 1]).
__device__ __forceinline__ int owner(const int32_t* end, int n, int32_t p) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (end[mid] > p)
            hi = mid;
        else
            lo = mid + 1;
    }
    return lo;
}

// Inclusive sums of x and y over the workgroup, on top of the carries.
__device__ __forceinline__ void scan2(int32_t& x, int32_t& y, int32_t (*wave_sums)[2], int32_t& cx, int32_t& cy) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t ox = __shfl_up(x, d), oy = __shfl_up(y, d);
        if (lane >= d) {
            x += ox;
            y += oy;
        }
    }
    if (lane == 63) {
        wave_sums[wave][0] = x;
        wave_sums[wave][1] = y;
    }
    __syncthreads();
    int32_t tx = 0, ty = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        if (w == wave) {
            x += cx + tx;
            y += cy + ty;
        }
        tx += wave_sums[w][0];
        ty += wave_sums[w][1];
    }
    cx += tx;
    cy += ty;
}

// One workgroup for the whole batch.  The only coupling between sequences is
// two running sums over b (pages given back, pages taken), so each sequence's
// step is computed by one thread and both sums by one scan; the pages that move
// are then dealt to all threads by their place in the sums (a sequence may move
// none or thousands), and a token's slot comes straight from the old table or
// from the stack, so that nothing written here is read back but the pages just
// released.  What bounds it is latency: one launch, a load of the state, the
// scan, a load of the pages, a store.  (5 us with 64 sequences; 22 us with 4,096,
// four rounds of the scan and searches twice as deep.)
__global__ void __launch_bounds__(kPlanThreads) cache_plan_kernel(PlanArgs a) {
    extern __shared__ int32_t lds[];
    __shared__ int32_t wave_sums[2][kPlanWaves][2];
    const sv_cache_tables_t& t = a.t;
    const int32_t B = t.batch, M = t.max_pages, N = t.num_pages;
    const int32_t room = M << a.page_shift;  // (M * page_size fits: checked on the host)
    int32_t* const length = lds;             // tokens kept
    int32_t* const count = lds + B;          // tokens wanted, -1: bad
    int32_t* const held = lds + 2 * B;       // pages kept
    int32_t* const gone = lds + 3 * B;       // inclusive sums of the pages given back
    int32_t* const more = lds + 4 * B;       // inclusive sums of the pages wanted
    const int32_t depth0 = min(max(t.free_count[0], 0), N);
    int32_t given = 0, wanted = 0;
    for (int32_t first = 0, k = 0; first < B; first += kPlanThreads, k ^= 1) {
        const int32_t b = first + (int32_t)threadIdx.x;
        int32_t back = 0, extra = 0;
        if (b < B) {
            int32_t len = t.lengths[b], cnt = t.counts[b];
            int32_t h = min(max(t.held[b], 0), M);
            const bool over = a.release != nullptr && a.release[b] != 0;
            const int32_t want = (a.new_tokens != nullptr) ? a.new_tokens[b] : a.max_new;
            const int32_t acc = (a.accepted != nullptr) ? a.accepted[b] : cnt - 1;
            if (over) {
                back = h;
                len = cnt = h = 0;
            }
            bool bad = want < 0 || want > a.max_new;
            if (cnt > 0) {
                if (acc < -1 || acc >= cnt)
                    bad = true;
                else
                    len = (int32_t)((uint32_t)len + (uint32_t)(acc + 1));  // (a corrupt sum turns out too long below)
            }
            // (the sum of two non-negative int32 fits an unsigned one)
            if (len < 0 || (!bad && (uint32_t)len + (uint32_t)want > (uint32_t)room)) bad = true;
            if (!bad) extra = max(0, (int32_t)(((uint32_t)(len + want) + (1u << a.page_shift) - 1) >> a.page_shift) - h);
            length[b] = len;
            count[b] = bad ? -1 : want;
            held[b] = h;
        }
        scan2(back, extra, wave_sums[k], given, wanted);
        if (b < B) {
            gone[b] = back;
            more[b] = extra;
        }
    }
    __syncthreads();
    // the pages of ended sequences, onto the stack
    const int32_t depth = min(given, N - depth0) + depth0;
    if (given > 0) {
        for (int32_t p = threadIdx.x; p < given; p += kPlanThreads) {
            const int b = owner(gone, B, p);
            int32_t* const from = t.block_table + (int64_t)b * M + (p - (b > 0 ? gone[b - 1] : 0));
            const int32_t page = *from;
            *from = -1;
            if (depth0 + p < N) t.free_pages[depth0 + p] = page;
        }
        __syncthreads();
    }
    // the sums are ordered: the sequences served are those up to the last sum within the stack
    int32_t taken = wanted;
    if (wanted > depth) {
        const int b = owner(more, B, depth);
        taken = b > 0 ? more[b - 1] : 0;
    }
    for (int32_t p = threadIdx.x; p < taken; p += kPlanThreads) {
        const int b = owner(more, B, p);
        t.block_table[(int64_t)b * M + held[b] + (p - (b > 0 ? more[b - 1] : 0))] = t.free_pages[depth - 1 - p];
    }
    for (int32_t b = threadIdx.x; b < B; b += kPlanThreads) {
        const int32_t before = b > 0 ? more[b - 1] : 0, extra = more[b] - before;
        const bool short_of = extra > 0 && more[b] > taken;
        t.lengths[b] = length[b];
        t.counts[b] = short_of ? -1 : count[b];
        t.held[b] = held[b] + (short_of ? 0 : extra);
    }
    if (threadIdx.x == 0) t.free_count[0] = depth - taken;
    if (a.own_slots == 0) return;
    const int32_t mask = (1 << a.page_shift) - 1;
    const int32_t total = B * a.max_new;
    for (int32_t at = threadIdx.x; at < total; at += kPlanThreads) {
        const int32_t b = at / a.max_new, i = at - b * a.max_new;
        const int32_t before = b > 0 ? more[b - 1] : 0;
        const bool short_of = more[b] > before && more[b] > taken;
        int32_t slot = -1, position = -1;
        if (i < count[b] && !short_of) {
            const int32_t place = length[b] + i, j = place >> a.page_shift;
            const int32_t page = (j < held[b]) ? t.block_table[(int64_t)b * M + j]
                                               : t.free_pages[depth - 1 - (before + j - held[b])];
            if ((uint32_t)page < (uint32_t)N) slot = (page << a.page_shift) + (place & mask);
            position = a.position_base + place;
        }
        a.slots[at] = slot;
        if (a.positions != nullptr) a.positions[at] = position;
    }
}

// Slots and positions of a large plan, from the tables that the kernel above left.
__global__ void __launch_bounds__(256) cache_slots_kernel(PlanArgs a) {
    const sv_cache_tables_t& t = a.t;
    const int32_t b = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
    if (i >= a.max_new) return;
    int32_t slot = -1, position = -1;
    if (i < t.counts[b]) {
        const int32_t place = t.lengths[b] + i;
        const int32_t page = t.block_table[(int64_t)b * t.max_pages + (place >> a.page_shift)];
        if ((uint32_t)page < (uint32_t)t.num_pages)
            slot = (page << a.page_shift) + (place & ((1 << a.page_shift) - 1));
        position = a.position_base + place;
    }
    a.slots[(int64_t)b * a.max_new + i] = slot;
    if (a.positions != nullptr) a.positions[(int64_t)b * a.max_new + i] = position;
}

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------

// A copy, 16 bytes a thread and tensor.  Bound by memory: every byte is read
// once and written once, in runs of head_dim elements on both sides.  (9,032 tokens
// of 8 heads of 128, 74 MB: 14 us, 5.2 TB/s, from memory; 447 tokens, 3.7 MB: 3.2 us,
// the latency of a launch and of two loads, the slot's and the row's.)
__global__ void __launch_bounds__(256) cache_append_kernel(sv_cache_append_desc_t d, uint32_t chunks_head,
                                                           uint32_t chunks_token, int32_t page_shift,
                                                           uint32_t total) {
    const uint32_t stride = gridDim.x * 256;
    const uint32_t slots_end = (uint32_t)d.num_pages << page_shift;
    for (uint64_t at = blockIdx.x * 256 + threadIdx.x; at < total; at += stride) {
        const uint32_t token = (uint32_t)at / chunks_token, rest = (uint32_t)at - token * chunks_token;
        const uint32_t head = rest / chunks_head, chunk = rest - head * chunks_head;
        const uint32_t slot = (uint32_t)d.slots[token];
        if (slot >= slots_end) continue;
        const uint32_t b = token / (uint32_t)d.max_new, i = token - b * (uint32_t)d.max_new;
        const int64_t to = (int64_t)(slot >> page_shift) * d.page_stride +
                           ((int64_t)(head << page_shift) + (slot & ((1u << page_shift) - 1))) * d.head_dim + chunk * 8;
        const u32x4 k = *(const u32x4*)((const uint16_t*)d.k + b * d.k_stride[0] + i * d.k_stride[1] +
                                        head * d.k_stride[2] + chunk * 8);
        const u32x4 v = *(const u32x4*)((const uint16_t*)d.v + b * d.v_stride[0] + i * d.v_stride[1] +
                                        head * d.v_stride[2] + chunk * 8);
        *(u32x4*)((uint16_t*)d.k_cache + to) = k;
        *(u32x4*)((uint16_t*)d.v_cache + to) = v;
    }
}

bool tables_null(const sv_cache_tables_t& t) {
    return t.lengths == nullptr || t.counts == nullptr || t.held == nullptr || t.block_table == nullptr ||
           t.free_pages == nullptr || t.free_count == nullptr;
}

sv_status_t launched() { return hipGetLastError() == hipSuccess ? SV_OK : SV_ERR_HIP; }

}  // namespace
}  // namespace sv

extern "C" {

sv_status_t spec_cache_init(const sv_cache_tables_t* tables, int32_t first_page, hipStream_t stream) {
    if (tables == nullptr || sv::tables_null(*tables)) return SV_ERR_NULL;
    const sv_cache_tables_t& t = *tables;
    if (!sv::cache_table_sizes_ok(t.batch, t.max_pages, t.num_pages, t.page_size)) return SV_ERR_SHAPE;
    if (first_page < 0 || first_page > t.num_pages) return SV_ERR_SHAPE;
    const int64_t most = (int64_t)t.batch * t.max_pages > t.num_pages ? (int64_t)t.batch * t.max_pages : t.num_pages;
    const int64_t blocks = (most + 255) / 256;
    hipLaunchKernelGGL(sv::cache_init_kernel, dim3((uint32_t)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, stream, t,
                       first_page);
    return sv::launched();
}

sv_status_t spec_cache_plan(const sv_cache_tables_t* tables, const int32_t* accepted_len, const int32_t* new_tokens,
                            const int32_t* release, int32_t max_new, int32_t position_base, int32_t* slots,
                            int32_t* positions, hipStream_t stream) {
    if (tables == nullptr || sv::tables_null(*tables) || slots == nullptr) return SV_ERR_NULL;
    const sv_cache_tables_t& t = *tables;
    if (!sv::cache_table_sizes_ok(t.batch, t.max_pages, t.num_pages, t.page_size)) return SV_ERR_SHAPE;
    if (max_new < 1 || (int64_t)t.batch * max_new > INT_MAX) return SV_ERR_SHAPE;
    if (position_base < 0 || (int64_t)position_base + (int64_t)t.max_pages * t.page_size > INT_MAX) return SV_ERR_PARAM;
    sv::PlanArgs a{};
    a.t = t;
    a.accepted = accepted_len;
    a.new_tokens = new_tokens;
    a.release = release;
    a.slots = slots;
    a.positions = positions;
    a.max_new = max_new;
    a.position_base = position_base;
    a.page_shift = sv::page_shift(t.page_size);
    a.own_slots = (int64_t)t.batch * max_new <= sv::kPlanOwnSlots ? 1 : 0;
    hipLaunchKernelGGL(sv::cache_plan_kernel, dim3(1), dim3(sv::kPlanThreads), 5 * sizeof(int32_t) * (size_t)t.batch,
                       stream, a);
    if (a.own_slots == 0)
        hipLaunchKernelGGL(sv::cache_slots_kernel, dim3(((uint32_t)max_new + 255) / 256, (uint32_t)t.batch), dim3(256), 0,
                           stream, a);
    return sv::launched();
}

sv_status_t spec_cache_append(const sv_cache_append_desc_t* desc, hipStream_t stream) {
    if (desc == nullptr) return SV_ERR_NULL;
    const sv_cache_append_desc_t& d = *desc;
    if (d.k == nullptr || d.v == nullptr || d.k_cache == nullptr || d.v_cache == nullptr || d.slots == nullptr)
        return SV_ERR_NULL;
    const sv_status_t st = sv::check_cache(d.dtype, d.batch, d.max_new, d.kv_heads, d.head_dim, d.num_pages, d.page_size,
                                           d.page_stride);
    if (st != SV_OK) return st;
    const int64_t chunks_token = (int64_t)d.kv_heads * (d.head_dim / 8);
    if (chunks_token > INT_MAX || (int64_t)d.batch * d.max_new * chunks_token > INT_MAX) return SV_ERR_SHAPE;
    if (!sv::aligned16(d.k) || !sv::aligned16(d.v) || !sv::aligned16(d.k_cache) || !sv::aligned16(d.v_cache) ||
        !sv::strides_ok(d.k_stride) || !sv::strides_ok(d.v_stride))
        return SV_ERR_PARAM;
    const uint32_t total = (uint32_t)((int64_t)d.batch * d.max_new * chunks_token);
    const uint32_t blocks = (total + 255) / 256;
    hipLaunchKernelGGL(sv::cache_append_kernel, dim3(blocks < sv::kAppendBlocks ? blocks : sv::kAppendBlocks), dim3(256),
                       0, stream, d, (uint32_t)(d.head_dim / 8), (uint32_t)chunks_token, sv::page_shift(d.page_size),
                       total);
    return sv::launched();
}

}  // extern "C"
