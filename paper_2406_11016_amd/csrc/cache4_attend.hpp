// Attention over a cache in 4 bits for gfx950 (MI355X): kernels of spec_cache_attend4.
// (Included by the sources of the two storage types.)
//
// The work is cut as for caches in 16 bits (cache_attend.hpp).  Tasks of many rows are
// that kernel's, whose matrix instructions then bound it, with tiles widened on their way to
// LDS; tasks of few rows go by cache4_direct.hpp.  (8 sequences of up to 999 tokens behind 2,000,
// 156 GFLOP: 201 us and 17.7 for the join, 188 and 17.8 in 16 bits, with 28 % fewer vector instructions; 128 rows with keys
// from the L2: 1,000 TFLOP/s.)
#pragma once

#include "cache4_direct.hpp"
#include "cache_attend.hpp"

namespace sv {
namespace {

// A kernel's tasks of a kind: kRows > 0, waves that split the rows of tiles; kRows < 0, -kRows row tiles of 16 for
// few rows; 0, there are none.
template <int D, int kRows>
constexpr int kTaskLds = kRows > 0 ? kTiles<In4, D> : kRows < 0 ? Direct<D>::lds(-kRows) : 0;
template <int D, int kPrefix, int kRows>
constexpr int kLds4 = kTaskLds<D, kPrefix> > kTaskLds<D, kRows> ? kTaskLds<D, kPrefix> : kTaskLds<D, kRows>;

// Workgroups of a CU at a time, which the registers have to be enough for (and attend4_plan counts on).
template <int D, int kPrefix, int kRows>
constexpr int kResident = D > 128 && !(kPrefix == 0 && kRows == -1) ? 1 : 2;

struct Shared4 {
    float wave_stats[4][2][48];
    __attribute__((aligned(8))) int flags[2];  // poison and special values, or the poison of two tasks in turn
};

template <class T, int D, int kRows, Kind kKind>
__device__ __forceinline__ void run4(const AttendArgs& a, const Totals& t, const Deal& deal, const Batch& batch, uint32_t w,
                                     char* smem, Shared4& shared) {
    if constexpr (kRows > 0)
        run<T, In4, D, kRows, kKind>(a, t, deal, batch, w, smem, (float(*)[2][32])shared.wave_stats, &shared.flags[0],
                                     &shared.flags[1]);
    else
        run_direct<T, D, -kRows, kKind>(a, t, deal, batch, w, smem, shared.wave_stats, shared.flags);
}

template <class T, int D, int kPrefix, int kRows>
__global__ void __launch_bounds__(kThreads, (kResident<D, kPrefix, kRows>)) attend4_kernel(AttendArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ uint32_t wave_sums[4][2];
    __shared__ Shared4 shared;
    const Split& split = a.split;
    int32_t* const words = (int32_t*)(smem + kLds4<D, kPrefix, kRows>);
    const Batch batch{words, (uint32_t*)words + split.batch + 1, words + 2 * (split.batch + 1)};
    if (threadIdx.x == 0) shared.flags[0] = shared.flags[1] = 0;
    const Totals t = sum_batch(split, batch, wave_sums);
    if (blockIdx.x == 0)  // for the kernel that joins the parts
        for (int b = threadIdx.x; b <= split.batch; b += kThreads) {
            a.cum_tokens[b] = batch.cum_tokens[b];
            a.cum_cost[b] = batch.cum_cost[b];
            if (b == 0) *a.totals = t;
        }
    if constexpr (kPrefix == 0) {
        if (blockIdx.x < t.own.groups)
            run4<T, D, kRows, kJoined>(a, t, t.own, batch, place_in_xcd(blockIdx.x, t.own.groups), smem, shared);
    } else if (blockIdx.x < t.prefix.groups) {
        run4<T, D, kPrefix, kShared>(a, t, t.prefix, batch, place_in_xcd(blockIdx.x, t.prefix.groups), smem, shared);
    } else if (blockIdx.x - t.prefix.groups < t.own.groups) {
        run4<T, D, kRows, kOwn>(a, t, t.own, batch, blockIdx.x - t.prefix.groups, smem, shared);
    }
}

template <class T, int D>
sv_status_t launch4(const AttendArgs& a, hipStream_t stream) {
    const AttendPlan& plan = a.split.plan;
    auto go = [&](auto prefix, auto own) {
        constexpr int kPrefix = decltype(prefix)::value, kRows = decltype(own)::value;
        hipLaunchKernelGGL((attend4_kernel<T, D, kPrefix, kRows>), dim3((uint32_t)plan.groups), dim3(kThreads),
                           (kLds4<D, kPrefix, kRows>) + batch_bytes(a), stream, a);
    };
    constexpr std::integral_constant<int, 0> none{};
    constexpr std::integral_constant<int, -1> few{};
    constexpr int kMost = kMaxTaskRows<D> / 32;
    constexpr std::integral_constant<int, kMost> most{};
    const int prefix = plan.joined ? 0 : plan.prefix_direct ? -1 : 1;
    if constexpr (D > 128) {
        constexpr std::integral_constant<int, 1> one{};
        const bool own_one = !plan.own_direct && plan.own_rows == 32, prefix_one = plan.prefix_rows == 32;
        if (plan.own_direct)
            prefix == 0 ? go(none, few) : prefix < 0 ? go(few, few) : prefix_one ? go(one, few) : go(most, few);
        else if (own_one)
            prefix == 0 ? go(none, one) : prefix_one ? go(one, one) : go(most, one);
        else
            prefix == 0 ? go(none, most) : go(most, most);
    } else {
        // (a prefix of few rows in all is for any of up to 48: the rows that there are not cost little there)
        constexpr std::integral_constant<int, -2> more{};
        constexpr std::integral_constant<int, -3> some{};
        constexpr std::integral_constant<int, 2> two{};
        const bool prefix_two = plan.prefix_rows == 64;
        auto direct = [&](auto own) { prefix == 0 ? go(none, own) : prefix_two ? go(two, own) : go(most, own); };
        if (plan.prefix_direct)
            go(some, few);
        else if (plan.own_direct)
            plan.own_rows == 16 ? direct(few) : plan.own_rows == 32 ? direct(more) : direct(some);
        else if (plan.own_rows == 64)
            prefix == 0 ? go(none, two) : prefix_two ? go(two, two) : go(most, two);
        else
            prefix == 0 ? go(none, most) : go(most, most);
    }
    if (plan.whole_tasks) return hipGetLastError() == hipSuccess ? SV_OK : SV_ERR_HIP;
    return launch_join<T, D>(a, stream);
}

template <class T>
sv_status_t launch4_dim(const AttendArgs& a, int32_t head_dim, hipStream_t stream) {
    switch (head_dim) {
        case 64: return launch4<T, 64>(a, stream);
        case 80: return launch4<T, 80>(a, stream);
        case 96: return launch4<T, 96>(a, stream);
        case 128: return launch4<T, 128>(a, stream);
        default: return launch4<T, 256>(a, stream);
    }
}

}  // namespace
}  // namespace sv
