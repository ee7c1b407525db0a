// Attention of a step's new tokens to the paged cache, behind a prefix that the
// batch shares, for gfx950 (MI355X): kernels of spec_cache_attend.
// (Included by the sources of the two storage types.)
//
// Work is cut into tasks of up to 128 query rows of one key/value head (a row
// is a token and one of its heads) against a run of keys, and a task into units
// of kKeys keys.  The rows of the whole batch share the prefix's tasks, and each
// sequence has tasks of its own for its own keys (where those are many and full,
// they take the prefix along, see joined_pays).  The units of all tasks in
// order are dealt to the grid's workgroups in equal runs, so lengths need not be
// known on the host and few long sequences fill the chip as well as many short
// ones; what a workgroup computes of a task is a part (running maximum, sum and
// unnormalised output of every row), and a second kernel joins a row's parts.
//
// What bounds it, at head_dim 128 with 4 heads to a key/value head: many sequences
// without a prefix, the memory (64 sequences of 0 to 4,096 cached tokens, 815 MB:
// 165 us, 4.9 TB/s); rows that share many keys, the issue of the matrix
// and vector instructions by turns (8 sequences of up to 999 tokens behind 2,000, 156
// GFLOP: 190 us, 820 TFLOP/s; 64 of up to 9 behind 16,384, 124 GFLOP: 147 us, 845); few
// rows and keys, the latency of a workgroup's run (the batch's sums 2 us, finding the
// task 1 to 2, its first tiles 3, writing its part 3: one sequence of 11 tokens
// behind 1,900, 14 us).  The join takes 3 to 18 us.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

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

namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

#define SV_LDS __attribute__((address_space(3)))

// kBias: the largest weight of a row in log2, but for rises of the maximum that are let pass (up to 8).
struct AttF16 {
    // 2^15 is the largest power of two in fp16, so weights down to 2^-31 of the largest are
    // not lost to 0 (2^-24 without it)
    static constexpr float kBias = 7.0f;
    typedef _Float16 V8 __attribute__((ext_vector_type(8)));
    typedef _Float16 V4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x16 mma(V8 a, V8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ bool special(uint32_t bits) { return (bits & 0x7c00u) == 0x7c00u; }
    static __device__ __forceinline__ float value(uint32_t bits) {
        return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    }
};
struct AttBF16 {
    // bf16 holds numbers up to fp32's largest, 2^128: so the sums of 2^20 largest weights (2^8 more
    // for the time being) and any finite values are finite, and what is lost at the other end are products
    // below 2^-98 (2^-126 without it)
    static constexpr float kBias = -28.0f;
    typedef __bf16 V8 __attribute__((ext_vector_type(8)));
    typedef __bf16 V4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x16 mma(V8 a, V8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ bool special(uint32_t bits) { return (bits & 0x7f80u) == 0x7f80u; }
    static __device__ __forceinline__ float value(uint32_t bits) { return __uint_as_float(bits << 16); }
};

constexpr int kThreads = 256;
constexpr int kKeys = kAttendKeys;

// Scores, in log2 units, up to which a weight's argument is taken in one fused
// multiply-add, score * scale - reference: the reference there is a product rounded to 32
// bits, so all weights of a row are off by one common factor, 2^(2^-12) at most.  Behind it the factor
// would not fit the weights' type in the end, and a score loses its reference first.
constexpr float kFarScores = 4096.0f;

// A value that is the same in every lane, in a scalar register.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

// The same value, of which the compiler knows nothing: what is computed from it is
// computed there, not kept in registers from before.
template <class X>
__device__ __forceinline__ X forget(X x) {
    asm volatile("" : "+v"(x));
    return x;
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// max or sum over the two halves of the wave, in every lane
__device__ __forceinline__ float halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The batch in LDS: sums over it before each sequence, and its lengths (-1: bad).
struct Batch {
    int32_t* cum_tokens;  // [batch + 1]
    uint32_t* cum_cost;   // [batch + 1]
    int32_t* lengths;     // [batch]
};
__device__ __forceinline__ Sequence sequence(const Batch& batch, int32_t b) {
    const int32_t length = uniform(batch.lengths[b]);
    return Sequence{uniform(batch.cum_tokens[b + 1]) - uniform(batch.cum_tokens[b]), max(length, 0), length < 0};
}

// Every workgroup sums the batch for itself (a few loads and one scan: 2 us, less than
// a launch of its own).
__device__ __forceinline__ Totals sum_batch(const Split& a, const Batch& batch, uint32_t (*wave_sums)[2]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (a.batch + kThreads - 1) / kThreads;
    const int b0 = min(tid * each, a.batch), b1 = min(b0 + each, a.batch);
    if (a.plan.own_tiles > 4) {  // a wave a sequence, its row tiles by lane
        for (int b = uniform(wave); b < a.batch; b += kThreads / 64) {
            const Sequence s = sequence(a, b);
            uint32_t cost = 0;
            for (int32_t rt = lane; rt < a.plan.own_tiles; rt += 64) cost += tile_cost(a, s, rt);
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) cost += __shfl_xor(cost, m);
            if (lane == 0) batch.cum_cost[b + 1] = cost;
        }
        __syncthreads();
    }
    uint32_t tokens = 0, cost = 0;
    for (int b = b0; b < b1; ++b) {
        const Sequence s = sequence(a, b);
        tokens += s.count;
        if (a.plan.own_tiles > 4) {
            cost += batch.cum_cost[b + 1] * (uint32_t)a.kv_heads;
        } else {
            for (int32_t rt = 0; rt < a.plan.own_tiles; ++rt) cost += tile_cost(a, s, rt) * (uint32_t)a.kv_heads;
        }
        batch.cum_tokens[b + 1] = tokens;
        batch.cum_cost[b + 1] = cost;
        batch.lengths[b] = s.bad ? -1 : s.length;
    }
    uint32_t t = tokens, u = cost;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t ot = __shfl_up(t, d), ou = __shfl_up(u, d);
        if (lane >= d) {
            t += ot;
            u += ou;
        }
    }
    if (lane == 63) {
        wave_sums[wave][0] = t;
        wave_sums[wave][1] = u;
    }
    __syncthreads();
    uint32_t bt = t - tokens, bu = u - cost;
    for (int w = 0; w < wave; ++w) {
        bt += wave_sums[w][0];
        bu += wave_sums[w][1];
    }
    for (int b = b0; b < b1; ++b) {
        batch.cum_tokens[b + 1] += bt;
        batch.cum_cost[b + 1] += bu;
    }
    if (tid == 0) {
        batch.cum_tokens[0] = 0;
        batch.cum_cost[0] = 0;
    }
    __syncthreads();
    return totals(a, uniform(batch.cum_tokens[a.batch]), uniform(batch.cum_cost[a.batch]));
}

// A sequence's own task that holds place `at` of the cost of one key/value head: its
// row tile, and where its cost starts.  64 tiles at a time, one a lane.
__device__ __forceinline__ int32_t find_tile(const Split& a, const Sequence& s, uint32_t at, uint32_t& start) {
    start = 0;
    if (a.plan.own_tiles == 1) return 0;
    const int lane = forget((int)threadIdx.x) & 63;
    uint32_t before = 0;
    for (int32_t base = 0; base < a.plan.own_tiles; base += 64) {
        const uint32_t own = (base + lane < a.plan.own_tiles) ? tile_cost(a, s, base + lane) : 0u;
        uint32_t end = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = (uint32_t)__builtin_amdgcn_ds_bpermute((lane - d) * 4, (int)end);
            if (lane >= d) end += o;
        }
        const uint64_t over = __ballot(before + end > at);
        if (over != 0) {
            const int l = __builtin_ctzll(over);
            start = before + (uint32_t)__builtin_amdgcn_readlane((int)(end - own), l);
            return base + l;
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)end, 63);
    }
    return 0;  // (not reached: `at` is below the sum of all tiles)
}

// A task, in scalar registers.
__device__ __forceinline__ Segment uniform(Segment g) {
    g.task = uniform(g.task);
    g.task_start = uniform(g.task_start);
    g.units = uniform(g.units);
    g.prefix_units = uniform(g.prefix_units);
    g.offset = uniform(g.offset);
    g.kv_head = uniform(g.kv_head);
    g.b = uniform(g.b);
    g.row0 = uniform(g.row0);
    g.count = uniform(g.count);
    g.length = uniform(g.length);
    g.bad = uniform((int32_t)g.bad) != 0;
    return g;
}
template <class SequenceOf>
__device__ __forceinline__ Segment own_task_at(const Split& a, const uint32_t* cum_cost, uint32_t u, SequenceOf sequence_of) {
    return uniform(own_task(a, cum_cost, u, sequence_of, [&](const Sequence& s, uint32_t at, uint32_t& start) {
        return find_tile(a, s, at, start);
    }));
}

// What a workgroup's tasks are.
enum Kind : int {
    kShared,  // the prefix's, for rows of the whole batch
    kOwn,     // the sequences' own keys
    kJoined   // both in one task, first the prefix
};

// ---------------------------------------------------------------------------
// one segment
// ---------------------------------------------------------------------------

template <int D>
struct Shape {
    static constexpr int kPitch = D <= 64 ? 64 : D <= 128 ? 128 : 256;  // elements of a row in LDS
    static constexpr int kChunks = kPitch / 8;                         // of 16 bytes
    static constexpr int kTile = kKeys * kPitch * 2;                   // bytes of a tile of K or of V
    static constexpr int kStage = 2 * kTile;                           // of both
    static constexpr int kSteps = D / 16;                              // products over head_dim
    static constexpr int kOuts = (D + 31) / 32;                        // 32-wide pieces of the output
    static constexpr int kRowsLoad = 1024 / (kPitch * 2);              // rows of one wave-wide load
    static constexpr int kLoads = 16 / kRowsLoad;                      // loads of a wave for its run of 16 rows
};

// Rows of K and V lie in LDS with their 16-byte chunks permuted by the row, so
// that both reads are free of bank conflicts: 16 lanes that read the same chunk
// of 16 consecutive rows (K), and 8 rows of 64 adjacent bytes (V, transposing).
template <int D>
__device__ __forceinline__ int swizzle(int row) {
    if constexpr (Shape<D>::kPitch == 64) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    return ((row & 3) << 2) | ((row >> 2) & 3);
}

// 16 bytes a lane from memory straight to LDS at `lds` + 16 * lane.  The
// compiler's own form of this load is followed by waits for every load in
// flight wherever LDS is read; here the waits are written out.  (M0 holds the
// LDS address of the load, which reads it at issue; it is left as it was.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, const void* base, uint32_t offset) {
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0)
                 : "s"(lds), "v"(offset), "s"(base)
                 : "memory");
}
// Own loads to LDS have landed, own LDS reads are done; then the workgroup's
// barrier.  (The wait is the compiler's own instruction, so that it knows that
// nothing is in flight: it would else wait for the next unit's loads where it
// first needs a register that was loaded before the loop.)
__device__ __forceinline__ void stage_barrier() {
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

// Nothing is moved across: the reads written before a block of matrix products are
// issued before it, so that their latency passes behind it.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// Own LDS accesses are done; then the workgroup's barrier.  (Loads and stores of
// memory stay under way.)
__device__ __forceinline__ void lds_barrier() {
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

// Whether this thread's share of a tile holds infinities or NaN; `clear` makes them zeros.
template <class T, int D>
__device__ __forceinline__ bool special_chunks(char* tile, bool clear) {
    using S = Shape<D>;
    uint32_t found = 0;
    const uint32_t ones = forget(~0u);
#pragma unroll 1
    for (int at = forget((int)threadIdx.x) * 16; at < S::kTile; at += kThreads * 16) {
        // (a chunk behind head_dim holds what was there before: nothing reads it)
        if (D != S::kPitch && (((at / 16) % S::kChunks) ^ swizzle<D>(at / (S::kPitch * 2))) * 8 >= D) continue;
        u32x4 x = *(u32x4*)(tile + at);
        uint32_t here = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool low = T::special(x[i] & 0xffffu), high = T::special(x[i] >> 16);
            x[i] &= (low ? 0u : ones >> 16) | (high ? 0u : ones << 16);
            here |= (uint32_t)low | (uint32_t)high;
        }
        if (clear && here) *(u32x4*)(tile + at) = x;
        found |= here;
    }
    return found != 0;
}

// A workgroup's way through its run of the work: the segment at hand, and the
// pages that this wave stages of it, a run of 16 rows of each unit.
template <int D, Kind kKind>
struct Work {
    using S = Shape<D>;
    const AttendArgs& a;
    const Totals& t;
    const Batch& batch;
    const uint32_t lds;         // LDS address of the tiles
    const uint32_t group, end;  // this workgroup, and where its run of the cost ends
    Segment g;                  // first .. end: units of the task's keys
    int64_t place;              // of its part
    bool whole;                 // it is the whole task, and has no part
    uint32_t at;                // place in the cost behind it
    uint32_t paged;             // lane l has the place in the caches of this wave's rows of unit `paged` + l
    uint32_t row_low, row_high;
    bool poison;                // (one of them would have been on a page that there is not)

    // To the next segment; false if there is none.
    __device__ __forceinline__ bool advance() {
        if (at >= end) return false;
        if constexpr (kKind == kShared)
            g = uniform(prefix_task(a.split, t, at));
        else
            g = own_task_at(a.split, batch.cum_cost, at, [&](int32_t b) { return sequence(batch, b); });
        cut(g, at, end);
        if (g.first == g.end) return false;  // (the run ends within the task's cost of starting)
        whole = kKind == kJoined && whole_task(a.split, g);
        place = part_place(a.split, g, group);
        at = g.task_start + g.end;
        g.first += g.offset;
        g.end += g.offset;
        poison = g.bad;
        paged = g.first;
        look_up();
        if constexpr (kKind != kShared) look_behind();
        return true;
    }
    // A sequence with a page that there is not has no outputs: pages that only later row tiles need.
    __device__ __forceinline__ void look_behind() {
        const int end = own_end(a.split, g), last = g.length + g.count - 1;
        if (g.bad || end > last) return;
        const int32_t* const table = a.block_table + (int64_t)g.b * a.split.max_pages;
        for (int j = ((end - 1) >> a.split.page_shift) + 1 + forget((int)threadIdx.x); j <= last >> a.split.page_shift;
             j += kThreads)
            if ((uint32_t)table[j] >= (uint32_t)a.num_pages) poison = true;
    }
    // Whether unit u is of the prefix, its first key there or in the sequence, and the last key that there is.
    __device__ __forceinline__ bool in_prefix(uint32_t u) const {
        return kKind == kShared || (kKind == kJoined && u < g.prefix_units);
    }
    __device__ __forceinline__ int first_key(uint32_t u) const {
        return (int)(kKind != kJoined || u < g.prefix_units ? u : u - g.prefix_units) * kKeys;
    }
    __device__ __forceinline__ int last_key(bool prefix) const {
        return prefix ? a.prefix_len - 1 : own_end(a.split, g) - 1;
    }
    __device__ __forceinline__ void look_up() {
        const int lane = forget((int)threadIdx.x) & 63, wave = uniform((int32_t)(threadIdx.x >> 6));
        const uint32_t u = smaller(paged + lane, g.end - 1);
        const bool prefix = in_prefix(u);
        const int32_t* const table = prefix ? a.prefix_table : a.block_table + (int64_t)max(g.b, 0) * a.split.max_pages;
        const int first = run_start(first_key(u), wave, last_key(prefix));
        int page = (prefix || !g.bad) ? table[first >> a.split.page_shift] : 0;
        if ((uint32_t)page >= (uint32_t)a.num_pages) {
            page = 0;
            poison = true;
        }
        const int64_t row = (int64_t)page * a.page_stride + (int64_t)(g.kv_head << a.split.page_shift) * D +
                            (first & ((1 << a.split.page_shift) - 1)) * D;
        row_low = (uint32_t)row;
        row_high = (uint32_t)(row >> 32);
    }
    // This wave's first row of unit u, in the caches.
    __device__ __forceinline__ int64_t row_of(uint32_t u) {
        if (u - paged == 64) {
            paged = u;
            look_up();
        }
        const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)row_low, (int)(u - paged));
        const uint32_t high = (uint32_t)__builtin_amdgcn_readlane((int)row_high, (int)(u - paged));
        return (int64_t)((uint64_t)high << 32 | low);
    }
    // And the last of its 16 rows that there is: those behind repeat it.
    __device__ __forceinline__ int last_row(uint32_t u) const {
        const int last = last_key(in_prefix(u));
        return last - run_start(first_key(u), uniform((int32_t)(threadIdx.x >> 6)), last);
    }
    // This wave's 16 rows of a unit of K (V), to its place in LDS.
    template <bool kFull>
    __device__ __forceinline__ void stage(const uint16_t* cache, int64_t row, int last, uint32_t to) const {
        const uint32_t lane = (uint32_t)forget((int)threadIdx.x) & 63;
        const int load_row = (int)(lane / S::kChunks), load_chunk = (int)(lane % S::kChunks);
        const int wave = uniform((int32_t)(threadIdx.x >> 6));
#pragma unroll
        for (int j = 0; j < S::kLoads; ++j) {
            const int in_run = j * S::kRowsLoad + load_row;
            const int chunk = load_chunk ^ swizzle<D>(load_row) ^ swizzle<D>(j * S::kRowsLoad);
            const uint32_t offset = (uint32_t)((kFull ? load_row : min(in_run, last)) * D + chunk * 8) * 2;
            if (D == S::kPitch || chunk * 8 < D)
                load_to_lds(lds + to + wave * (16 * S::kPitch * 2) + j * 1024,
                            cache + row + (kFull ? j * S::kRowsLoad * D : 0), offset);
        }
    }
    __device__ __forceinline__ void stage_first() {
        const int64_t row = row_of(g.first);
        const int last = last_row(g.first);
        stage<false>(a.k_cache, row, last, 0);
        stage<false>(a.v_cache, row, last, S::kTile);
    }
};

// The part of a task's rows over a run of its units.  The four waves are WR x WK x
// WD: WR split the rows (32 each), WK a unit's blocks of 32 keys, and WD the
// output's head_dim (those do the same scores twice; it is for tasks of few rows,
// which wait for memory).
//
// The products are taken transposed.  S^T = K Q^T leaves a query row's scores in
// the registers of two lanes (l and l + 32), so the maximum and the sum over the
// keys need one exchange between lanes, and the running maximum, the sum and the
// rescaling of the output are one value a lane.  P^T then is the B operand of
// O^T = V^T P^T as it stands, with V^T from LDS by transposing reads in the same order
// of keys.  It is rounded to the storage type for that, half a step a weight: what is
// rounded off would be a second product, half of a unit's matrix instructions again.
// (The sum of the weights is of the unrounded ones.)
//
// K runs one unit ahead of V: while one unit's scores become weights, on the
// vector units, the matrix units make the next one's scores, product by product in
// between (the two overlap in one wave only if its instructions alternate).  Both
// are staged two deep in LDS, with one barrier between units.
template <class T, int D, int WR, Kind kKind>
__device__ __forceinline__ bool segment(Work<D, kKind>& work, char* smem, float (*wave_stats)[2][32], int* poison_flag,
                                        int* special_flag) {
    using S = Shape<D>;
    using V8 = typename T::V8;
    constexpr int WK = WR == 4 ? 1 : 2, WD = 4 / (WR * WK);
    constexpr int NS = 2 / WK;                        // blocks of 32 keys of a wave
    constexpr int kPieces = (S::kOuts + WD - 1) / WD;  // pieces of the output of a wave: every WD-th
    constexpr int kMmas = NS * S::kSteps;              // products of a unit's scores
    constexpr int kAhead = kMmas < 4 ? kMmas : 4;      // those of them whose reads of K are under way
    constexpr int kMmasV = 2 * NS * kPieces, kAheadV = kMmasV < 4 ? kMmasV : 4;  // the same of the output and V
    // (`lane` is forgotten where a part of the work begins: what is made from it there would else be kept in registers
    // from before the loops on)
    const int tid = threadIdx.x, lane = forget(tid & 63), half = lane >> 5;
    const int wave = uniform(tid >> 6);
    const int wr = wave % WR, wk = wave / WR % WK, wd = wave / (WR * WK);
    const AttendArgs& a = work.a;
    const Segment g = work.g;
    const int32_t* const cum_tokens = work.batch.cum_tokens;

    // the row of this lane
    struct Row {
        int b, token, head;
        bool live;
    };
    auto row_of = [&](int lane) {
        const int row = g.row0 + wr * 32 + (lane & 31);
        const int flat = (int)((uint32_t)row / (uint32_t)a.split.group);
        Row r{g.b, flat, g.kv_head * a.split.group + (row - flat * a.split.group), flat < g.count};
        if (kKind == kShared) {
            r.live = flat < cum_tokens[a.split.batch];
            r.b = r.live ? find(cum_tokens, a.split.batch, flat) : 0;
            r.token = r.live ? flat - cum_tokens[r.b] : 0;
        }
        return r;
    };
    const Row mine = row_of(lane);
    const int own_limit = g.length + mine.token + 1;  // keys of its own that this row sees
    const int own_first = kKind == kShared ? 0 : own_common(a.split, g);
    // (of the segment at hand, not of the one that `work` has turned to)
    auto in_prefix = [&](uint32_t u) { return kKind == kShared || (kKind == kJoined && u < g.prefix_units); };

    V8 q[S::kSteps];
    {
        const uint16_t* const from =
            a.q + mine.b * a.q_stride[0] + mine.token * a.q_stride[1] + mine.head * a.q_stride[2] + half * 8;
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s) {
            u32x4 x = {0, 0, 0, 0};
            if (mine.live) x = *(const u32x4*)(from + 16 * s);
            q[s] = __builtin_bit_cast(V8, x);
        }
    }
    f32x16 o[kPieces];
    float top, sum = 0.0f;  // top: scores as they come from the product
    bool far;               // some row's is beyond kFarScores: the scores of the unit at hand have lost it already

    // Places of this lane's reads.  The swizzle flips bits of the chunk's number
    // only, so a read's constant part comes by an exclusive or (chunk) or as an
    // offset (key).  V's 4 keys x 16 values blocks are transposed by the read: lane i
    // of 16 gets column i.
    const int block0 = wk * NS * (32 * S::kPitch * 2);
    const int k_at = block0 + (lane & 31) * (S::kPitch * 2) + ((half ^ swizzle<D>(lane & 31)) * 16);
    int v_at[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = lane & 15, r = 8 * j + 4 * half + i / 4;
        const int chunk = ((lane >> 4) & 1) * 2 + (i % 4) / 2;
        v_at[j] = block0 + r * (S::kPitch * 2) + (((chunk + 4 * wd) ^ swizzle<D>(r)) * 16) + (i & 1) * 8;
    }

    // Key 0 of unit u, the keys that this row sees of its sequence or prefix, and whether a row sees less than all.
    auto base_of = [&](uint32_t u) { return (int)(kKind != kJoined || in_prefix(u) ? u : u - g.prefix_units) * kKeys; };
    auto limit_of = [&](uint32_t u) { return in_prefix(u) ? a.prefix_len : own_limit; };
    auto partial_of = [&](uint32_t u) {
        return base_of(u) + kKeys > (in_prefix(u) ? a.prefix_len : own_first);
    };
    auto k_read = [&](const char* tile, int m) {  // K's rows and columns of product m
        return *(const V8*)(tile + (k_at ^ (m / NS * 32)) + m % NS * (32 * S::kPitch * 2));
    };
    // Unit u's scores of keys that a row does not see, and then their maximum.
    auto mask = [&](uint32_t u, f32x16(&p)[NS]) {
        const int key = base_of(u) + wk * NS * 32 + 4 * half, limit = limit_of(u);
        float most = -INFINITY;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < 16; ++i) {  // key of register i: 8 (i / 4) + 4 half + i % 4
                p[s][i] = key + s * 32 + 8 * (i / 4) + i % 4 < limit ? p[s][i] : -INFINITY;
                most = fmaxf(most, p[s][i]);
            }
        return most;
    };
    // Whether, and then the scores without it.
    auto look_far = [&]() {
        far = __any(fabsf(top * a.scale_log2) > kFarScores && top != -INFINITY);
    };
    auto take_off = [&](f32x16(&p)[NS]) {
        if (!far) return;
        const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int s = 0; s < NS; ++s) p[s] -= ref;
    };
    // Moves the reference of the weights to unit u's maximum: they stay relative to a maximum of earlier units as
    // long as the new one is within 2^8 of it, so nothing is rescaled for small rises.
    auto refer = [&](auto full, uint32_t u, f32x16(&p)[NS], float most) {
        if (!decltype(full)::value && partial_of(u)) most = mask(u, p);
        most = halves_max(most);
        // (the difference of two scores near one another is exact; next to a far one a.lazy would be rounded)
        if (__any(most - top > a.lazy)) {
            const float now = fmaxf(top, most);
            const float by = (now == -INFINITY) ? 1.0f : exp2_hw((top - now) * a.scale_log2);
            sum *= by;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) o[i] *= by;
            top = now;
            look_far();
        }
        take_off(p);
    };
    // One unit: p's scores are masked and referred to; `next` gets the scores of the unit after it.  The segment's
    // even units lie in the first two tiles of LDS (K, V), its odd ones in the others.  `full`: it and the two units
    // behind it are of the same segment, of one table, and every row sees all their keys.
    int64_t row = 0;  // this wave's first row of the unit whose K was staged last
    auto step = [&](auto full, uint32_t u, auto odd, f32x16(&p)[NS], f32x16(&next)[NS]) {
        constexpr bool kFull = decltype(full)::value;
        constexpr int kHere = decltype(odd)::value * S::kStage, kThere = S::kStage - kHere;
        const bool more = kFull || u + 1 < g.end;
        char* const v_tile = smem + kHere + S::kTile;
        float shift = (far || top == -INFINITY) ? T::kBias : fmaf(-top, a.scale_log2, T::kBias);
        float add = 0.0f;
        auto weigh = [&](int from, int to) {
#pragma unroll
            for (int i = from; i < to; ++i) {
                p[i / 16][i % 16] = exp2_hw(fmaf(p[i / 16][i % 16], a.scale_log2, shift));
                add += p[i / 16][i % 16];
            }
        };

        stage_barrier();  // K of the next unit and V of this one are there, and every wave has done with those before
        if (more) {
            shift = forget(shift);  // (else the weights' arguments are made before this branch, for both)
            work.template stage<kFull>(a.v_cache, row, kFull ? 0 : work.last_row(u + 1), kThere + S::kTile);
            if (kFull || u + 2 < g.end) {
                row = work.row_of(u + 2);
                work.template stage<kFull>(a.k_cache, row, kFull ? 0 : work.last_row(u + 2), kHere);
            }
            const char* const tile = smem + kThere;
            V8 k[kAhead + 1];
#pragma unroll
            for (int m = 0; m < kAhead; ++m) k[m] = k_read(tile, m);
#pragma unroll
            for (int s = 0; s < NS; ++s) next[s] = f32x16(0.0f);
#pragma unroll
            for (int m = 0; m < kMmas; ++m) {
                in_order();
                if (m + kAhead < kMmas) k[(m + kAhead) % (kAhead + 1)] = k_read(tile, m + kAhead);
                next[m % NS] = T::mma(k[m % (kAhead + 1)], q[m / NS], next[m % NS]);
                weigh(m * NS * 16 / kMmas, (m + 1) * NS * 16 / kMmas);
            }
            in_order();
        } else {
            weigh(0, NS * 16);
        }
        sum += add;

        bool special = false;
        if (!kFull && partial_of(u)) {
            if (__any(special_chunks<T, D>(v_tile, false))) *special_flag = 1;
            lds_barrier();
            special = uniform(*special_flag) != 0;
        }
        if (special) {
            // A masked key's weight is 0, but 0 times an infinity or NaN is not.
            // Rows take such values from the keys that they see, here; then they
            // are zeros for the product.
            const int key0 = base_of(u) + wk * NS * 32, limit = limit_of(u), half = forget(lane) >> 5;
#pragma unroll 1
            for (int k = 0; k < NS * 32; ++k) {
                const bool sees = key0 + k < limit;
                const char* const v_row = v_tile + block0 + k * (S::kPitch * 2) + half * 8;
#pragma unroll
                for (int i = 0; i < kPieces; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const u32x2 x = *(const u32x2*)(v_row + ((4 * (i * WD + wd) + r) ^ swizzle<D>(k)) * 16);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t bits = (x[e / 2] >> (16 * (e % 2))) & 0xffffu;
                            if (sees && T::special(bits)) o[i][4 * r + e] += T::value(bits);
                        }
                    }
            }
            lds_barrier();
            special_chunks<T, D>(v_tile, true);
            if (tid == 0) *special_flag = 0;
            lds_barrier();
        }
        // product m: 16 keys (m / kPieces) for one piece of the output
        auto v_read = [&](int m) {
            i16x4 x[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
                x[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SV_LDS i16x4*)(SV_LDS char*)(
                    v_tile + (v_at[j] ^ (m % kPieces * WD * 64)) + m / kPieces * (16 * S::kPitch * 2)));
            return __builtin_bit_cast(V8, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
        };
        V8 v[kAheadV + 1], w8;
#pragma unroll
        for (int m = 0; m < kAheadV; ++m) v[m] = v_read(m);
        float most = -INFINITY;
#pragma unroll
        for (int m = 0; m < kMmasV; ++m) {
            const int block = m / kPieces;
            if (m % kPieces == 0) {
                f32x8 w;
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = p[block / 2][8 * (block % 2) + i];
                w8 = __builtin_convertvector(w, V8);
            }
            in_order();
            if (m + kAheadV < kMmasV) v[(m + kAheadV) % (kAheadV + 1)] = v_read(m + kAheadV);
            o[m % kPieces] = T::mma(v[m % (kAheadV + 1)], w8, o[m % kPieces]);
#pragma unroll
            for (int i = m * NS * 16 / kMmasV; i < (m + 1) * NS * 16 / kMmasV; ++i) most = fmaxf(most, next[i / 16][i % 16]);
        }
        in_order();
        if (more) refer(full, u + 1, next, most);
    };

    f32x16 scores[2][NS];
    {
        stage_barrier();  // the first unit
        if (g.first + 1 < g.end) {
            row = work.row_of(g.first + 1);
            work.template stage<false>(a.k_cache, row, work.last_row(g.first + 1), S::kStage);
        }
        float most = -INFINITY;
#pragma unroll
        for (int s = 0; s < NS; ++s) scores[0][s] = f32x16(0.0f);
        V8 k[kAhead + 1];
#pragma unroll
        for (int m = 0; m < kAhead; ++m) k[m] = k_read(smem, m);
#pragma unroll
        for (int m = 0; m < kMmas; ++m) {
            in_order();
            if (m + kAhead < kMmas) k[(m + kAhead) % (kAhead + 1)] = k_read(smem, m + kAhead);
            scores[0][m % NS] = T::mma(k[m % (kAhead + 1)], q[m / NS], scores[0][m % NS]);
        }
        in_order();
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, scores[0][s][i]);
        if (partial_of(g.first)) most = mask(g.first, scores[0]);
        top = halves_max(most);
        look_far();
        take_off(scores[0]);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) o[i] = f32x16(0.0f);
    }
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, 1> k1{};
    uint32_t u = g.first;
    while (u < g.end) {
        // up to here every row sees all keys of the units, which are of the table of unit u
        const uint32_t full = in_prefix(u)
                                  ? smaller(g.end, (uint32_t)a.prefix_len / kKeys)
                                  : smaller(g.end, (kKind == kJoined ? g.prefix_units : 0u) + (uint32_t)own_first / kKeys);
        for (; u + 4 <= full; u += 2) {
            step(std::true_type(), u, k0, scores[0], scores[1]);
            step(std::true_type(), u + 1, k1, scores[1], scores[0]);
        }
        step(std::false_type(), u, k0, scores[0], scores[1]);
        if (u + 1 < g.end) step(std::false_type(), u + 1, k1, scores[1], scores[0]);
        u += 2;
    }

    // ---- join the waves that split the keys, then write
    auto finish = [&](int lane, bool whole, int64_t place) {
        const int half = lane >> 5;
        if constexpr (WK > 1) {
            if (half == 0) {
                wave_stats[wave][0][lane] = top;
                wave_stats[wave][1][lane] = sum;
            }
            lds_barrier();
            const float(*const other)[32] = wave_stats[wave + (wk == 0 ? WR : -WR)];
            const float other_top = other[0][lane & 31], now = fmaxf(top, other_top);
            const float ref = (now == -INFINITY) ? 0.0f : now;
            const float by = exp2_hw((top - ref) * a.scale_log2);
            const float own = by * sum, others = exp2_hw((other_top - ref) * a.scale_log2) * other[1][lane & 31];
            sum = wk == 0 ? own + others : others + own;
            top = now;
            // piece i of the output is summed by the wave wk = i % WK
            f32x4* const box = (f32x4*)(smem + S::kStage);  // [row block, head_dim part][piece][4][lane]
            const int pair = wr + wd * WR;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                o[i] *= by;
                if (i % WK != wk) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const f32x4 x = {o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
                        box[((pair * kPieces + i) * 4 + r) * 64 + lane] = x;
                    }
                }
            }
            lds_barrier();
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                if (i % WK == wk) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const f32x4 x = box[((pair * kPieces + i) * 4 + r) * 64 + lane];
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[i][4 * r + e] += x[e];
                    }
                }
            }
            lds_barrier();  // every wave has emptied its boxes
        }
        const bool nan = *poison_flag != 0;
        const float by = nan ? forget(NAN) : whole ? 1.0f / sum : 1.0f;
        if (!whole && half == 0 && wk == 0 && wd == 0) {
            a.part_max[place + wr * 32 + lane] = top;
            a.part_sum[place + wr * 32 + lane] = sum;
        }
        // A lane has 16 values of its row; they go out by way of LDS, 8 lanes a row, in
        // whole lines of 128 bytes.
        f32x4* const turn = (f32x4*)(smem + S::kStage + wave * 4096);  // [row][8], chunks flipped by row
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            if (i % WK != wk) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const f32x4 x = {o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
                turn[(lane & 31) * 8 + ((2 * r + half) ^ (lane & 7))] = x * by;
            }
            __builtin_amdgcn_wave_barrier();
            const int d = 32 * (i * WD + wd) + 4 * (lane & 7);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = 8 * j + lane / 8;
                const f32x4 x = turn[row * 8 + ((lane & 7) ^ (row & 7))];
                if (d >= D) continue;
                if (whole) {
                    const Row to = row_of(row);
                    if (to.live)
                        *(u32x2*)(a.out + to.b * a.out_stride[0] + to.token * a.out_stride[1] + to.head * a.out_stride[2] + d) =
                            __builtin_bit_cast(u32x2, __builtin_convertvector(x, typename T::V4));
                } else {
                    *(f32x4*)(a.part_out + (place + wr * 32 + row) * D + d) = x;
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    };
    sum = halves_sum(sum);
    if (work.poison) *poison_flag = 1;
    const bool whole = kKind == kJoined && work.whole;
    const int64_t place = work.place;
    const bool more = work.advance();
    lds_barrier();  // every wave has done with the tiles
    if (more) work.stage_first();  // (into the first two; what follows works in the others)
    finish(forget(lane), whole, place);
    lds_barrier();  // they and the flag are free again
    if (tid == 0) *poison_flag = 0;
    return more;
}

template <class T, int D, int WR, Kind kKind>
__device__ __forceinline__ void run(const AttendArgs& a, const Totals& t, const Deal& deal, const Batch& batch, uint32_t w,
                                    char* smem, float (*wave_stats)[2][32], int* poison_flag, int* special_flag) {
    Work<D, kKind> work{a, t, batch, (uint32_t)(uintptr_t)(SV_LDS char*)smem, w, group_start(deal, w + 1),
                        {}, 0, false, group_start(deal, w), 0, 0, 0, false};
    bool more = work.advance();
    if (more) work.stage_first();
    while (more) more = segment<T, D, WR>(work, smem, wave_stats, poison_flag, special_flag);
}

// Workgroups go round the 8 XCDs.  Those of one XCD take adjoining runs of the tasks
// that share keys, to read them through one L2.
__device__ __forceinline__ uint32_t place_in_xcd(uint32_t block, uint32_t groups) {
    const uint32_t xcd = block % 8;
    return xcd * (groups / 8) + smaller(xcd, groups % 8) + block / 8;
}

// kPrefix and kRows: waves that split the rows of the prefix's tasks (0: there are
// none, a sequence's tasks begin with it) and of the sequences' own.
template <class T, int D, int kPrefix, int kRows>
__global__ void __launch_bounds__(kThreads, (D > 128 ? 1 : 2)) attend_kernel(AttendArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ uint32_t wave_sums[4][2];
    __shared__ float wave_stats[4][2][32];
    __shared__ int poison_flag, special_flag;
    const Split& split = a.split;
    int32_t* const words = (int32_t*)(smem + 2 * Shape<D>::kStage);
    const Batch batch{words, (uint32_t*)words + split.batch + 1, words + 2 * (split.batch + 1)};
    if (threadIdx.x == 0) poison_flag = special_flag = 0;
    const Totals t = sum_batch(split, batch, wave_sums);
    if (blockIdx.x == 0)  // for the kernel that joins the parts
        for (int b = threadIdx.x; b <= split.batch; b += kThreads) {
            a.cum_tokens[b] = batch.cum_tokens[b];
            a.cum_cost[b] = batch.cum_cost[b];
            if (b == 0) *a.totals = t;
        }
    if constexpr (kPrefix == 0) {
        if (blockIdx.x < t.own.groups)
            run<T, D, kRows, kJoined>(a, t, t.own, batch, place_in_xcd(blockIdx.x, t.own.groups), smem, wave_stats,
                                      &poison_flag, &special_flag);
    } else if (blockIdx.x < t.prefix.groups) {
        run<T, D, kPrefix, kShared>(a, t, t.prefix, batch, place_in_xcd(blockIdx.x, t.prefix.groups), smem, wave_stats,
                                    &poison_flag, &special_flag);
    } else if (blockIdx.x - t.prefix.groups < t.own.groups) {
        run<T, D, kRows, kOwn>(a, t, t.own, batch, blockIdx.x - t.prefix.groups, smem, wave_stats, &poison_flag,
                               &special_flag);
    }
}

// ---------------------------------------------------------------------------
// joining the parts
// ---------------------------------------------------------------------------

// One row of the output from its parts, by one wave: first the parts' statistics, a
// part a lane, and their outputs, D / 4 lanes a part, as many parts side by side
// as fit the wave and four such rounds under way at a time.  Bound by the latency of
// its loads, so those of the first round go out together with the statistics'.
template <int D>
struct Joiner {
    static constexpr int kLanes = D / 4, kTeams = 64 / kLanes, kAhead = 4;
    const AttendArgs& a;
    int lane, team, d;
    int count;        // of up to 64 parts at a time, those that there are, in the first lanes:
    int64_t at;       // their row places
    float most, part_sum;
    f32x4 x[kAhead];  // outputs of the first ones

    __device__ __forceinline__ explicit Joiner(const AttendArgs& args) : a(args) {
        lane = threadIdx.x & 63;
        team = min(lane / kLanes, kTeams - 1);
        d = (lane % kLanes) * 4;
    }
    __device__ __forceinline__ void load(int k0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (j > 0 && k0 + j * kTeams >= count) break;
            const int k = min(k0 + j * kTeams + team, count - 1);
            const int64_t from = ((int64_t)__shfl((int)(at >> 32), k) << 32) | (uint32_t)__shfl((int)(uint32_t)at, k);
            x[j] = *(const f32x4*)(a.part_out + from * D + d);
        }
    }
    // The parts base .. base + 63 of n; `place(k)` is the row place of part k, or -1.
    template <class Place>
    __device__ __forceinline__ void fetch(int base, int n, Place place) {
        at = (base + lane < n) ? place(base + lane) : -1;
        const uint64_t there = __ballot(at >= 0);
        count = __popcll(there);
        if (count == 0) return;
        if (count < 64) {
            const int slot = at >= 0 ? __popcll(there & ((1ull << lane) - 1)) : 63;  // (63 is no part's here)
            const int low = __builtin_amdgcn_ds_permute(slot * 4, (int)(uint32_t)at);
            const int high = __builtin_amdgcn_ds_permute(slot * 4, (int)(at >> 32));
            at = ((int64_t)high << 32) | (uint32_t)low;
        }
        most = lane < count ? a.part_max[at] : -INFINITY;
        part_sum = lane < count ? a.part_sum[at] : 0.0f;
        load(0);
    }
    // Joins what was fetched, and the parts behind it: maximum, sum and, in the first kLanes lanes, output.
    float top, sum;
    f32x4 out;
    template <class Place>
    __device__ __forceinline__ void join(int n, Place place) {
        top = -INFINITY;
        sum = 0.0f;
        out = f32x4(0.0f);
        for (int base = 0;;) {
            if (count > 0) {
                float now = fmaxf(top, most);
#pragma unroll
                for (int m = 1; m < 64; m <<= 1) now = fmaxf(now, __shfl_xor(now, m));
                const float ref = now == -INFINITY ? 0.0f : now;
                const float before = exp2_hw((top - ref) * a.scale_log2);
                const float by = lane < count ? exp2_hw((most - ref) * a.scale_log2) : 0.0f;
                sum = before * sum + by * part_sum;
                out *= before;
                top = now;
                for (int k0 = 0;;) {
#pragma unroll
                    for (int j = 0; j < kAhead; ++j) {
                        const int k = k0 + j * kTeams + team;
                        const float w = __shfl(by, min(k, count - 1));
                        if (k < count) out += w * x[j];
                    }
                    k0 += kAhead * kTeams;
                    if (k0 >= count) break;
                    load(k0);
                }
            }
            base += 64;
            if (base >= n) break;
            fetch(base, n, place);
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
        f32x4 all = out;
#pragma unroll
        for (int t = 1; t < kTeams; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) all[e] += __shfl(out[e], (lane + t * kLanes) & 63);
        out = all;
    }
    template <class T>
    __device__ __forceinline__ void write(uint16_t* to) const {
        if (lane >= kLanes) return;
        *(u32x2*)(to + d) = __builtin_bit_cast(u32x2, __builtin_convertvector(out * (1.0f / sum), typename T::V4));
    }
};

// One row from many parts, by a workgroup: its waves join every fourth part, and the
// first wave joins those.
template <class T, int D, class Place>
__device__ __forceinline__ void join_by_block(const AttendArgs& a, int n, Place place, uint16_t* to, float (*box)[D + 4]) {
    constexpr int kWaves = kThreads / 64;
    const int wave = uniform((int32_t)(threadIdx.x >> 6));
    auto every = [&](int k) { return place(kWaves * k + wave); };
    const int parts = (n - wave + kWaves - 1) / kWaves;
    Joiner<D> own(a);
    own.fetch(0, parts, every);
    own.join(parts, every);
    if (own.lane < Joiner<D>::kLanes) *(f32x4*)&box[wave][own.d] = own.out;
    if (own.lane == 0) {
        box[wave][D] = own.top;
        box[wave][D + 1] = own.sum;
    }
    __syncthreads();
    if (wave == 0) {
        float now = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) now = fmaxf(now, box[w][D]);
        const float ref = now == -INFINITY ? 0.0f : now;
        own.sum = 0.0f;
        own.out = f32x4(0.0f);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float by = exp2_hw((box[w][D] - ref) * a.scale_log2);
            own.sum += by * box[w][D + 1];
            own.out += by * *(const f32x4*)&box[w][own.d];
        }
        own.template write<T>(to);
    }
    __syncthreads();  // the box is free again
}

// Parts from which a row is joined by a workgroup, not by a wave, and behind a prefix
// rows up to which it is.  (One sequence of 30,000 keys, 8 to 64 rows at head_dim 256, 256
// parts: 27 to 42 us with the attention, and 55 to 78 by waves; behind 4,000 keys 20 to 23,
// and 25 to 29.  But 2,048 rows of about 32 parts: 43, and 40 by waves.)
constexpr int kBlockParts = 16;
constexpr int64_t kBlockRows = 1024;

// Rows of a batch with a shared prefix: every row has parts of both.  A wave a row.
// (14,304 rows of about 8 parts, 59 MB: 17 us; 352 rows of 9: 4.3.)
template <class T, int D, bool kBlock>
__global__ void __launch_bounds__(kThreads) attend_join_rows_kernel(AttendArgs a) {
    __shared__ __attribute__((aligned(16))) float box[kBlock ? kThreads / 64 : 1][D + 4];
    const Split& split = a.split;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t row = kBlock ? block : block * (kThreads / 64) + uniform((int32_t)(threadIdx.x >> 6));
    if (row >= (int64_t)split.batch * split.max_new * a.q_heads) return;
    const int head = (int)((uint32_t)row % (uint32_t)a.q_heads);
    const uint32_t flat = (uint32_t)row / (uint32_t)a.q_heads;
    const int token = (int)(flat % (uint32_t)split.max_new), b = (int)(flat / (uint32_t)split.max_new);
    const Sequence s = sequence(split, b);
    if (token >= s.count) return;
    const Totals& t = *a.totals;
    const int kv_head = head / split.group, g = head - kv_head * split.group;
    const Parts own =
        own_parts(split, t, s, a.cum_cost[b], a.cum_cost[b + 1] - a.cum_cost[b], b, token, kv_head, g);
    const int prefix = (int)(kChunkParts * t.chunks), r = (a.cum_tokens[b] + token) * split.group + g;
    auto place = [&](int k) {
        return k < prefix ? prefix_part(split, t, kv_head, r, (uint32_t)k) : own.first + (k - prefix) * own.step;
    };
    uint16_t* const to = a.out + b * a.out_stride[0] + token * a.out_stride[1] + head * a.out_stride[2];
    if constexpr (kBlock) {
        join_by_block<T, D>(a, prefix + own.n, place, to, box);
    } else {
        Joiner<D> parts(a);
        parts.fetch(0, prefix + own.n, place);
        parts.join(prefix + own.n, place);
        parts.template write<T>(to);
    }
}

// Tasks that the workgroups' borders cut: block x looks at the border before
// workgroup x + 1; the blocks of the borders that cut a task share its rows, of which
// block y has kJoinRows.  (Of 32,768 rows in two parts each, and of 65,408: 11.0
// and 16.4 us with 16 rows a block, 11.5 and 21.7 with 8, 15.6 and 15.9 with 32.)
constexpr int kJoinRows = 16;

// The same from two parts each, which is what there is where tasks are many: a team of
// D / 4 lanes a row, and all rows' loads under way at a time.  (Of 32,768 and of 65,408
// rows: 9.1 and 16.3 us, 4.1 TB/s.)
template <class T, int D, class RowOut>
__device__ __forceinline__ void join_two(const AttendArgs& a, int64_t first, int64_t second, int r0, RowOut row_out) {
    constexpr int kLanes = D / 4, kTeams = 64 / kLanes * (kThreads / 64), kEach = (kJoinRows + kTeams - 1) / kTeams;
    const int lane = threadIdx.x & 63, team = (int)(threadIdx.x >> 6) * (64 / kLanes) + lane / kLanes;
    const int d = (lane % kLanes) * 4;
    if (lane / kLanes >= 64 / kLanes) return;
    uint16_t* to[kEach];
    float most[kEach][2], sum[kEach][2];
    f32x4 x[kEach][2];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int r = i * kTeams + team;
        to[i] = r < kJoinRows ? row_out(r0 + r) : nullptr;
        if (to[i] == nullptr) continue;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int64_t at = (k == 0 ? first : second) + r0 + r;
            most[i][k] = a.part_max[at];
            sum[i][k] = a.part_sum[at];
            x[i][k] = *(const f32x4*)(a.part_out + at * D + d);
        }
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (to[i] == nullptr) continue;
        const float top = fmaxf(most[i][0], most[i][1]), ref = top == -INFINITY ? 0.0f : top;
        const float w0 = exp2_hw((most[i][0] - ref) * a.scale_log2), w1 = exp2_hw((most[i][1] - ref) * a.scale_log2);
        f32x4 all = w0 * x[i][0];
        all += w1 * x[i][1];
        all *= 1.0f / (w0 * sum[i][0] + w1 * sum[i][1]);
        *(u32x2*)(to[i] + d) = __builtin_bit_cast(u32x2, __builtin_convertvector(all, typename T::V4));
    }
}
template <class T, int D>
__global__ void __launch_bounds__(kThreads) attend_join_tasks_kernel(AttendArgs a) {
    __shared__ __attribute__((aligned(16))) float box[kThreads / 64][D + 4];
    const Split& split = a.split;
    const Totals& t = *a.totals;
    const uint32_t w = blockIdx.x + 1;
    if (w >= t.own.groups) return;
    const Segment g = own_task_at(split, a.cum_cost, group_start(t.own, w), [&](int32_t b) { return sequence(split, b); });
    uint32_t w0, w1;
    if (!cuts_task(t, g, w, w0, w1)) return;
    const int borders = (int)(w1 - w0), n = 1 + borders, mine = (int)(w - w0) - 1;
    const int end = (int)(blockIdx.y + 1) * kJoinRows;
    int r = (int)blockIdx.y * kJoinRows;  // (`place` is that of row r)
    auto row_out = [&](int of) -> uint16_t* {
        const int row = g.row0 + of, token = row / split.group;
        const int head = g.kv_head * split.group + (row - token * split.group);
        return token < g.count ? a.out + g.b * a.out_stride[0] + token * a.out_stride[1] + head * a.out_stride[2] : nullptr;
    };
    if (n == 2) {
        join_two<T, D>(a, first_cut_part(split, w0, 0).first, later_cut_parts(split, w0, w1, 0).first, (int)blockIdx.y * kJoinRows,
                       row_out);
        return;
    }
    auto place = [&](int k) {
        const Parts first = first_cut_part(split, w0, r), later = later_cut_parts(split, w0, w1, r);
        return k == 0 ? first.first : later.first + (k - 1) * later.step;
    };
    if (n >= kBlockParts) {
#pragma unroll 1
        for (r += mine; r < end; r += borders) {
            uint16_t* const to = row_out(r);
            if (to == nullptr) return;
            join_by_block<T, D>(a, n, place, to, box);
        }
        return;
    }
#pragma unroll 1
    for (r += mine * (kThreads / 64) + uniform((int32_t)(threadIdx.x >> 6)); r < end; r += borders * (kThreads / 64)) {
        uint16_t* const to = row_out(r);
        if (to == nullptr) return;
        Joiner<D> parts(a);
        parts.fetch(0, n, place);
        parts.join(n, place);
        parts.template write<T>(to);
    }
}

// (at head_dim 256 a task has at most 64 rows, see task_rows)
template <int D>
constexpr int kMaxTaskRows = D > 128 ? 64 : 128;

template <class T, int D>
sv_status_t launch(const AttendArgs& a, hipStream_t stream) {
    const size_t lds = 2 * Shape<D>::kStage + 3 * sizeof(int32_t) * ((size_t)a.split.batch + 1);
    const uint32_t groups = (uint32_t)a.split.plan.groups;
    auto go = [&](auto prefix, auto own) {
        hipLaunchKernelGGL((attend_kernel<T, D, decltype(prefix)::value, decltype(own)::value>), dim3(groups),
                           dim3(kThreads), lds, stream, a);
    };
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, 1> k1{};
    constexpr std::integral_constant<int, 2> k2{};
    constexpr std::integral_constant<int, kMaxTaskRows<D> / 32> k4{};
    const int own = a.split.plan.own_rows / 32, prefix = a.split.plan.joined ? 0 : a.split.plan.prefix_rows / 32;
    if (prefix == 0)
        own == 1 ? go(k0, k1) : own == 2 ? go(k0, k2) : go(k0, k4);
    else if (prefix == 1)
        go(k1, k1);
    else if (prefix == 2)
        own == 1 ? go(k2, k1) : go(k2, k2);
    else
        own == 1 ? go(k4, k1) : own == 2 ? go(k4, k2) : go(k4, k4);
    if (a.split.plan.joined) {
        if (groups > 1)
            hipLaunchKernelGGL((attend_join_tasks_kernel<T, D>), dim3(groups - 1, a.split.plan.own_rows / kJoinRows),
                               dim3(kThreads), 0, stream, a);
    } else {
        constexpr int kRowsBlock = kThreads / 64;
        const int64_t rows = (int64_t)a.split.batch * a.split.max_new * a.q_heads;
        const bool by_block = rows <= kBlockRows && (int64_t)groups >= kBlockParts * pooled_tasks(a.split);
        // (one dimension of a launch has fewer than 2^32 threads: 2^26 rows, of the 2^31 that a call may have)
        const int64_t blocks = by_block ? rows : (rows + kRowsBlock - 1) / kRowsBlock, most = 1 << 20;
        const dim3 grid((uint32_t)(blocks < most ? blocks : most), (uint32_t)((blocks + most - 1) / most));
        if (by_block)
            hipLaunchKernelGGL((attend_join_rows_kernel<T, D, true>), grid, dim3(kThreads), 0, stream, a);
        else
            hipLaunchKernelGGL((attend_join_rows_kernel<T, D, false>), grid, dim3(kThreads), 0, stream, a);
    }
    return hipGetLastError() == hipSuccess ? SV_OK : SV_ERR_HIP;
}

template <class T>
sv_status_t launch_dim(const AttendArgs& a, int32_t head_dim, hipStream_t stream) {
    switch (head_dim) {
        case 64: return launch<T, 64>(a, stream);
        case 80: return launch<T, 80>(a, stream);
        case 96: return launch<T, 96>(a, stream);
        case 128: return launch<T, 128>(a, stream);
        default: return launch<T, 256>(a, stream);
    }
}

}  // namespace
}  // namespace sv
