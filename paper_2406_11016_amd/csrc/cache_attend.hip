// Attention of a step's new tokens to the paged cache, behind a prefix that the
// batch shares, for gfx950 (MI355X): kernels and C ABI of spec_cache_attend.
//
// Work is cut into tasks of up to kRows query rows of one key/value head (a row
// is a token and one of its heads) against a run of keys, and a task into units
// of kKeys keys.  The rows of the whole batch share the prefix's tasks; each
// sequence has tasks of its own for its own keys.  The units of all tasks in
// order are dealt to the grid's workgroups in equal runs, so lengths need not be
// known on the host and few long sequences fill the chip as well as many short
// ones; what a workgroup computes of a task is a part (running maximum, sum and
// unnormalised output of every row), and a second kernel joins a row's parts.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cache_split.hpp"
#include "spec_cache.h"

namespace sv {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

#define SV_LDS __attribute__((address_space(3)))

struct AttF16 {
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
    uint32_t* cum_units;  // [batch + 1] units before each sequence's own
    float* part_out;      // parts: rows x head_dim, fp32
    float* part_max;      // maximum (scores in log2 units)
    float* part_sum;
};

// A value that is the same in every lane, in a scalar register.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

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

// Sums over the batch before each sequence: tokens and units, [batch + 1] each.
// Every workgroup makes them for itself (a few loads and one scan).
__device__ __forceinline__ Totals sum_batch(const Split& a, int32_t* cum_tokens, uint32_t* cum_units,
                                            uint32_t (*wave_sums)[2]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (a.batch + kThreads - 1) / kThreads;
    const int b0 = min(tid * each, a.batch), b1 = min(b0 + each, a.batch);
    uint32_t tokens = 0, units = 0;
    for (int b = b0; b < b1; ++b) {
        const Sequence s = sequence(a, b);
        tokens += s.count;
        units += sequence_units(a, s) * (uint32_t)a.kv_heads;
        cum_tokens[b + 1] = tokens;
        cum_units[b + 1] = units;
    }
    uint32_t t = tokens, u = units;
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
    uint32_t bt = t - tokens, bu = u - units;
    for (int w = 0; w < wave; ++w) {
        bt += wave_sums[w][0];
        bu += wave_sums[w][1];
    }
    for (int b = b0; b < b1; ++b) {
        cum_tokens[b + 1] += bt;
        cum_units[b + 1] += bu;
    }
    if (tid == 0) {
        cum_tokens[0] = 0;
        cum_units[0] = 0;
    }
    __syncthreads();
    return totals(a, uniform(cum_tokens[a.batch]), uniform(cum_units[a.batch]));
}

// A sequence's own task that holds its unit `at` of one key/value head: its row
// tile, and the unit at which it starts.  64 tiles at a time, one a lane.
__device__ __forceinline__ int32_t find_tile(const Split& a, const Sequence& s, uint32_t at, uint32_t& start) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int32_t base = 0; base < a.plan.own_tiles; base += 64) {
        const uint32_t own = (base + lane < a.plan.own_tiles) ? tile_units(a, s, base + lane) : 0u;
        uint32_t end = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(end, d);
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
    start = before;
    return a.plan.own_tiles - 1;  // (not reached: `at` is below the sum of all tiles)
}

// The task of unit u, in scalar registers.
__device__ __forceinline__ Segment task_at(const Split& a, const Totals& t, const uint32_t* cum_units, uint32_t u) {
    Segment g = locate(a, t, cum_units, u, [&](const Sequence& s, uint32_t at, uint32_t& start) {
        return find_tile(a, s, at, start);
    });
    g.task = uniform(g.task);
    g.task_start = uniform(g.task_start);
    g.units = uniform(g.units);
    g.prefix_units = uniform(g.prefix_units);
    g.kv_head = uniform(g.kv_head);
    g.b = uniform(g.b);
    g.row0 = uniform(g.row0);
    g.count = uniform(g.count);
    g.length = uniform(g.length);
    g.bad = uniform((int32_t)g.bad) != 0;
    return g;
}

// ---------------------------------------------------------------------------
// one segment
// ---------------------------------------------------------------------------

template <int D>
struct Shape {
    static constexpr int kPitch = D <= 64 ? 64 : D <= 128 ? 128 : 256;  // elements of a row in LDS
    static constexpr int kChunks = kPitch / 8;                         // of 16 bytes
    static constexpr int kTile = kKeys * kPitch * 2;                   // bytes of a tile of K or of V
    static constexpr int kSteps = D / 16;                              // products over head_dim
    static constexpr int kOuts = (D + 31) / 32;                        // 32-wide pieces of the output
    static constexpr int kRowsLoad = 1024 / (kPitch * 2);              // rows of one wave-wide load
    static constexpr int kLoads = 32 / kRowsLoad;                      // loads of a wave for its 32 rows
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
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
// Own LDS reads done, then the workgroup's barrier.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// Whether this thread's share of a tile holds infinities or NaN; `clear` makes them zeros.
template <class T, int D>
__device__ __forceinline__ int special_chunks(char* tile, bool clear) {
    using S = Shape<D>;
    uint32_t found = 0;
#pragma unroll 1
    for (int at = threadIdx.x * 16; at < S::kTile; at += kThreads * 16) {
        // (a chunk behind head_dim holds what was there before: nothing reads it)
        if (D != S::kPitch && (((at / 16) % S::kChunks) ^ swizzle<D>(at / (S::kPitch * 2))) * 8 >= D) continue;
        u32x4 x = *(u32x4*)(tile + at);
        uint32_t here = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool low = T::special(x[i] & 0xffffu), high = T::special(x[i] >> 16);
            x[i] &= (low ? 0u : 0xffffu) | (high ? 0u : 0xffff0000u);
            here |= (uint32_t)low | (uint32_t)high;
        }
        if (clear && here) *(u32x4*)(tile + at) = x;
        found |= here;
    }
    return (int)found;
}

// The part of a task's rows over a run of its units.  Four waves: WR of them
// split the rows (32 each), 4 / WR the 32-key blocks of a unit.
//
// The products are taken transposed.  S^T = K Q^T leaves a query row's scores in
// the registers of two lanes (l and l + 32), so the maximum and the sum over the
// keys need one exchange between lanes, and the running maximum, the sum and the
// rescaling of the output are one value a lane.  P^T then is the B operand of
// O^T = V^T P^T as it stands (after rounding to the storage type), with V^T from
// LDS by transposing reads in the same order of keys.
template <class T, int D, int WR>
__device__ void segment(const AttendArgs& a, const Segment& g, const int32_t* cum_tokens, char* smem,
                        float (*wave_stats)[2][32], int* poison_flag, bool whole, int64_t place) {
    using S = Shape<D>;
    using V8 = typename T::V8;
    constexpr int WK = 4 / WR, NS = 4 / WK;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = uniform(tid >> 6);
    const int wr = wave % WR, wk = wave / WR;
    const uint32_t lds_k = (uint32_t)(uintptr_t)(SV_LDS char*)smem, lds_v = lds_k + S::kTile;

    // the row of this lane
    const int row = g.row0 + wr * 32 + (lane & 31);
    int b = g.b, token = 0, head = 0;
    bool live;
    {
        const int flat = row / a.split.group;
        head = g.kv_head * a.split.group + (row - flat * a.split.group);
        if (g.b < 0) {
            live = flat < cum_tokens[a.split.batch];
            b = live ? find(cum_tokens, a.split.batch, flat) : 0;
            token = live ? flat - cum_tokens[b] : 0;
        } else {
            live = flat < g.count;
            token = flat;
        }
    }
    V8 q[S::kSteps];
    {
        const uint16_t* const from = a.q + b * a.q_stride[0] + token * a.q_stride[1] + head * a.q_stride[2] + half * 8;
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s) {
            u32x4 x = {0, 0, 0, 0};
            if (live) x = *(const u32x4*)(from + 16 * s);
            q[s] = __builtin_bit_cast(V8, x);
        }
    }
    const int own_limit = g.length + token + 1;                    // keys of its own that this row sees
    const int own_first = own_common(a.split, g), own_last = own_end(a.split, g) - 1;

    bool poison = g.bad;
    f32x16 o[S::kOuts];
#pragma unroll
    for (int i = 0; i < S::kOuts; ++i) o[i] = f32x16(0.0f);
    float top = -INFINITY, sum = 0.0f;  // top: scores as they come from the product

    // Loads of one unit: a wave stages 32 keys, in two runs of 16 that each lie in one page.
    const uint16_t *run_k[2], *run_v[2];
    int run_row[2];
    auto turn = [&](uint32_t u) {  // to unit u: its pages
        const bool pre = u < g.prefix_units;
        const int base = (int)(pre ? u : u - g.prefix_units) * kKeys;
        const int last = pre ? a.prefix_len - 1 : own_last;
        const int32_t* const table = pre ? a.prefix_table : a.block_table + (int64_t)max(g.b, 0) * a.split.max_pages;
        const int mask = (1 << a.split.page_shift) - 1;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int first = run_start(base, wave * 2 + r, last);
            int page = 0;
            if (pre || !g.bad) page = table[first >> a.split.page_shift];
            if ((uint32_t)page >= (uint32_t)a.num_pages) {
                page = 0;
                poison = true;
            }
            const int64_t at = (int64_t)page * a.page_stride + (int64_t)((g.kv_head << a.split.page_shift)) * D;
            run_k[r] = a.k_cache + at + (int64_t)(first & mask) * D;
            run_v[r] = a.v_cache + at + (int64_t)(first & mask) * D;
            run_row[r] = last - first;  // rows of the run behind this one repeat it
        }
    };
    const int load_row = lane / S::kChunks, load_chunk = lane % S::kChunks;
    auto stage = [&](const uint16_t* const (&run)[2], uint32_t lds) {
#pragma unroll
        for (int j = 0; j < S::kLoads; ++j) {
            constexpr int kRun = S::kLoads / 2;
            const int r = j / kRun;
            const int in_run = (j % kRun) * S::kRowsLoad + load_row;
            const int chunk = load_chunk ^ swizzle<D>(r * 16 + in_run);
            const uint32_t offset = (uint32_t)(min(in_run, run_row[r]) * D + chunk * 8) * 2;
            if (D == S::kPitch || chunk * 8 < D) load_to_lds(lds + wave * (32 * S::kPitch * 2) + j * 1024, run[r], offset);
        }
    };

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
        v_at[j] = S::kTile + block0 + r * (S::kPitch * 2) + ((chunk ^ swizzle<D>(r)) * 16) + (i & 1) * 8;
    }
    // 8 values of V of the 16 keys from `key` on, in the order of the weights' registers
    auto read_v = [&](int key, int out) {
        i16x4 v[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
            v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (SV_LDS i16x4*)(SV_LDS char*)(smem + (v_at[j] ^ (out * 64)) + key * (S::kPitch * 2)));
        return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
    };

    turn(g.first);
    stage(run_k, lds_k);
    stage(run_v, lds_v);
    for (uint32_t u = g.first; u < g.end; ++u) {
        const bool pre = u < g.prefix_units;
        const int base = (int)(pre ? u : u - g.prefix_units) * kKeys;
        const int limit = pre ? a.prefix_len : own_limit;
        const bool partial = base + kKeys > (pre ? a.prefix_len : own_first);
        const bool more = u + 1 < g.end;

        wait_loads<S::kLoads>();
        lds_barrier();  // this unit's K is there
        f32x16 p[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) p[s] = f32x16(0.0f);
#pragma unroll
        for (int c = 0; c < S::kSteps; ++c) {
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const V8 k = *(const V8*)(smem + (k_at ^ (c * 32)) + s * (32 * S::kPitch * 2));
                p[s] = T::mma(k, q[c], p[s]);
            }
        }
        lds_barrier();  // every wave has read it
        if (more) {
            turn(u + 1);
            stage(run_k, lds_k);
        }

        // scores to weights; key of register i: 8 (i / 4) + 4 half + i % 4
        if (partial) {
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = base + (wk * NS + s) * 32 + 8 * (i / 4) + 4 * half + (i % 4);
                    p[s][i] = key < limit ? p[s][i] : -INFINITY;
                }
        }
        float most = -INFINITY;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, p[s][i]);
        most = halves_max(most);
        // Weights are relative to a maximum of earlier units as long as the new
        // one is within 2^8 of it: nothing is rescaled for small rises.
        if (__any(most > top + a.lazy)) {
            const float now = fmaxf(top, most);
            const float by = (now == -INFINITY) ? 1.0f : exp2_hw((top - now) * a.scale_log2);
            sum *= by;
#pragma unroll
            for (int i = 0; i < S::kOuts; ++i) o[i] *= by;
            top = now;
        }
        const float shift = (top == -INFINITY) ? 0.0f : -top * a.scale_log2;
        float add = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[s][i] = exp2_hw(fmaf(p[s][i], a.scale_log2, shift));
                add += p[s][i];
            }
        sum += add;

        if (more)
            wait_loads<S::kLoads>();
        else
            wait_loads<0>();
        lds_barrier();  // this unit's V is there
        if (partial && __syncthreads_or(special_chunks<T, D>(smem + S::kTile, false))) {
            // A masked key's weight is 0, but 0 times an infinity or NaN is not.
            // Rows take such values from the keys that they see, here; then they
            // are zeros for the product.
            const int key0 = wk * NS * 32;
#pragma unroll 1
            for (int k = 0; k < NS * 32; ++k) {
                const bool sees = base + key0 + k < limit;
                const int sw = swizzle<D>(k);
#pragma unroll
                for (int i = 0; i < S::kOuts; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const u32x2 x = *(const u32x2*)(smem + S::kTile + (key0 + k) * (S::kPitch * 2) +
                                                        ((4 * i + r) ^ sw) * 16 + half * 8);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t bits = (x[e / 2] >> (16 * (e % 2))) & 0xffffu;
                            if (sees && T::special(bits)) o[i][4 * r + e] += T::value(bits);
                        }
                    }
            }
            __syncthreads();
            special_chunks<T, D>(smem + S::kTile, true);
            __syncthreads();
        }
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                f32x8 w;
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = p[s][8 * kb + i];
                const V8 w8 = __builtin_convertvector(w, V8);
#pragma unroll
                for (int i = 0; i < S::kOuts; ++i)
                    o[i] = T::mma(__builtin_bit_cast(V8, read_v(s * 32 + kb * 16, i)), w8, o[i]);
            }
        lds_barrier();  // every wave has read V
        if (more) stage(run_v, lds_v);
    }

    // ---- join the waves that split the keys, then write
    sum = halves_sum(sum);
    top *= a.scale_log2;
    if (poison) *poison_flag = 1;
    if constexpr (WK > 1) {
        float(*const mine)[32] = wave_stats[wave];
        if (half == 0) {
            mine[0][lane] = top;
            mine[1][lane] = sum;
        }
        __syncthreads();
        float now = -INFINITY;
#pragma unroll
        for (int k = 0; k < WK; ++k) now = fmaxf(now, wave_stats[wr + k * WR][0][lane & 31]);
        const float ref = (now == -INFINITY) ? 0.0f : now;
        float all = 0.0f;
#pragma unroll
        for (int k = 0; k < WK; ++k)
            all += wave_stats[wr + k * WR][1][lane & 31] * exp2_hw(wave_stats[wr + k * WR][0][lane & 31] - ref);
        const float by = exp2_hw(top - ref);
        // piece i of the output is summed by the wave wk = i % WK
        f32x4* const box = (f32x4*)smem;  // [from][row block][piece][4][lane]
#pragma unroll
        for (int i = 0; i < S::kOuts; ++i) {
            o[i] *= by;
            if (i % WK != wk) {
                const int from = wk < i % WK ? wk : wk - 1;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const f32x4 x = {o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
                    box[(((from * WR + wr) * S::kOuts + i) * 4 + r) * 64 + lane] = x;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < S::kOuts; ++i) {
            if (i % WK == wk) {
#pragma unroll
                for (int from = 0; from < WK - 1; ++from)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const f32x4 x = box[(((from * WR + wr) * S::kOuts + i) * 4 + r) * 64 + lane];
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[i][4 * r + e] += x[e];
                    }
            }
        }
        top = now;
        sum = all;
    } else {
        __syncthreads();
    }
    const bool nan = *poison_flag != 0;
    if (whole) {
        const float by = nan ? NAN : 1.0f / sum;
        uint16_t* const to = a.out + b * a.out_stride[0] + token * a.out_stride[1] + head * a.out_stride[2];
#pragma unroll
        for (int i = 0; i < S::kOuts; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = 32 * i + 8 * r + 4 * half;
                if (live && i % WK == wk && d < D) {
                    f32x4 x = {o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
                    x *= by;
                    *(u32x2*)(to + d) = __builtin_bit_cast(u32x2, __builtin_convertvector(x, typename T::V4));
                }
            }
    } else {
        const int64_t at = place + wr * 32 + (lane & 31);
        if (half == 0 && wk == 0) {
            a.part_max[at] = top;
            a.part_sum[at] = sum;
        }
        float* const to = a.part_out + at * D;
#pragma unroll
        for (int i = 0; i < S::kOuts; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = 32 * i + 8 * r + 4 * half;
                if (i % WK == wk && d < D) {
                    f32x4 x = {o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
                    if (nan) x = f32x4(NAN);
                    *(f32x4*)(to + d) = x;
                }
            }
    }
    __syncthreads();  // LDS and the flag are free again
    if (tid == 0) *poison_flag = 0;
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads, (D > 128 ? 1 : 2)) attend_kernel(AttendArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ uint32_t wave_sums[4][2];
    __shared__ float wave_stats[4][2][32];
    __shared__ int poison_flag;
    const Split& split = a.split;
    int32_t* const cum_tokens = (int32_t*)(smem + 2 * Shape<D>::kTile);
    uint32_t* const cum_units = (uint32_t*)(cum_tokens + split.batch + 1);
    if (threadIdx.x == 0) poison_flag = 0;
    const Totals t = sum_batch(split, cum_tokens, cum_units, wave_sums);
    if (blockIdx.x == 0)  // for the kernel that joins the parts
        for (int b = threadIdx.x; b <= split.batch; b += kThreads) {
            a.cum_tokens[b] = cum_tokens[b];
            a.cum_units[b] = cum_units[b];
        }
    if (blockIdx.x >= t.groups) return;
    // Workgroups go round the 8 XCDs; those of one XCD take adjoining runs, so
    // that the tasks that share keys read them through one L2.
    const uint32_t w = (t.groups % 8 == 0) ? (blockIdx.x % 8) * (t.groups / 8) + blockIdx.x / 8 : blockIdx.x;
    const uint32_t end = group_start(t, w + 1);
    for (uint32_t u = group_start(t, w); u < end;) {
        Segment g = task_at(split, t, cum_units, u);
        g.first = u - g.task_start;
        g.end = smaller(g.units, end - g.task_start);
        const bool whole = whole_task(split, g);
        const int64_t place = part_place(split, g, w);
        const int waves = (g.b < 0 ? split.plan.prefix_rows : split.plan.own_rows) / 32;
        if (waves == 1)
            segment<T, D, 1>(a, g, cum_tokens, smem, wave_stats, &poison_flag, whole, place);
        else if (waves == 2 || D > 128)
            segment<T, D, 2>(a, g, cum_tokens, smem, wave_stats, &poison_flag, whole, place);
        else if constexpr (D <= 128)
            segment<T, D, 4>(a, g, cum_tokens, smem, wave_stats, &poison_flag, whole, place);
        u = g.task_start + g.end;
    }
}

// ---------------------------------------------------------------------------
// joining the parts
// ---------------------------------------------------------------------------

template <class T, int D>
__device__ __forceinline__ void join(const AttendArgs& a, const Parts (&parts)[2], int d, uint16_t* to) {
    float top = -INFINITY;
    for (int l = 0; l < 2; ++l)
        for (int k = 0; k < parts[l].n; ++k) top = fmaxf(top, a.part_max[parts[l].first + k * parts[l].step]);
    f32x4 out = f32x4(0.0f);
    float sum = 0.0f;
    for (int l = 0; l < 2; ++l)
        for (int k = 0; k < parts[l].n; ++k) {
            const int64_t at = parts[l].first + k * parts[l].step;
            const float by = exp2_hw(a.part_max[at] - top);
            sum += by * a.part_sum[at];
            out += by * *(const f32x4*)(a.part_out + at * D + d);
        }
    out *= 1.0f / sum;
    *(u32x2*)(to + d) = __builtin_bit_cast(u32x2, __builtin_convertvector(out, typename T::V4));
}

// Rows of a batch with a shared prefix: every row has parts of both.
template <class T, int D>
__global__ void __launch_bounds__(kThreads) attend_join_rows_kernel(AttendArgs a) {
    constexpr int kLanes = D / 4, kRowsBlock = kThreads / kLanes;
    const Split& split = a.split;
    const int lane = threadIdx.x % kLanes;
    const int64_t row = (int64_t)blockIdx.x * kRowsBlock + threadIdx.x / kLanes;
    if (threadIdx.x >= kRowsBlock * kLanes || row >= (int64_t)split.batch * split.max_new * a.q_heads) return;
    const int head = (int)(row % a.q_heads);
    const int64_t flat = row / a.q_heads;
    const int token = (int)(flat % split.max_new), b = (int)(flat / split.max_new);
    const Sequence s = sequence(split, b);
    if (token >= s.count) return;
    const Totals t = totals(split, a.cum_tokens[split.batch], a.cum_units[split.batch]);
    const int kv_head = head / split.group, g = head - kv_head * split.group;
    const Parts parts[2] = {prefix_parts(split, t, a.cum_tokens[b], token, kv_head, g),
                            own_parts(split, t, s, a.cum_units[b], a.cum_units[b + 1] - a.cum_units[b], b, token,
                                      kv_head, g)};
    join<T, D>(a, parts, lane * 4, a.out + b * a.out_stride[0] + token * a.out_stride[1] + head * a.out_stride[2]);
}

// Tasks that the workgroups' borders cut: block x looks at the border before
// workgroup x + 1, and joins the task that it cuts if it is the first to.
template <class T, int D>
__global__ void __launch_bounds__(kThreads) attend_join_tasks_kernel(AttendArgs a) {
    const Split& split = a.split;
    const Totals t = totals(split, uniform(a.cum_tokens[split.batch]), uniform(a.cum_units[split.batch]));
    const uint32_t w = blockIdx.x + 1;
    if (w >= t.groups) return;
    const uint32_t u = group_start(t, w);
    const Segment g = task_at(split, t, a.cum_units, u);
    const uint32_t w0 = group_of(t, g.task_start), w1 = group_of(t, g.task_start + g.units - 1);
    if (u == g.task_start || w != w0 + 1) return;
    constexpr int kLanes = D / 4;
    for (int at = threadIdx.x; at < split.plan.own_rows * kLanes; at += kThreads) {
        const int r = at / kLanes, d = (at - r * kLanes) * 4, row = g.row0 + r;
        const int token = row / split.group, head = g.kv_head * split.group + (row - token * split.group);
        if (token >= g.count) continue;
        const Parts parts[2] = {first_cut_part(split, w0, r), later_cut_parts(split, w0, w1, r)};
        join<T, D>(a, parts, d, a.out + g.b * a.out_stride[0] + token * a.out_stride[1] + head * a.out_stride[2]);
    }
}

template <class T, int D>
sv_status_t launch(const AttendArgs& a, hipStream_t stream) {
    const size_t lds = 2 * Shape<D>::kTile + 2 * sizeof(int32_t) * ((size_t)a.split.batch + 1);
    const uint32_t groups = (uint32_t)a.split.plan.groups;
    hipLaunchKernelGGL((attend_kernel<T, D>), dim3(groups), dim3(kThreads), lds, stream, a);
    if (a.split.plan.joined) {
        if (groups > 1)
            hipLaunchKernelGGL((attend_join_tasks_kernel<T, D>), dim3(groups - 1), dim3(kThreads), 0, stream, a);
    } else {
        constexpr int kRowsBlock = kThreads / (D / 4);
        const int64_t rows = (int64_t)a.split.batch * a.split.max_new * a.q_heads;
        hipLaunchKernelGGL((attend_join_rows_kernel<T, D>), dim3((uint32_t)((rows + kRowsBlock - 1) / kRowsBlock)),
                           dim3(kThreads), 0, stream, a);
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

extern "C" {

size_t spec_cache_attend_workspace_bytes(int32_t batch, int32_t max_new, int32_t q_heads, int32_t kv_heads,
                                         int32_t head_dim) {
    return sv::attend_workspace_bytes(batch, max_new, q_heads, kv_heads, head_dim);
}

sv_status_t spec_cache_attend(const sv_cache_attend_desc_t* desc, hipStream_t stream) {
    if (desc == nullptr) return SV_ERR_NULL;
    const sv_cache_attend_desc_t& d = *desc;
    const sv_status_t st = sv::check_attend(d);
    if (st != SV_OK) return st;
    sv::AttendArgs a{};
    const sv::AttendPlan plan =
        sv::attend_plan(d.batch, d.max_new, d.q_heads, d.kv_heads, d.head_dim, d.prefix_len > 0);
    a.split = sv::make_split(d, plan);
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
    a.cum_units = reinterpret_cast<uint32_t*>(ws + plan.cum_bytes);
    a.part_max = reinterpret_cast<float*>(ws + 2 * plan.cum_bytes);
    a.part_sum = a.part_max + plan.rows;
    a.part_out = a.part_sum + plan.rows;
    return d.dtype == SV_F16 ? sv::launch_dim<sv::AttF16>(a, d.head_dim, stream)
                             : sv::launch_dim<sv::AttBF16>(a, d.head_dim, stream);
}

}  // extern "C"
