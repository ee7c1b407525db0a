// Attention over a cache in 4 bits for few rows (up to 48 of a key/value head), where
// the cache's bytes are what bounds it, for gfx950 (MI355X).
// (Included by cache4_attend.hpp; the split of the work is cache_attend.hpp's.)
//
// What it reaches, at head_dim 128: 128 sequences of 4 rows behind 4,096 to 8,192 keys,
// 854 MB, 167 us (5.1 TB/s); 64 of 36 rows behind 2,048 to 4,096, 222 MB, 70 us.  (Of 77, in a process's first calls, a
// workgroup's units take 43 (5.1 TB/s) and starts and ends the others: the batch's sums 2, the
// first task, its page, Q and its first loads 6, a task's end and the next one's start 7.)
// With the keys in the L2, 16, 32 and 48 rows run at 530, 745 and 890 to 960 TFLOP/s.
#pragma once

#include "cache_attend.hpp"

namespace sv {
namespace {

typedef int i32x2 __attribute__((ext_vector_type(2)));

// Products of 16 x 16 with 32 between them.
__device__ __forceinline__ f32x4 mma16(AttF16::V8 a, AttF16::V8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(AttBF16::V8 a, AttBF16::V8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// Two values of byte kByte of the codes.
template <int kByte>
__device__ __forceinline__ uint32_t wide_pair(AttF16, uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, kByte));
}
template <int kByte>
__device__ __forceinline__ uint32_t wide_pair(AttBF16, uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte));
}
// Scales' bytes up to which all values are finite.
__device__ __forceinline__ uint32_t last_finite(AttF16) { return 127 + 13; }
__device__ __forceinline__ uint32_t last_finite(AttBF16) { return 127 + 125; }

// max or sum over the four lanes that share a row (l, l + 16, l + 32, l + 48), in each
__device__ __forceinline__ float quarters_max(float x) {
    x = halves_max(x);
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quarters_sum(float x) {
    x = halves_sum(x);
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int D>
struct Direct {
    static constexpr int kRow = D / 2, kBlocks = packed_blocks(D);
    // Products over head_dim have 32 of it, 8 in each quarter of the wave.  A quarter takes what a wide load of a row
    // brings: 32 values at D >= 128, of a block each, 16 below; what is left of D = 80 and 96 comes in a load of its own.
    static constexpr int kWide = D >= 128 ? 32 : 16, kWides = D / (4 * kWide), kRest = D - 4 * kWide * kWides;
    static constexpr int kSteps = kWides * kWide / 8 + (kRest > 0 ? 1 : 0);
    static constexpr int kScales = kWides + (kRest > 0 ? 1 : 0);
    static constexpr int kPieces = kBlocks;                    // blocks of 32 of the output, each with V's scales
    static constexpr int kTile = kKeys * kRow;                 // V of a unit, as it comes from memory
    static constexpr int kVScales = kPieces * kKeys * 4;       // and its scales, in fp32, [piece][key]
    static constexpr int kWave = 2 * kTile + kVScales;         // LDS of a wave
    // Q of several row tiles lies in LDS, for all waves, in the order in which they read it (there are no registers for it)
    static constexpr bool q_in_lds(int tiles) { return tiles > 1; }
    static constexpr int lds(int tiles) { return 4 * kWave + (q_in_lds(tiles) ? tiles * kSteps * 1024 : 0); }
    // When the waves' outputs are joined, 16 rows of some pieces at a time go through each wave's LDS but for its first
    // buffer, to which the next task's first values are on their way.
    static constexpr int kBoxPieces = D >= 128 ? D / 64 : 1, kBoxes = kPieces / kBoxPieces;
    static constexpr int kPitch = 32 * kBoxPieces + 4;         // floats of a row there
    static_assert(16 * kPitch * 4 <= kWave - kTile && kBoxes * kBoxPieces == kPieces, "they fit");
    // first value of product s for a quarter, and (a lane's number of) its scale
    static constexpr __device__ int value(int s, int quarter) {
        const int in = kWide / 8, j = s / in;
        return j < kWides ? 4 * kWide * j + kWide * quarter + 8 * (s % in) : 4 * kWide * kWides + 8 * quarter;
    }
    static constexpr __device__ int scale(int s) { return s / (kWide / 8); }
    static constexpr __device__ bool there(int s, int quarter) { return value(s, quarter) < D; }
    // V's rows lie in LDS with their 16-byte chunks permuted, so that the transposing reads, 16 bytes of 32 keys at a time,
    // go over all banks (rows of 40 and 48 bytes do by themselves)
    static constexpr __device__ int swizzle(int key) {
        return D == 64 ? (key >> 3) & 1 : D == 128 ? (key >> 2) & 3 : D == 256 ? (key >> 1) & 7 : 0;
    }
};

// K of a unit on its way, for this lane: row l % 16 of each run, its quarter's values.
template <int D>
struct KeysComing {
    uint32_t codes[4][Direct<D>::kSteps];
    uint32_t scale[4][Direct<D>::kScales];
};

// A workgroup's run of tasks of RT tiles of 16 rows.  Each of the four waves takes
// every fourth unit of a task, for all rows, and stages it alone, so no wave waits for
// another until the parts of the four are joined at the task's end.
//
// K goes from memory to registers and is widened there: 16 bytes a lane are a whole block of a key
// at D = 128, the A operand of S^T = K Q^T as they stand if Q's values are taken in the
// same order.  V goes to LDS as it is; a transposing read of bytes gives a lane 8 keys'
// codes of two neighbouring values of the output, a byte has one scale (its
// key's, of this block of 32), so one instruction widens both, and two permutations make
// the rows of the A operands of O^T = V^T P^T, even and odd.  P^T is its B operand as it
// comes from S^T, rounded to the storage type as in the 16-bit kernels.
//
// The next unit's loads go out before this one's work, and the next task's first ones
// before this one's parts are joined, so a wave always has some of the cache on its way (8.5 KB at
// D = 128).
template <class T, int D, int RT, Kind kKind>
__device__ __forceinline__ void run_direct(const AttendArgs& a, const Totals& t, const Deal& deal, const Batch& batch,
                                           uint32_t group_number, char* smem, float (*wave_stats)[2][48], int* flags) {
    using S = Direct<D>;
    using V8 = typename T::V8;
    const int wave = forget_scalar(uniform((int32_t)(threadIdx.x >> 6)));
    const uint32_t run_start = group_start(deal, group_number), run_end = group_start(deal, group_number + 1);
    Work<In4Direct, D, kKind> work{a, t, batch, (uint32_t)(uintptr_t)(SV_LDS char*)smem, group_number, run_end,
                                   {}, 0, false, run_start, 0, 0, 0, 0, false, wave, flags + 1};
    if (!work.advance()) return;
    const int lane = lane_again<In4Direct>(), quarter = lane >> 4, of16 = lane & 15;
    char* const mine = smem + wave * S::kWave;
    const uint32_t mine_lds = work.lds + wave * S::kWave;
    float* const v_scales = (float*)(mine + 2 * S::kTile);

    struct Row {
        int b, token, head;
        bool live;
    };
    auto row_of = [&](const Segment& g, int in_task) {
        const int group = forget_scalar(a.split.group);  // (see Work::advance)
        const int row = g.row0 + in_task;
        const int flat = (int)((uint32_t)row / (uint32_t)group);
        Row r{g.b, flat, g.kv_head * group + (row - flat * group), flat < g.count};
        if (kKind == kShared) {
            r.live = flat < batch.cum_tokens[a.split.batch];
            r.b = r.live ? find(batch.cum_tokens, a.split.batch, flat) : 0;
            r.token = r.live ? flat - batch.cum_tokens[r.b] : 0;
        }
        return r;
    };

    // ---- Q: B operands of the products, those of several row tiles made by one wave each, for LDS
    constexpr bool kQInLds = S::q_in_lds(RT);
    constexpr int kQs = kQInLds ? (RT * S::kSteps + 3) / 4 : S::kSteps;  // of a wave
    V8* const q_lds = (V8*)(smem + 4 * S::kWave);                        // [product][row tile][lane]
    V8 q[kQs];
    auto load_q = [&]() {
        // (what is made from it would else be kept in registers from before)
        const int lane = lane_again<In4Direct>(), quarter = lane >> 4, of16 = lane & 15;
#pragma unroll
        for (int i = 0; i < kQs; ++i) {
            const int at = kQInLds ? 4 * i + wave : i, s = kQInLds ? at / RT : i, r = kQInLds ? at % RT : 0;
            u32x4 x = {0, 0, 0, 0};
            if (s < S::kSteps) {
                const Row row = row_of(work.g, r * 16 + of16);
                const uint16_t* const from =
                    a.q + row.b * a.q_stride[0] + row.token * a.q_stride[1] + row.head * a.q_stride[2];
                if (row.live && S::there(s, quarter)) x = *(const u32x4*)(from + S::value(s, quarter));
            }
            q[i] = __builtin_bit_cast(V8, x);
        }
    };
    auto keep_q = [&]() {
        if constexpr (kQInLds) {
            const int lane = lane_again<In4Direct>();
#pragma unroll
            for (int i = 0; i < kQs; ++i)
                if (4 * i + wave < RT * S::kSteps) q_lds[(4 * i + wave) * 64 + lane] = q[i];
        }
    };

    // ---- a unit's loads
    auto run_at = [&](int at) {  // bytes before the rows of a run
        const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)work.row_low, at);
        const uint32_t high = (uint32_t)__builtin_amdgcn_readlane((int)work.row_high, at);
        return (int64_t)((uint64_t)high << 32 | low);
    };
    auto fetch_v = [&](uint32_t u, int buffer, uint32_t(&vs)[2]) {
        if (u - work.paged == 64) {
            work.paged = u;
            work.look_up();
        }
        const int at = (int)(u - work.paged);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const char* const v_from = (const char*)a.v_cache + run_at(at + r);
            // 16 bytes a lane
            constexpr int kChunks = S::kRow / 16;
#pragma unroll
            for (int c = 0; c < 16 * S::kRow; c += 1024) {
                uint32_t offset = (uint32_t)lane * 16;
                if (S::kRow % 32 == 0) {
                    const int place = lane + c / 16, key = place / kChunks, chunk = place % kChunks;
                    offset = (uint32_t)(key * S::kRow + ((chunk ^ S::swizzle(key)) * 16));
                }
                if (16 * S::kRow - c >= 1024 || lane * 16 < 16 * S::kRow - c)
                    load_to_lds(mine_lds + buffer * S::kTile + r * (16 * S::kRow) + c, v_from, offset);
            }
        }
        // V's scales, a key a lane
        const uint32_t low = (uint32_t)__shfl((int)work.row_low, at + quarter);
        const uint32_t high = (uint32_t)__shfl((int)work.row_high, at + quarter);
        const uint32_t scales = (uint32_t)__shfl((int)work.row_scales, at + quarter);
        const char* const from = (const char*)a.v_cache + (int64_t)((uint64_t)high << 32 | low) + scales +
                                 (uint32_t)(of16 * S::kBlocks);
        if constexpr (S::kBlocks == 2) {
            vs[0] = *(const uint16_t*)from;
        } else if constexpr (S::kBlocks == 3) {
            vs[0] = (uint32_t)*(const uint8_t*)from | (uint32_t)*(const uint8_t*)(from + 1) << 8 |
                    (uint32_t)*(const uint8_t*)(from + 2) << 16;
        } else if constexpr (S::kBlocks == 4) {
            vs[0] = *(const uint32_t*)from;
        } else {
            const u32x2 x = *(const u32x2*)from;
            vs[0] = x[0];
            vs[1] = x[1];
        }
    };

    auto fetch_k = [&](uint32_t u, KeysComing<D>& k) {  // (behind fetch_v)
        const int at = (int)(u - work.paged);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const char* const k_from = (const char*)a.k_cache + run_at(at + r);
            const char* const k_scales = k_from + (uint32_t)__builtin_amdgcn_readlane((int)work.row_scales, at + r);
#pragma unroll
            for (int j = 0; j < S::kWides; ++j) {
                const char* const from = k_from + (uint32_t)(of16 * S::kRow + (4 * j + quarter) * (S::kWide / 2));
                if constexpr (S::kWide == 32) {
                    const u32x4 x = *(const u32x4*)from;
#pragma unroll
                    for (int e = 0; e < 4; ++e) k.codes[r][4 * j + e] = x[e];
                } else {
                    const u32x2 x = *(const u32x2*)from;
                    k.codes[r][2 * j] = x[0];
                    k.codes[r][2 * j + 1] = x[1];
                }
                const uint32_t block = (uint32_t)(of16 * S::kBlocks + (4 * j + quarter) * S::kWide / 32);
                k.scale[r][j] = *(const uint8_t*)(k_scales + block);
            }
            if constexpr (S::kRest > 0) {
                uint32_t x = 0;
                if (S::there(S::kSteps - 1, quarter))
                    x = *(const uint32_t*)(k_from + (uint32_t)(of16 * S::kRow + 32 + 4 * quarter));
                k.codes[r][S::kSteps - 1] = x;
                k.scale[r][S::kScales - 1] = *(const uint8_t*)(k_scales + (uint32_t)(of16 * S::kBlocks + 2));
            }
        }
    };

    // K of the next unit goes out with V before this one's work or, where there are no registers for both, when this one's K
    // has been used, into its registers.
    constexpr bool kLate = RT > 1 || D > 128;
    KeysComing<D> k[kLate ? 1 : 2];
    uint32_t vs[2][2] = {};
    auto fetch_first = [&]() {
        const uint32_t u = work.g.first + wave;
        if (u < work.g.end) {
            fetch_v(u, 0, vs[0]);
            fetch_k(u, k[0]);
        }
    };
    fetch_first();
    load_q();
    keep_q();
    if constexpr (kQInLds) lds_barrier();

    for (;;) {
        const Segment g = work.g;
        // keys that the lane's row of tile r sees (rarely needed, so not kept)
        auto limit_of = [&](int r) {
            return kKind == kShared ? a.prefix_len : g.length + row_of(g, r * 16 + (lane_again<In4Direct>() & 15)).token + 1;
        };
        f32x4 o[RT][S::kPieces][2];
        float top[RT], sum[RT];
        bool far[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
#pragma unroll
            for (int p = 0; p < S::kPieces; ++p) o[r][p][0] = o[r][p][1] = f32x4(0.0f);
            top[r] = -INFINITY;
            sum[r] = 0.0f;
            far[r] = false;
        }
        const int own_first = kKind == kShared ? 0 : own_common(a.split, g);
        const int last = work.last_key(kKind == kShared);  // the last key that there is

        // ---- a unit's work
        auto look_far = [&](int r) { far[r] = fabsf(top[r] * a.scale_log2) > kFarScores && top[r] != -INFINITY; };
        auto compute = [&](uint32_t u, int buffer, const KeysComing<D>& k, const uint32_t(&vs_in)[2], auto after_scores) {
            const int key0 = (int)u * kKeys;
            const bool partial = key0 + kKeys > (kKind == kShared ? a.prefix_len : own_first);
            const char* const v_tile = mine + buffer * S::kTile;
            uint32_t vs[2] = {vs_in[0], vs_in[1]};
            // Blocks of V that are not finite, of keys that some rows see and others do not (else they have weights, or
            // no row sees them): their products are made one by one, see below.
            uint64_t special = 0;
            if (partial) {
                const int key = key0 + lane;
                if (key > last) vs[0] = vs[1] = 0;  // (scales like any)
                uint32_t most = 0;
#pragma unroll
                for (int p = 0; p < S::kPieces; ++p) most = max(most, (vs[p / 4] >> (8 * (p % 4))) & 255u);
                special = __ballot(most > last_finite(T()));
            }
            if (special != 0 && (special >> lane & 1)) vs[0] = vs[1] = 0;
#pragma unroll
            for (int p = 0; p < S::kPieces; ++p)
                v_scales[p * kKeys + lane] = __uint_as_float(((vs[p / 4] >> (8 * (p % 4))) & 255u) << 23);

            f32x4 w[RT][4];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int n = 0; n < 4; ++n) w[r][n] = f32x4(0.0f);
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) {
                if (RT > 1) in_order();  // (nor has it registers for more of Q)
                V8 y[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) y[r] = kQInLds ? q_lds[(s * RT + r) * 64 + lane] : q[kQInLds ? 0 : s];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const float by = __uint_as_float(k.scale[n][S::scale(s)] << 23);
                    const V8 x = __builtin_bit_cast(V8, T::wide(k.codes[n][s], by));
#pragma unroll
                    for (int r = 0; r < RT; ++r) w[r][n] = mma16(x, y[r], w[r][n]);
                }
            }
            after_scores();
            // weights
            V8 weights[RT][2];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if (partial) {
                    const int limit = limit_of(r);
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (key0 + 16 * n + 4 * quarter + i >= limit) w[r][n][i] = -INFINITY;
                }
                float most = -INFINITY;
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) most = fmaxf(most, w[r][n][i]);
                // (as in the 16-bit kernels: the weights' reference follows the maximum where it rises by more than 2^8, row by row, so
                // that keys which only other rows see change nothing)
                if (__any(most - top[r] > a.lazy)) {
                    most = quarters_max(most);
                    const bool rises = most - top[r] > a.lazy;
                    const float now = rises ? most : top[r];
                    const float by = rises ? exp2_hw((top[r] - now) * a.scale_log2) : 1.0f;
                    sum[r] *= by;
#pragma unroll
                    for (int p = 0; p < S::kPieces; ++p) {
                        o[r][p][0] *= by;
                        o[r][p][1] *= by;
                    }
                    top[r] = now;
                    look_far(r);
                }
                if (__any(far[r])) {
                    const float ref = far[r] ? top[r] : 0.0f;
#pragma unroll
                    for (int n = 0; n < 4; ++n) w[r][n] -= ref;
                }
                const float shift = (far[r] || top[r] == -INFINITY) ? T::kBias : fmaf(-top[r], a.scale_log2, T::kBias);
                float add = 0.0f;
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w[r][n][i] = exp2_hw(fmaf(w[r][n][i], a.scale_log2, shift));
                        add += w[r][n][i];
                    }
                sum[r] += add;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    f32x8 x;
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = w[r][2 * b + i / 4][i % 4];
                    weights[r][b] = __builtin_convertvector(x, V8);
                }
            }
            if (special != 0) {
                // Rows take the products of such blocks from the keys that they see.
#pragma unroll 1
                for (uint64_t left = special; left != 0; left &= left - 1) {
                    const int key = __builtin_ctzll(left), n = key >> 4, i = key & 3, from = of16 + 16 * ((key >> 2) & 3);
                    const uint32_t s0 = (uint32_t)__builtin_amdgcn_readlane((int)vs_in[0], key);
                    const uint32_t s1 = (uint32_t)__builtin_amdgcn_readlane((int)vs_in[1], key);
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        float weight = 0.0f;
#pragma unroll
                        for (int j = 0; j < 16; ++j) weight = (j == 4 * n + i) ? (float)weights[r][j / 8][j % 8] : weight;
                        weight = __shfl(weight, from);
                        const bool sees = key0 + key < limit_of(r);
#pragma unroll
                        for (int p = 0; p < S::kPieces; ++p) {
                            if (32 * p + 8 * quarter >= D) continue;
                            const float scale = __uint_as_float((((p < 4 ? s0 : s1) >> (8 * (p % 4))) & 255u) << 23);
                            const int chunk = (p ^ S::swizzle(key)) * 16 + 4 * quarter;
                            const u32x4 x = T::wide(*(const uint32_t*)(v_tile + key * S::kRow + chunk), scale);
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (sees) o[r][p][e % 2][e / 2] += weight * T::value((x[e / 2] >> (16 * (e % 2))) & 0xffffu);
                        }
                    }
                }
            }
            // O^T += V^T P^T, 32 keys and 32 values of head_dim at a time
            struct Step {
                i32x2 codes;
                f32x4 scales[2];
            };
            auto read = [&](int m) {
                // (lane i of 16 reads half i % 2 of the 16 bytes of the quarter's key i / 2: 4 of the first 16
                // keys, 4 of the others, the order in which P has them)
                const int b = m / S::kPieces, p = m % S::kPieces;
                const int j = of16 / 2, key = 32 * b + 16 * (j / 4) + 4 * quarter + j % 4;
                Step x;
                x.codes = __builtin_amdgcn_ds_read_tr8_b64_v2i32((SV_LDS i32x2*)(SV_LDS char*)(
                    v_tile + key * S::kRow + ((p ^ S::swizzle(key)) * 16) + (of16 % 2) * 8));
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    x.scales[h] = *(const f32x4*)(v_scales + p * kKeys + 32 * b + 16 * h + 4 * quarter);
                return x;
            };
            constexpr int kAll = 2 * S::kPieces;
            Step steps[2];
            steps[0] = read(0);
#pragma unroll
            for (int m = 0; m < kAll; ++m) {
                const int b = m / S::kPieces, p = m % S::kPieces;
                if (m + 1 < kAll) steps[(m + 1) % 2] = read(m + 1);
                in_order();  // (what else the compiler would read ahead there are no registers for)
                const Step& x = steps[m % 2];
                uint32_t pair[8];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    pair[4 * h] = wide_pair<0>(T(), (uint32_t)x.codes[h], x.scales[h][0]);
                    pair[4 * h + 1] = wide_pair<1>(T(), (uint32_t)x.codes[h], x.scales[h][1]);
                    pair[4 * h + 2] = wide_pair<2>(T(), (uint32_t)x.codes[h], x.scales[h][2]);
                    pair[4 * h + 3] = wide_pair<3>(T(), (uint32_t)x.codes[h], x.scales[h][3]);
                }
                u32x4 even, odd;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    even[e] = __builtin_amdgcn_perm(pair[2 * e + 1], pair[2 * e], 0x05040100u);
                    odd[e] = __builtin_amdgcn_perm(pair[2 * e + 1], pair[2 * e], 0x07060302u);
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    o[r][p][0] = mma16(__builtin_bit_cast(V8, even), weights[r][b], o[r][p][0]);
                    o[r][p][1] = mma16(__builtin_bit_cast(V8, odd), weights[r][b], o[r][p][1]);
                }
            }
        };

        {
            uint32_t u = g.first + wave;
            auto turn = [&](auto odd) {
                constexpr int kHere = decltype(odd)::value, kThere = 1 - kHere;
                const bool more = u + 4 < g.end;
                own_loads_landed();
                if (more) {
                    fetch_v(u + 4, kThere, vs[kThere]);
                    if constexpr (!kLate) fetch_k(u + 4, k[kThere]);
                }
                in_order();
                compute(u, kHere, k[kLate ? 0 : kHere], vs[kHere], [&]() {
                    if constexpr (kLate) {
                        in_order();
                        if (more) fetch_k(u + 4, k[0]);
                        in_order();
                    }
                });
                u += 4;
            };
            // (two at a time, so that registers keep their places)
            while (u < g.end) {
                turn(std::integral_constant<int, 0>());
                if (u >= g.end) break;
                turn(std::integral_constant<int, 1>());
            }
        }

        // ---- the next task's first loads
        int* const flag = work.flag;  // (set where this task has a page that there is not)
        const bool whole = kKind == kJoined && work.whole;
        const int64_t place = work.place;
        const bool more = work.advance();
        in_order();
        if (more) {
            fetch_first();
            if constexpr (!kQInLds) load_q();
        }
        in_order();

        // ---- join the four waves' parts, some pieces of a row tile at a time, then write
        const int again = lane_again<In4Direct>(), my_row = again & 15, my_quarter = again >> 4;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            sum[r] = quarters_sum(sum[r]);
            if (my_quarter == 0) {
                wave_stats[wave][0][r * 16 + my_row] = top[r];
                wave_stats[wave][1][r * 16 + my_row] = sum[r];
            }
        }
        lds_barrier();
        const bool nan = *flag != 0;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float now = -INFINITY;
#pragma unroll
            for (int x = 0; x < 4; ++x) now = fmaxf(now, wave_stats[x][0][r * 16 + my_row]);
            const float ref = now == -INFINITY ? 0.0f : now;
            const float by = exp2_hw((top[r] - ref) * a.scale_log2);
            // 16 threads a row, 4 values at a time
            const int row = 4 * wave + my_quarter, in = r * 16 + row;
            float most = -INFINITY, total = 0.0f;
#pragma unroll
            for (int x = 0; x < 4; ++x) most = fmaxf(most, wave_stats[x][0][in]);
            const float reference = most == -INFINITY ? 0.0f : most;
#pragma unroll
            for (int x = 0; x < 4; ++x)
                total += exp2_hw((wave_stats[x][0][in] - reference) * a.scale_log2) * wave_stats[x][1][in];
            const Row to = row_of(g, in);
            const float times = nan ? forget(NAN) : whole ? 1.0f / total : 1.0f;
            if (!whole && my_row == 0) {
                a.part_max[place + in] = most;
                a.part_sum[place + in] = total;
            }
#pragma unroll
            for (int c = 0; c < S::kBoxes; ++c) {
                float* const box = (float*)(mine + S::kTile) + my_row * S::kPitch + 8 * my_quarter;
#pragma unroll
                for (int e = 0; e < S::kBoxPieces; ++e) {
                    const int p = c * S::kBoxPieces + e;
                    const f32x4 x = o[r][p][0] * by, y = o[r][p][1] * by;
                    *(f32x4*)(box + 32 * e) = f32x4{x[0], y[0], x[1], y[1]};
                    *(f32x4*)(box + 32 * e + 4) = f32x4{x[2], y[2], x[3], y[3]};
                }
                lds_barrier();
#pragma unroll
                for (int j = 0; j < (8 * S::kBoxPieces + 15) / 16; ++j) {
                    const int in_box = 4 * (my_row + 16 * j), d = 32 * c * S::kBoxPieces + in_box;
                    if (in_box >= 32 * S::kBoxPieces || d >= D) continue;
                    f32x4 x = f32x4(0.0f);
#pragma unroll
                    for (int from = 0; from < 4; ++from)
                        x += *(const f32x4*)((const float*)(smem + from * S::kWave + S::kTile) + row * S::kPitch + in_box);
                    x *= times;
                    if (!whole)
                        *(f32x4*)(a.part_out + (place + in) * D + d) = x;
                    else if (to.live)
                        *(u32x2*)(a.out + to.b * a.out_stride[0] + to.token * a.out_stride[1] + to.head * a.out_stride[2] +
                                  d) = __builtin_bit_cast(u32x2, __builtin_convertvector(x, typename T::V4));
                }
                lds_barrier();
            }
        }
        if (!more) break;
        if (wave == 0 && again == 0) *flag = 0;
        if constexpr (kQInLds) {
            load_q();
            keep_q();
        }
        lds_barrier();  // (the flag and the statistics are free, too)
    }
}

}  // namespace
}  // namespace sv
