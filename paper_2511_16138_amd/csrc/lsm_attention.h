// Attention over a paged cache: the device code and the plan that the kernels of lsm_attention.hip (pages of 16 bits) and lsm_window.hip (pages of 8 bits,
// windows) have in common.
#pragma once
#include <hip/hip_runtime.h>

#include "lsm_common.h"
#include "lsm_pages.h"

namespace lsm {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int kType>
struct Half;
template <>
struct Half<LSM_BF16> {  // decode8: eight codes of type e4m3 times a power of two; where that is NaN or infinite, so are they
    typedef __bf16 type;
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    static constexpr uint32_t kExponent = 0x7F80;
    static __device__ __forceinline__ x8 decode8(uint32_t lo, uint32_t hi, float scale) {
        const x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true)};
        return x8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
    }
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Half<LSM_FP16> {
    typedef _Float16 type;
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    static constexpr uint32_t kExponent = 0x7C00;
    static __device__ __forceinline__ x8 decode8(uint32_t lo, uint32_t hi, float scale) {
        const x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true),
                         __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true)};
        return x8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
    }
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

constexpr uint32_t kThreads = 256, kWaves = kThreads / kWave;
constexpr uint32_t kWaveRows = 32;                      // rows of a wave: the columns of one product
constexpr uint32_t kWideRows = kWaveRows * kWaves;      // a wide tile: each wave has rows of its own, all go over the same keys
constexpr uint32_t kNarrowRows = kWaveRows;             // a narrow tile: all waves have the same rows, each goes over keys of its own
constexpr uint32_t kSplitKeys = 64;                     // ranges of keys are whole numbers of this

struct AttentionArgs {
    static constexpr bool kIn8 = false, kWindow = false;
    const void* q;
    void* out;
    float* lse;
    const void *k, *v;
    int64_t q_token, q_head, out_token, out_head;               // elements
    uint64_t k_head, v_head;                                    // bytes
    uint32_t k_page, k_token, v_page, v_token;
    const int32_t *group_offsets, *prefix_tables, *prefix_lens, *q_offsets, *own_tables, *own_lens;
    uint32_t n_tokens, n_requests, n_groups, n_pages, page_shift, kv_heads, share, rows;
    uint32_t share_part;  // for divisions by share, see divide
    uint64_t prefix_width, own_width;
    float scale;  // of the exponent of two
    // The plan.  Stage 0: rows packed by group over the prefix; stage 1: rows packed by request over its own pages, or over the
    // prefix and its own pages (`whole`).
    uint32_t whole, tiles[2], splits[2], wide[2], combos[2], combos_part[2], least[2], items0;
    uint32_t joined;     // the parts are joined by another kernel
    uint32_t search[2];  // search_step of groups and requests
    float* part_out;  // [split of either stage][KV head][row][head_dim]
    float2* part_ml;  // [split of either stage][KV head][row]: maximum in units of the exponent of two, sum; kNoPart = there is no part
};
constexpr float kNoPart = -1.f;  // no sum of weights

// kIn8: pages of 8 bits with scales (k_page and so on are bytes as they are there); kWindow: a token sees the last `window` tokens and the first `sinks`.
template <bool kIn8_, bool kWindow_>
struct WindowArgs : AttentionArgs {
    static constexpr bool kIn8 = kIn8_, kWindow = kWindow_;
    const uint8_t *k_scales, *v_scales;
    int64_t k_scale_page, k_scale_block, k_scale_head, v_scale_page, v_scale_block, v_scale_head;  // bytes
    int32_t window, sinks;
};

// x / d for x < 2^31, given part_of(d): a division takes forty instructions, and a workgroup's first pass over its instructions is most of a short call.
inline uint32_t part_of(uint32_t d) { return 0xFFFFFFFFu / d; }
__device__ __forceinline__ uint32_t divide(uint32_t x, uint32_t d, uint32_t part) {
    const uint32_t q = __umulhi(x, part);  // or one too small
    return x - q * d >= d ? q + 1 : q;
}

// The largest power of 64 below n, 1 for n = 1: a wave looks at every so many of n things first.
inline uint32_t search_step(uint64_t n) {
    uint32_t step = 1;
    while ((uint64_t)step * kWave < n) step *= kWave;
    return step;
}

// Splitting units of a range of keys.
__device__ __forceinline__ uint32_t split_units(uint32_t units, uint32_t splits, uint32_t least) {
    const uint32_t each = splits == 1 ? units : (units + splits - 1) / splits;
    return each < least ? least : each;
}
__device__ __forceinline__ uint32_t units_of(uint32_t keys) { return (keys + kSplitKeys - 1) / kSplitKeys; }

__device__ __forceinline__ uint32_t clamp_u32(int32_t v, uint64_t most) { return v < 0 ? 0 : (uint64_t)v > most ? (uint32_t)most : (uint32_t)v; }
__device__ __forceinline__ uint32_t prefix_len(const AttentionArgs& a, uint32_t g) { return clamp_u32(a.prefix_lens[g], a.prefix_width << a.page_shift); }
__device__ __forceinline__ uint32_t token_of_request(const AttentionArgs& a, uint32_t r) { return clamp_u32(a.q_offsets[r], a.n_tokens); }

// The last i < n with start(i) <= x, for start(0) <= x and start not descending; every lane of the wave calls and gets it.  first_step: search_step(n).
template <typename F>
__device__ __forceinline__ uint32_t last_not_above(uint32_t n, uint32_t first_step, uint64_t x, F start) {
    const uint32_t lane = threadIdx.x & (kWave - 1);
    uint32_t at = 0;
    for (uint32_t step = first_step; step != 0; step /= kWave) {
        const uint32_t i = at + lane * step;
        const int count = __popcll(__ballot(i < n && start(i) <= x));
        at += count > 0 ? (count - 1) * step : 0;
    }
    return at;
}
__device__ __forceinline__ uint32_t group_of(const AttentionArgs& a, uint32_t request) {
    return last_not_above(a.n_groups, a.search[0], request, [&](uint32_t g) { return (uint64_t)clamp_u32(a.group_offsets[g], a.n_requests); });
}

// exchange with the lane 32 further or back
__device__ __forceinline__ float other_half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What a workgroup works on.
struct Item {
    uint32_t row0, row_end;        // rows [row0, row_end) of the KV head
    const int32_t* table[2];       // pages of the two segments of keys: the prefix, the request's own
    uint32_t len[2];               // their lengths
    uint32_t unit0, unit1;         // splitting units of this range; the first segment has units_of(len[0]) of them
    uint64_t part;                 // the first row of its part: of this range, this KV head
    uint32_t token0, hidden;       // own keys that token t sees: t - token0 + 1 + len[1] - (new tokens), as hidden = that for t = token0, minus 1, wrapped
    uint32_t sink_units, window_unit;  // with a window: the units before sink_units and from window_unit on are worked on, and counted through in unit0 and unit1
};

// Copies twice 16 bytes a lane from global memory straight into LDS: lane i's from `from` + offset to `to` + kAt + 16 i, then kAt + 1024 + 16 i.  No register is
// written, so the compiler, which would otherwise wait for all copies before any LDS read, need not know; whoever reads the tile waits by wait_loads.
// `from` comes out of vector instructions (readlane), and a vector memory instruction that reads a scalar register needs five wait states after
// a vector instruction's write to it.  The compiler adds none before inline assembly, and may move `from` between two statements of it, so each statement
// has its own: the addition to m0 and four of s_nop 3.  m0 itself needs one before the copy.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // m0 is the compiler's own register; it keeps nothing there from one instruction to the next
template <int kAt>
__device__ __forceinline__ void copy_to_lds(uint64_t from, uint32_t offset0, uint32_t offset1, uint32_t to) {
    asm volatile(
        "s_add_u32 m0, %3, %4\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %2\n\t"
        "s_add_u32 m0, %3, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"v"(offset0),
        "v"(offset1), "s"(from), "s"(to), "n"(kAt), "n"(kAt + 1024)
        : "memory", "m0", "scc");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }
// Until at most kLeft of this wave's vector memory operations are under way, and none of its LDS ones.
template <int kLeft>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLeft) : "memory");
}

// Until none of this wave's LDS operations is under way.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// A score that exceeds the maximum that weights are relative to by less than this (as an exponent of two) does not move it: weights are
// at most 2^8 then, far from the end of either type, and the accumulators need not be scaled for every new maximum.
constexpr float kSlack = 8.f;

// A team of kTeam waves goes over tiles of kKeys keys: copies them through LDS and multiplies.  kHead = head_dim.
//
// Scores are computed transposed, keys times queries, so that a lane holds scores of one row (row = lane % 32) and the
// running maximum and sum are a lane's own, but for one exchange with the lane 32 away.  The lane's scores, rounded, are in the
// layout that the second product, values transposed times weights, wants as its right operand if its sum over keys takes them in the order
// 0-3, 8-11 | 4-7, 12-15 of every 16; its left operand, four keys at a time of one column of the values, is what the transposing LDS read gives.
// In LDS the 16-byte words of a row are permuted by the row's number so that neither read has bank conflicts.
template <int kType, int kHead, int kTeam, int kKeys>
struct Team {
    typedef typename Half<kType>::type T;
    typedef typename Half<kType>::x8 x8;
    typedef typename Half<kType>::x2 x2;
    static constexpr uint32_t kWords = kHead / 8;                                 // 16-byte words of a row
    static constexpr uint32_t kRowsPerLoad = kWave / kWords;                      // rows that one copy of a wave brings: all of one page
    static constexpr uint32_t kLoads = kKeys / (kRowsPerLoad * kTeam);            // copies of a wave for the keys of a tile, and for the values
    static constexpr uint32_t kBytes = kKeys * kHead * 2;                         // of a tile of keys, or of values
    static_assert(kKeys % (kRowsPerLoad * kTeam) == 0 && kKeys % 32 == 0 && kKeys <= 64 && kRowsPerLoad <= LSM_MIN_PAGE_TOKENS, "");

    static __device__ __forceinline__ uint32_t key_word(uint32_t row, uint32_t word) {  // where a 16-byte word of a key's row is
        return kWords >= 16 ? word ^ (row & 15) : word ^ ((row >> 1) & 7);
    }
    static __device__ __forceinline__ uint32_t value_word(uint32_t row, uint32_t word) {
        const uint32_t by = kWords >= 16 ? 2 * (row & 3) + ((row >> 2) & 1) : 2 * ((row >> 1) & 1) + ((row >> 2) & 1);
        return word ^ (by * 2);
    }

    x8 query[kHead / 16];
    f32x16 acc[kHead / 32];
    float most, sum;  // what the row's weights are relative to: the largest score so far, less at most kSlack; this lane's share of the sum

    __device__ __forceinline__ void start() {
#pragma unroll
        for (uint32_t i = 0; i < kHead / 32; i++)
#pragma unroll
            for (int j = 0; j < 16; j++) acc[i][j] = 0.f;
        most = -__builtin_inff(), sum = 0.f;
    }

    typedef f32x16 Scores[kKeys / 32];
    typedef x8 Weights[kKeys / 16];

    // Product i of a tile's scores: keys i % kGroups * 32 .. + 31, elements i / kGroups * 16 .. + 15.  Its left operand, from the keys in LDS:
    static constexpr uint32_t kGroups = kKeys / 32, kScores = kHead / 16 * kGroups, kAhead = 4;
    static __device__ __forceinline__ x8 key_operand(const char* keys, uint32_t i) {
        const uint32_t lane = threadIdx.x & (kWave - 1), row = i % kGroups * 32 + (lane & 31), h = lane >> 5;
        return *reinterpret_cast<const x8*>(keys + row * kHead * 2 + key_word(row, 2 * (i / kGroups) + h) * 16);
    }

    // The scores of a tile's keys.  LDS reads go four products ahead, here and below, and the scheduler leaves the order as it is written.
    __device__ __forceinline__ void score(const char* keys, Scores& s) const {
#pragma unroll
        for (uint32_t b = 0; b < kGroups; b++)
#pragma unroll
            for (int j = 0; j < 16; j++) s[b][j] = 0.f;
        x8 k[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; i++) k[i] = key_operand(keys, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t i = 0; i < kScores; i++) {
            s[i % kGroups] = Half<kType>::mfma(k[i % kAhead], query[i / kGroups], s[i % kGroups]);
            if (i + kAhead < kScores) k[i % kAhead] = key_operand(keys, i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // present: which of the tile's keys there are; limit: how many of them this lane's row may see.
    static __device__ __forceinline__ void mask(Scores& s, uint64_t present, int32_t limit) {
        const uint32_t h = (threadIdx.x & (kWave - 1)) >> 5;
#pragma unroll
        for (int b = 0; b < kKeys / 32; b++) {
            const int32_t rest = limit - b * 32;
            uint32_t see = rest <= 0 ? 0 : rest >= 32 ? ~0u : (1u << rest) - 1;
            see = (see & (uint32_t)(present >> (b * 32))) >> (4 * h);
#pragma unroll
            for (int j = 0; j < 16; j++) s[b][j] = (see >> (8 * (j / 4) + j % 4)) & 1 ? s[b][j] : -__builtin_inff();
        }
    }

    // see: which of the tile's keys this lane's row sees and there are.
    static __device__ __forceinline__ void mask_bits(Scores& s, uint64_t see) {
        const uint32_t h = (threadIdx.x & (kWave - 1)) >> 5;
#pragma unroll
        for (int b = 0; b < kKeys / 32; b++) {
            const uint32_t mine = (uint32_t)(see >> (b * 32)) >> (4 * h);
#pragma unroll
            for (int j = 0; j < 16; j++) s[b][j] = (mine >> (8 * (j / 4) + j % 4)) & 1 ? s[b][j] : -__builtin_inff();
        }
    }

    // The largest of a lane's scores.
    static __device__ __forceinline__ float largest(const Scores& s) {
        float top = s[0][0];
#pragma unroll
        for (uint32_t b = 0; b < kGroups; b++)
#pragma unroll
            for (int j = 0; j < 16; j++) top = fmaxf(top, s[b][j]);
        return top;
    }

    // Brings the accumulators to what the next weights are relative to, given the lane's largest score; the addend of the weights' exponents.
    __device__ __forceinline__ float rebase(float top, float scale) {
        top = other_half_max(top);
        const bool moves = (top - most) * scale > kSlack;
        if (__any(moves)) {
            const float by = moves ? __builtin_amdgcn_exp2f((most - top) * scale) : 1.f;
            sum *= by;
#pragma unroll
            for (uint32_t i = 0; i < kHead / 32; i++)
#pragma unroll
                for (int j = 0; j < 16; j++) acc[i][j] *= by;
            most = moves ? top : most;
        }
        return most == -__builtin_inff() ? 0.f : -most * scale;  // a row that has seen nothing: all weights 0
    }

    // Weights 2 i and 2 i + 1 of a lane, rounded to nearest as the values are, since the matrix cores take operands of one type (the head of this file has the
    // error); the sum is of the weights before that.
    __device__ __forceinline__ void weight_pair(const Scores& s, Weights& p, uint32_t i, float scale, float base, float& more) {
        const uint32_t b = i / 8, j = i % 8 * 2;
        const f32x2 e = {__builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j], scale, base)), __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j + 1], scale, base))};
        const x2 w = __builtin_convertvector(e, x2);
        sum += e[0], more += e[1];
        p[i / 4][j % 8] = w[0], p[i / 4][j % 8 + 1] = w[1];
    }
    static constexpr uint32_t kPairs = kKeys / 4;

    __device__ __forceinline__ void weights(const Scores& s, Weights& p, float scale, float base) {
        float more = 0.f;
#pragma unroll
        for (uint32_t i = 0; i < kPairs; i++) weight_pair(s, p, i, scale, base, more);
        sum += more;
    }

    // The weights of a tile and, in the shadow of its products, the scores of the next one.
    __device__ __forceinline__ void weights_and_score(const Scores& s, Weights& p, float scale, float base, const char* next_keys, Scores& next) {
        float more = 0.f;
#pragma unroll
        for (uint32_t b = 0; b < kGroups; b++)
#pragma unroll
            for (int j = 0; j < 16; j++) next[b][j] = 0.f;
        x8 k[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; i++) k[i] = key_operand(next_keys, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t i = 0; i < kScores; i++) {
            next[i % kGroups] = Half<kType>::mfma(k[i % kAhead], query[i / kGroups], next[i % kGroups]);
            if (i + kAhead < kScores) k[i % kAhead] = key_operand(next_keys, i + kAhead);
#pragma unroll
            for (uint32_t j = i * kPairs / kScores; j < (i + 1) * kPairs / kScores; j++) weight_pair(s, p, j, scale, base, more);
            asm volatile("" : "+v"(sum), "+v"(more));  // here, in the products' shadow, and not behind them
            __builtin_amdgcn_sched_barrier(0);
        }
        sum += more;
    }

    // The left operand of product i of weigh: of columns i % kColumns * 32 .. + 31 the keys i / kColumns * 16 .. + 15.  16 lanes read a block of 4 keys x 16
    // columns, lane i of them gets column i.
    static constexpr uint32_t kColumns = kHead / 32, kProducts = kColumns * (kKeys / 16);
    static __device__ __forceinline__ x8 value_operand(const char* values, uint32_t i) {
        const uint32_t lane = threadIdx.x & (kWave - 1), h = lane >> 5, i16 = lane & 15, column = ((lane >> 4) & 1) * 16 + (i16 & 3) * 4;
        union {
            x8 all;
            s16x4 part[2];
        } u;
#pragma unroll
        for (uint32_t j = 0; j < 2; j++) {
            const uint32_t row = i / kColumns * 16 + 8 * j + 4 * h + (i16 >> 2), at = i % kColumns * 32 + column;
            const char* from = values + row * kHead * 2 + value_word(row, at >> 3) * 16 + (at & 4) * 2;
            u.part[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(from));
        }
        return u.all;
    }

    // Bits 15 and 31: whether either half of a word of two values is infinite or NaN, its exponent all ones.
    static __device__ __forceinline__ uint32_t not_finite(uint32_t two) {
        constexpr uint32_t k = Half<kType>::kExponent;
        return (two & (k | k << 16)) + ((0x8000 - k) | (0x8000 - k) << 16);
    }

    // Adds the values of a tile that are infinite or NaN to the rows that see their keys: there they decide the sum whatever their weight is.
    // seen: how many of the tile's keys this lane's row sees (int32_t), or which (uint64_t).
    static __device__ __forceinline__ bool sees(uint32_t row, int32_t seen) { return (int32_t)row < seen; }
    static __device__ __forceinline__ bool sees(uint32_t row, uint64_t seen) { return (seen >> row) & 1; }
    template <typename S>
    __device__ __forceinline__ void add_not_finite(const char* values, S seen) {
        const uint32_t h = (threadIdx.x & (kWave - 1)) >> 5;
#pragma unroll 1
        for (uint32_t row = 0; row < kKeys; row++) {
#pragma unroll
            for (uint32_t i = 0; i < kColumns * 4; i++) {
                const uint32_t column = i * 8 + h * 4;  // of the accumulators i / 4, elements i % 4 * 4 .. + 3
                union {
                    uint2 words;
                    T one[4];
                } v;
                v.words = *reinterpret_cast<const uint2*>(values + row * kHead * 2 + value_word(row, column >> 3) * 16 + (column & 4) * 2);
                const uint32_t bits[2] = {not_finite(v.words.x), not_finite(v.words.y)};
#pragma unroll
                for (uint32_t j = 0; j < 4; j++)
                    if (sees(row, seen) && ((bits[j / 2] >> (j % 2 * 16 + 15)) & 1)) acc[i / 4][i % 4 * 4 + j] += (float)v.one[j];
            }
        }
    }

    // The values, which are in LDS, by their weights; kLargest: and the largest of the next tile's scores.
    template <bool kLargest>
    __device__ __forceinline__ float weigh(const char* values, const Weights& p, const Scores& next) {
        float top = -__builtin_inff();
        x8 v[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; i++) v[i] = value_operand(values, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t i = 0; i < kProducts; i++) {
            acc[i % kColumns] = Half<kType>::mfma(v[i % kAhead], p[i / kColumns], acc[i % kColumns]);
            if (i + kAhead < kProducts) v[i % kAhead] = value_operand(values, i + kAhead);
            if (kLargest) {
#pragma unroll
                for (uint32_t j = i * kPairs / kProducts; j < (i + 1) * kPairs / kProducts; j++) top = fmaxf(fmaxf(top, next[j / 8][j % 8 * 2]), next[j / 8][j % 8 * 2 + 1]);
                asm volatile("" : "+v"(top));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        return top;
    }
};

// A wide tile's keys are copied by all waves together, a narrow one's by each wave for itself.
template <int kType, int kHead>
struct Shape {
    static constexpr int kWideKeys = 64, kNarrowKeys = kHead == 64 ? 64 : 32;
    typedef Team<kType, kHead, kWaves, kWideKeys> Wide;
    typedef Team<kType, kHead, 1, kNarrowKeys> Narrow;
    static constexpr uint32_t kWideLds = Wide::kBytes * 2 * 2, kNarrowLds = Narrow::kBytes * 2 * kWaves;
    static constexpr uint32_t kLds = (kWideLds > kNarrowLds ? kWideLds : kNarrowLds) + 16;  // and a word of each wave
    static constexpr uint32_t kSlicePitch = 68;  // floats between rows of a slice of 64 columns of results in LDS
    static constexpr uint32_t kOutLds = kWaves * 32 * kSlicePitch * 4 + kWaves * 32 * 8;
    static constexpr uint32_t kAllLds = kLds > kOutLds ? kLds : kOutLds;
    static_assert(kAllLds <= 160 * 1024, "");
};

// The first n of 64.
__device__ __forceinline__ uint64_t first_bits(int32_t n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }

template <int kType, int kHead, bool kWide, typename A>
__device__ __forceinline__ void attend(const A& a, const Item& w, uint32_t kv_head, char* lds) {
    typedef Shape<kType, kHead> S;
    typedef typename Half<kType>::type T;
    typedef typename Half<kType>::x8 x8;
    constexpr int kTeam = kWide ? kWaves : 1, kKeys = kWide ? S::kWideKeys : S::kNarrowKeys;
    typedef Team<kType, kHead, kTeam, kKeys> X;
    constexpr uint32_t kPerUnit = kSplitKeys / kKeys;
    constexpr uint64_t kAllKeys = kKeys == 64 ? ~0ull : (1ull << kKeys) - 1;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = threadIdx.x & (kWave - 1), n = lane & 31, h = lane >> 5;
    char* buffers = lds + (kWide ? 0 : wave * 2 * X::kBytes);

    X x;
    x.start();
    const uint32_t row = w.row0 + (kWide ? wave * 32 : 0) + n;
    const bool has_row = row < w.row_end;
    const uint32_t some_row = has_row ? row : w.row_end - 1;  // rows behind the last are copies of it, and left out in the end
    const uint32_t token = divide(some_row, a.share, a.share_part), head = kv_head * a.share + (some_row - token * a.share);
    {
        const T* from = static_cast<const T*>(a.q) + (int64_t)token * a.q_token + (int64_t)head * a.q_head + h * 8;
#pragma unroll
        for (uint32_t c = 0; c < kHead / 16; c++) x.query[c] = *reinterpret_cast<const x8*>(from + c * 16);
    }
    const int32_t sees = (int32_t)(token - w.token0 + w.hidden) + 1;  // own keys this row sees
    // tiles of this range: of the first segment, then of the second as far as any row of the tile sees
    const uint32_t units0 = units_of(w.len[0]), tile_rows = kWide ? kWideRows : kNarrowRows;
    const uint32_t last_row = w.row_end - w.row0 < tile_rows ? w.row_end - 1 : w.row0 + tile_rows - 1;
    const uint32_t first_row = w.row0 + (kWide ? wave * 32 : 0);
    const int32_t most_seen = (int32_t)(divide(last_row, a.share, a.share_part) - w.token0 + w.hidden) + 1;
    const int32_t least_seen = (int32_t)(divide(first_row, a.share, a.share_part) - w.token0 + w.hidden) + 1;  // of the rows of this wave
    const uint32_t seen = most_seen < 0 ? 0 : (uint32_t)most_seen < w.len[1] ? (uint32_t)most_seen : w.len[1];
    uint32_t units = a.n_pages == 0 ? 0 : units0 + units_of(seen);
    if (A::kWindow) units = units > w.window_unit ? units - (w.window_unit - w.sink_units) : units < w.sink_units ? units : w.sink_units;
    const uint32_t unit1 = w.unit1 < units ? w.unit1 : units;
    const uint32_t tile_end = unit1 * kPerUnit, step = kWide ? 1 : kWaves, second = units0 * kPerUnit;  // tiles from `second` on are of the second segment
    uint32_t t = w.unit0 * kPerUnit + (kWide ? 0 : wave);

    // With a window tiles are counted through those that are worked on; a tile's place among all of them:
    auto place_of = [&](uint32_t t) { return !A::kWindow || t < w.sink_units * kPerUnit ? t : t + (w.window_unit - w.sink_units) * kPerUnit; };
    // The first key that the window of a row's token reaches, as a place in prefix and own tokens; of this lane's row, of the last rows of the wave and of the tile.
    auto window_from = [&](uint32_t token) {
        if constexpr (A::kWindow) return (int32_t)(w.len[0] + token - w.token0 + w.hidden) + 1 - a.window;
        else return 0;
    };
    const uint32_t last_of_wave = first_row + 31 < w.row_end ? first_row + 31 : w.row_end - 1;
    const int32_t from = window_from(token), from_wave = window_from(divide(last_of_wave, a.share, a.share_part)), from_tile = window_from(divide(last_row, a.share, a.share_part));

    // Where the next tiles' tokens are, 16 of them a lane: addresses of keys and of values, and `there`: which of them have a page.  One load for 64 of these, and
    // no vector memory operations but the copies in between, which the waits below count.  Where there is no page any does: the scores of
    // keys that are not there are masked, and their values are zeroed in LDS.
    constexpr uint32_t kBlocks = kKeys / 16;  // lanes of a tile
    uint64_t k_at = 0, v_at = 0, there = 0, whole = 0;  // whole: which have a page and 16 tokens
    uint32_t first_tile = 0;                            // of lane 0
    uint32_t k_scale = 0, v_scale = 0;                  // of 8 bits: bits of the scales
    auto find_pages = [&](uint32_t t) {
        const uint32_t counted = t + lane / kBlocks * step, u = place_of(counted);
        const bool own = u >= second;
        const uint32_t at = (u - (own ? second : 0)) * kKeys + lane % kBlocks * 16, len = own ? seen : w.len[0];
        uint32_t page = ~0u;
        if (counted < tile_end && at < len) page = (uint32_t)(own ? w.table[1] : w.table[0])[at >> a.page_shift];
        there = __ballot(page < a.n_pages), whole = __ballot(page < a.n_pages && at + 16 <= len);
        if (page >= a.n_pages) page = 0;
        const uint32_t in_page = at & ((1u << a.page_shift) - 1);
        k_at = reinterpret_cast<uint64_t>(a.k) + kv_head * a.k_head + (uint64_t)page * a.k_page + in_page * a.k_token;
        v_at = reinterpret_cast<uint64_t>(a.v) + kv_head * a.v_head + (uint64_t)page * a.v_page + in_page * a.v_token;
        if constexpr (A::kIn8) {
            k_scale = (uint32_t)a.k_scales[(int64_t)page * a.k_scale_page + (int64_t)(in_page / LSM_SCALE_TOKENS) * a.k_scale_block + (int64_t)kv_head * a.k_scale_head] << 23;
            v_scale = (uint32_t)a.v_scales[(int64_t)page * a.v_scale_page + (int64_t)(in_page / LSM_SCALE_TOKENS) * a.v_scale_block + (int64_t)kv_head * a.v_scale_head] << 23;
        }
        first_tile = t;
    };
    auto first_lane = [&](uint32_t t) { return (kWide ? t - first_tile : (t - first_tile) / kWaves) * kBlocks; };
    // Which keys of tile t there are.
    auto keys_there = [&](uint32_t t) -> uint64_t {
        const uint32_t first = first_lane(t), all = (1u << kBlocks) - 1;
        if (((uint32_t)(whole >> first) & all) == all) return kAllKeys;
        const uint32_t u = place_of(t);
        const bool own = u >= second;
        const uint32_t at = (u - (own ? second : 0)) * kKeys, len = own ? seen : w.len[0], left = at < len ? len - at : 0;
        uint64_t keys = left >= (uint32_t)kKeys ? kAllKeys : (1ull << left) - 1;
#pragma unroll 1
        for (uint32_t i = 0; i < kBlocks; i++)
            if (!((there >> (first + i)) & 1)) keys &= ~(0xFFFFull << (i * 16));
        return keys;
    };
    // A wave copies whole sixteens of rows, or, where there are fewer of these than waves, an equal share of one.  One copy brings rows of one page, so
    // its address is a scalar, and what differs between its lanes does not change from tile to tile.
    constexpr uint32_t kMyBlocks = kWide ? 1 : kBlocks, kCopies = X::kLoads / kMyBlocks, kSharers = kWide ? kWaves / kBlocks : 1;
    static_assert(kMyBlocks * kCopies == X::kLoads && kCopies * kSharers * X::kRowsPerLoad == 16, "");
    uint32_t k_offset[kCopies], v_offset[kCopies];
#pragma unroll
    for (uint32_t j = 0; j < kCopies && !A::kIn8; j++) {
        const uint32_t r = (wave % kSharers * kCopies + j) * X::kRowsPerLoad + lane / X::kWords;
        k_offset[j] = r * a.k_token + X::key_word(r, lane % X::kWords) * 16, v_offset[j] = r * a.v_token + X::value_word(r, lane % X::kWords) * 16;
    }
    auto copy = [&](uint32_t t, uint64_t addresses, const uint32_t (&offset)[kCopies], uint32_t to) {
        const uint32_t first = first_lane(t) + (kWide ? wave / kSharers : 0);
        if (kWide) to += wave * (kCopies * X::kRowsPerLoad * kHead * 2);
#pragma unroll
        for (uint32_t i = 0; i < kMyBlocks; i++) {
            const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)addresses, (int)(first + i));
            const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(addresses >> 32), (int)(first + i));
            const uint64_t from = (uint64_t)hi << 32 | lo;
            const uint32_t at = to + i * 16 * kHead * 2;
            copy_to_lds<0>(from, offset[0], offset[1], at);
            if constexpr (kCopies >= 4) copy_to_lds<2048>(from, offset[2], offset[3], at);
            if constexpr (kCopies >= 8) copy_to_lds<4096>(from, offset[4], offset[5], at), copy_to_lds<6144>(from, offset[6], offset[7], at);
            static_assert(kCopies == 2 || kCopies == 4 || kCopies == 8, "");
        }
    };
    auto copy_keys = [&](uint32_t t, uint32_t to) { copy(t, k_at, k_offset, to); };
    auto copy_values = [&](uint32_t t, uint32_t to) { copy(t, v_at, v_offset, to); };
    // Of 8 bits a row is half as long: a load of 16 bytes a lane brings twice as many rows to registers.  They are converted to dtype there, once for all
    // waves that use them, and written to LDS as the copies of 16 bits would be, so that all that follows is the same.  Every code times a power of two is a number
    // of either type, but for what exceeds its range.
    constexpr uint32_t kRows8 = 2 * X::kRowsPerLoad, kWords8 = X::kWords / 2, kLoads8 = 16 / kRows8;
    static_assert(!A::kIn8 || (kSharers == 1 && kLoads8 >= 1), "");
    typedef uint32_t Word __attribute__((ext_vector_type(4)));
    struct Raw {
        Word word[kMyBlocks][kLoads8 ? kLoads8 : 1];
        uint32_t scale[kMyBlocks];
    };
    // What a lane's loads and stores go by is computed each time: kept in registers it would be spilled.
    auto lane_again = [&]() {
        uint32_t l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };
    auto fetch = [&](uint32_t t, uint64_t addresses, uint32_t scales, uint32_t token_stride, Raw& raw) {
        const uint32_t first = first_lane(t) + (kWide ? wave : 0), l = lane_again(), offset = l / kWords8 * token_stride + l % kWords8 * 16;
#pragma unroll
        for (uint32_t i = 0; i < kMyBlocks; i++) {
            const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)addresses, (int)(first + i));
            const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(addresses >> 32), (int)(first + i));
            raw.scale[i] = (uint32_t)__builtin_amdgcn_readlane((int)scales, (int)(first + i));
            // In global memory: an address that was a number may be any, and loads from any count as LDS operations too, which the waits below are for.
            const auto from = reinterpret_cast<const __attribute__((address_space(1))) char*>((uint64_t)hi << 32 | lo);
#pragma unroll
            for (uint32_t j = 0; j < kLoads8; j++) raw.word[i][j] = *reinterpret_cast<const __attribute__((address_space(1))) Word*>(from + j * kRows8 * token_stride + offset);
        }
    };
    // present: which of the tile's rows there are; zeros in place of the others
    auto put = [&](const Raw& raw, bool keys, uint32_t to, uint64_t present) {
        const uint32_t l = lane_again(), word = l % kWords8;
        if (kWide) to += wave * 16 * kHead * 2;
#pragma unroll
        for (uint32_t i = 0; i < kMyBlocks; i++) {
            const float scale = __uint_as_float(raw.scale[i]);
#pragma unroll
            for (uint32_t j = 0; j < kLoads8; j++) {
                const Word v = raw.word[i][j];
                const uint32_t r = j * kRows8 + l / kWords8;  // of the block; tiles begin with whole blocks, so LDS words are permuted by this number
                x8 lo = Half<kType>::decode8(v.x, v.y, scale), hi = Half<kType>::decode8(v.z, v.w, scale);
                if (present != kAllKeys && !((present >> ((kWide ? wave : i) * 16 + r)) & 1)) lo = x8{}, hi = x8{};  // the scale may be NaN, too
                const uint32_t at = to + i * 16 * kHead * 2 + r * kHead * 2 + (keys ? X::key_word(r, 2 * word) : X::value_word(r, 2 * word)) * 16;
                *reinterpret_cast<x8*>(lds + at) = lo;
                *reinterpret_cast<x8*>(lds + (at ^ 16)) = hi;
            }
        }
    };
    // values of keys that are not there: zeros, whatever the page holds
    auto zero_values = [&](uint64_t present, char* values) {
#pragma unroll 1
        for (uint32_t i = kWide ? threadIdx.x : lane; i < kKeys * X::kWords; i += kTeam * kWave)
            if (!((present >> (i / X::kWords)) & 1)) *reinterpret_cast<uint4*>(values + i * 16) = make_uint4(0, 0, 0, 0);
    };
    // With a window.  The place of a tile's first key among prefix and own tokens; whether a row whose window reaches back to `from` sees all keys of a tile that are
    // not behind it; which keys of a tile this lane's row sees.
    auto first_place = [&](uint32_t t) {
        const uint32_t u = place_of(t);
        return (int32_t)(u < second ? u * kKeys : w.len[0] + (u - second) * kKeys);
    };
    auto window_has = [&](uint32_t t, int32_t from) {
        if constexpr (A::kWindow) {
            const int32_t first = first_place(t);
            return from <= first || a.sinks >= first + kKeys;
        } else return true;
    };
    auto seen_keys = [&](uint32_t t) -> uint64_t {
        if constexpr (A::kWindow) {
            const uint32_t u = place_of(t);
            const int32_t first = first_place(t), limit = u < second ? kKeys : sees - (int32_t)((u - second) * kKeys);
            return first_bits(limit) & (~first_bits(from - first) | first_bits(a.sinks - first));
        } else return 0;
    };
    // A tile's values where some rows of the tile do not see all keys: an infinity or NaN among them would reach these rows too, as its product with a weight
    // of 0.  Such values are added to the rows that see them, and zeros take their places.
    const int32_t fewest_seen = (int32_t)(divide(w.row0, a.share, a.share_part) - w.token0 + w.hidden) + 1;  // of all rows
    auto keep_not_finite = [&](uint32_t t, char* values) {
        const int32_t before = (int32_t)((place_of(t) - second) * kKeys);
        const bool all_behind = place_of(t) < second || fewest_seen >= (int32_t)seen || fewest_seen >= before + kKeys;
        if (all_behind && (!A::kWindow || window_has(t, from_tile))) return;
        constexpr uint32_t kMine = kKeys * X::kWords / (kTeam * kWave);
        uint4* words = reinterpret_cast<uint4*>(values) + (kWide ? threadIdx.x : lane);
        uint32_t any = 0;
#pragma unroll
        for (uint32_t i = 0; i < kMine; i++) {
            const uint4 v = words[i * kTeam * kWave];
            any |= X::not_finite(v.x) | X::not_finite(v.y) | X::not_finite(v.z) | X::not_finite(v.w);
        }
        any = __ballot((any & 0x80008000u) != 0) != 0;
        if (kWide) {
            uint32_t* said = reinterpret_cast<uint32_t*>(lds + S::kLds - 16);
            if (lane == 0) said[wave] = any;
            wait_loads<63>();
            __builtin_amdgcn_s_barrier();
            const uint4 all = *reinterpret_cast<const uint4*>(said);
            any = all.x | all.y | all.z | all.w;
        }
        if (__builtin_amdgcn_readfirstlane((int)any) == 0) return;
        if constexpr (A::kWindow) {
            x.add_not_finite(values, seen_keys(t));
        } else {
            x.add_not_finite(values, sees - before);
        }
        wait_loads<63>();
        if (kWide) __builtin_amdgcn_s_barrier();
        auto finite = [&](uint32_t& two) {
            const uint32_t bits = X::not_finite(two);
            two = (bits & 0x8000u ? 0 : two & 0xFFFFu) | (bits & 0x80000000u ? 0 : two & 0xFFFF0000u);
        };
#pragma unroll 1
        for (uint32_t i = 0; i < kMine; i++) {
            uint4 v = words[i * kTeam * kWave];
            finite(v.x), finite(v.y), finite(v.z), finite(v.w);
            words[i * kTeam * kWave] = v;
        }
        wait_loads<63>();
        if (kWide) __builtin_amdgcn_s_barrier();
    };
    auto scores_masked = [&](uint32_t t, uint64_t present, typename X::Scores& s) {
        const bool own = place_of(t) >= second;
        const int32_t before = (int32_t)((place_of(t) - second) * kKeys);
        if constexpr (A::kWindow) {
            if (present != kAllKeys || (own && least_seen < before + kKeys) || !window_has(t, from_wave)) X::mask_bits(s, present & seen_keys(t));
        } else if (present != kAllKeys || (own && least_seen < before + kKeys)) X::mask(s, present, own ? sees - before : kKeys);
    };
    const uint32_t copies = lds_address(buffers);
    if (t < tile_end) find_pages(t);
    if constexpr (A::kIn8 && kWide) {
        // Buffers as below.  What is asked for lands in registers, and is put into LDS where few others are in use: the keys of two tiles ahead at the top of an
        // iteration, the next tile's values between scores and sums.  (Both at the end spill registers: 8 prompts 1,289 us.)
        if (t < tile_end) {
            Raw raw;
            fetch(t, k_at, k_scale, a.k_token, raw);
            uint64_t present = keys_there(t), present_next = t + 1 < tile_end ? keys_there(t + 1) : 0;
            put(raw, true, 0, kAllKeys);
            fetch(t, v_at, v_scale, a.v_token, raw);
            put(raw, false, 2 * X::kBytes, present);
            if (t + 1 < tile_end) {
                fetch(t + 1, k_at, k_scale, a.k_token, raw);
                put(raw, true, X::kBytes, kAllKeys);
                if (t + 2 < tile_end) fetch(t + 2, k_at, k_scale, a.k_token, raw);
            }
            wait_lds();
            __builtin_amdgcn_s_barrier();
            typename X::Scores s, next;
            typename X::Weights p;
            x.score(buffers, s);
            scores_masked(t, present, s);
            float top = X::largest(s);
            uint32_t buffer = 0;
            for (;;) {
                const char* next_keys = buffers + (buffer ^ X::kBytes);
                char* values = buffers + 2 * X::kBytes + buffer;
                wait_lds();
                __builtin_amdgcn_s_barrier();  // these values and the next keys are there, and everybody is done with these keys and the values before
                const bool more = t + 1 < tile_end;
                uint64_t present_after = 0;
                if (t + 2 < tile_end) put(raw, true, buffer, kAllKeys);
                if (more) fetch(t + 1, v_at, v_scale, a.v_token, raw);
                const float base = x.rebase(top, a.scale);
                keep_not_finite(t, values);
                x.weights_and_score(s, p, a.scale, base, next_keys, next);
                if (more) {
                    scores_masked(t + 1, present_next, next);
                    put(raw, false, 2 * X::kBytes + (buffer ^ X::kBytes), present_next);
                    if (t + 2 < tile_end) {
                        if (first_lane(t + 3) >= kWave) find_pages(t + 2);
                        present_after = keys_there(t + 2);
                        if (t + 3 < tile_end) fetch(t + 3, k_at, k_scale, a.k_token, raw);
                    }
                }
                top = x.template weigh<true>(values, p, next);
                if (!more) break;
                for (uint32_t b = 0; b < X::kGroups; b++) s[b] = next[b];
                t++, buffer ^= X::kBytes, present_next = present_after;
            }
        }
    } else if constexpr (A::kIn8) {
        // One buffer: this tile's keys go there from registers, and the next ones are asked for; likewise the values.  (Two tiles ahead, in as many registers as
        // there are, 96 decodes of up to 8,000 take 107 us for 105.)
        char* keys = buffers;
        char* values = keys + X::kBytes;
        if (t < tile_end) {
            Raw k, v;
            fetch(t, k_at, k_scale, a.k_token, k);
            fetch(t, v_at, v_scale, a.v_token, v);
            for (; t < tile_end; t += step) {
                const uint64_t present = keys_there(t);
                const bool more = t + step < tile_end;
                typename X::Scores s;
                typename X::Weights p;
                put(k, true, wave * 2 * X::kBytes, kAllKeys);
                if (more) {
                    if (first_lane(t + step) >= kWave) find_pages(t + step);
                    fetch(t + step, k_at, k_scale, a.k_token, k);
                }
                wait_lds();
                x.score(keys, s);
                scores_masked(t, present, s);
                x.weights(s, p, a.scale, x.rebase(X::largest(s), a.scale));
                put(v, false, wave * 2 * X::kBytes + X::kBytes, present);
                if (more) fetch(t + step, v_at, v_scale, a.v_token, v);
                wait_lds();
                keep_not_finite(t, values);
                x.template weigh<false>(values, p, s);
                wait_lds();
            }
        }
    } else if (kWide) {
        // Two buffers of keys and two of values.  While a tile's weights are computed the matrix cores are at the next one's scores, so keys are asked
        // for two tiles ahead and values one.  The last tile's next scores are of whatever the buffer holds, and nobody looks at them.
        if (t < tile_end) {
            copy_keys(t, copies);
            copy_values(t, copies + 2 * X::kBytes);
            uint64_t present = keys_there(t), present_next = 0;
            wait_loads<0>();
            __builtin_amdgcn_s_barrier();
            if (t + 1 < tile_end) {
                if (first_lane(t + 1) >= kWave) find_pages(t + 1);
                copy_keys(t + 1, copies + X::kBytes);
                present_next = keys_there(t + 1);
            }
            typename X::Scores s, next;
            typename X::Weights p;
            x.score(buffers, s);
            scores_masked(t, present, s);
            float top = X::largest(s);
            uint32_t buffer = 0;
            for (;;) {
                const char* next_keys = buffers + (buffer ^ X::kBytes);
                char* values = buffers + 2 * X::kBytes + buffer;
                wait_loads<0>();
                __builtin_amdgcn_s_barrier();  // these values and the next keys are there, and everybody is done with these keys and the values before
                const bool more = t + 1 < tile_end;
                uint64_t present_after = 0;
                if (more) {
                    copy_values(t + 1, copies + 2 * X::kBytes + (buffer ^ X::kBytes));
                    if (t + 2 < tile_end) {
                        if (first_lane(t + 2) >= kWave) find_pages(t + 2);
                        copy_keys(t + 2, copies + buffer);
                        present_after = keys_there(t + 2);
                    }
                }
                if (present != kAllKeys) {
                    zero_values(present, values);
                    wait_loads<63>();
                    __builtin_amdgcn_s_barrier();
                }
                const float base = x.rebase(top, a.scale);
                keep_not_finite(t, values);
                x.weights_and_score(s, p, a.scale, base, next_keys, next);
                if (more) scores_masked(t + 1, present_next, next);
                top = x.template weigh<true>(values, p, next);
                if (!more) break;
                for (uint32_t b = 0; b < X::kGroups; b++) s[b] = next[b];
                t++, buffer ^= X::kBytes, present = present_next, present_next = present_after;
            }
        }
    } else {
        // One buffer: the next keys are asked for once the scores are done with these, the next values once the sums are.
        char* keys = buffers;
        char* values = keys + X::kBytes;
        if (t < tile_end) {
            copy_keys(t, copies);
            copy_values(t, copies + X::kBytes);
            for (; t < tile_end; t += step) {
                const uint64_t present = keys_there(t);
                const bool more = t + step < tile_end;
                typename X::Scores s;
                typename X::Weights p;
                wait_loads<X::kLoads>();  // but for the values
                x.score(keys, s);
                wait_loads<63>();
                if (more) {
                    if (first_lane(t + step) >= kWave) find_pages(t + step);
                    copy_keys(t + step, copies);
                }
                scores_masked(t, present, s);
                x.weights(s, p, a.scale, x.rebase(X::largest(s), a.scale));
                if (more) wait_loads<X::kLoads>();  // but for the next keys
                else wait_loads<0>();
                if (present != kAllKeys) zero_values(present, values);
                keep_not_finite(t, values);
                x.template weigh<false>(values, p, s);
                wait_loads<63>();
                if (more) copy_values(t + step, copies + X::kBytes);
            }
        }
    }
    x.sum = other_half_sum(x.sum);
    x.most *= a.scale;

    // Results go through LDS, 64 columns at a time, to be written in whole rows; a narrow tile's waves are joined on the way.
    float* slices = reinterpret_cast<float*>(lds);
    float2* ml = reinterpret_cast<float2*>(lds + kWaves * 32 * S::kSlicePitch * 4);
    float by = 1.f, most = x.most, sum = x.sum;
    __syncthreads();
    if (!kWide) {
        if (h == 0) ml[wave * 32 + n] = make_float2(x.most, x.sum);
        __syncthreads();
        float2 each[kWaves];
        most = -__builtin_inff();
#pragma unroll
        for (uint32_t i = 0; i < kWaves; i++) each[i] = ml[i * 32 + n], most = fmaxf(most, each[i].x);
        const float base = most == -__builtin_inff() ? 0.f : most;
        sum = 0.f;
#pragma unroll
        for (uint32_t i = 0; i < kWaves; i++) sum += each[i].y * __builtin_amdgcn_exp2f(each[i].x - base);
        by = __builtin_amdgcn_exp2f(x.most - base);
    }
    if (!a.joined) by *= sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    if (has_row && h == 0 && (kWide || wave == 0)) {
        if (a.joined) a.part_ml[w.part + row] = make_float2(most, sum);
        else if (a.lse != nullptr) a.lse[(uint64_t)token * a.share * a.kv_heads + head] = sum == 0.f ? -__builtin_inff() : (most + log2f(sum)) * 0.69314718055994531f;
    }
    // eight columns of up to four rows a thread
    constexpr uint32_t kOutRows = (kWide ? kWideRows : kNarrowRows) * 8 / kThreads;
    const uint32_t column = (threadIdx.x & 7) * 8;
    uint64_t place[kOutRows];
#pragma unroll
    for (uint32_t i = 0; i < kOutRows; i++) {
        const uint32_t r = w.row0 + i * (kThreads / 8) + threadIdx.x / 8, tok = divide(r, a.share, a.share_part);
        place[i] = a.joined ? (w.part + r) * kHead + column : (uint64_t)tok * a.out_token + (uint64_t)(kv_head * a.share + (r - tok * a.share)) * a.out_head + column;
    }
#pragma unroll
    for (uint32_t s = 0; s < kHead / 64; s++) {
        if (s) __syncthreads();
#pragma unroll
        for (uint32_t d = 0; d < 2; d++)
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                const f32x16& v = x.acc[s * 2 + d];
                const float4 o = make_float4(v[j * 4] * by, v[j * 4 + 1] * by, v[j * 4 + 2] * by, v[j * 4 + 3] * by);
                *reinterpret_cast<float4*>(slices + (wave * 32 + n) * S::kSlicePitch + d * 32 + j * 8 + h * 4) = o;
            }
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < kOutRows; i++) {
            const uint32_t r = i * (kThreads / 8) + threadIdx.x / 8;
            if (w.row0 + r >= w.row_end) break;
            const float* from = slices + r * S::kSlicePitch + column;
            float4 lo = *reinterpret_cast<const float4*>(from), hi = *reinterpret_cast<const float4*>(from + 4);
            if (!kWide) {
#pragma unroll
                for (uint32_t u = 1; u < kWaves; u++) {
                    const float4 l = *reinterpret_cast<const float4*>(from + u * 32 * S::kSlicePitch), g = *reinterpret_cast<const float4*>(from + u * 32 * S::kSlicePitch + 4);
                    lo.x += l.x, lo.y += l.y, lo.z += l.z, lo.w += l.w, hi.x += g.x, hi.y += g.y, hi.z += g.z, hi.w += g.w;
                }
            }
            if (a.joined) {
                float4* to = reinterpret_cast<float4*>(a.part_out + place[i] + s * 64);
                to[0] = lo, to[1] = hi;
            } else {
                const float o[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                x8 v;
#pragma unroll
                for (int j = 0; j < 8; j++) v[j] = (T)o[j];
                *reinterpret_cast<x8*>(static_cast<T*>(a.out) + place[i] + s * 64) = v;
            }
        }
    }
}

// Owner i of rows [offset(i), offset(i + 1)) has the tiles from offset(i) / (rows of a tile) + i on: at least as many as it needs, at no one else's place.
__device__ __forceinline__ uint32_t tile_of(uint32_t token, uint32_t share, uint32_t rows_log, uint32_t owner) { return (token * share >> rows_log) + owner; }

struct Owner {
    uint32_t index, begin, end, len;  // its number, its tokens, the length of its keys
};
// The owner of a tile: the last one whose first tile is not behind it.  get(i) reads an owner (all of it in one go: a workgroup starts with
// little else to do than to wait for these); every lane of the wave calls.  Up to 64 owners are read at once; of more than that 64 that divide them, then 64 that divide
// those up to the next of these, and so on (one after the other: decodes of 16,384 requests of a few tokens, 8 KV heads 14,070 us for 1,460).
template <typename F>
__device__ __forceinline__ Owner owner_of(uint32_t n, uint32_t first_step, uint32_t tile, uint32_t share, uint32_t rows_log, F get) {
    const uint32_t lane = threadIdx.x & (kWave - 1);
    Owner found = {0, 0, 0, 0};
    for (uint32_t step = first_step;; step /= kWave) {
        const uint32_t i = found.index + lane * step;
        const Owner o = get(i < n ? i : n - 1);
        const int count = __popcll(__ballot(i < n && tile_of(o.begin, share, rows_log, i) <= tile));  // no more than there are such owners: offsets may descend
        if (count == 0) break;
        found.index += (uint32_t)(count - 1) * step;
        if (step > 1) continue;
        found.begin = (uint32_t)__builtin_amdgcn_readlane((int)o.begin, count - 1);
        found.end = (uint32_t)__builtin_amdgcn_readlane((int)o.end, count - 1);
        found.len = (uint32_t)__builtin_amdgcn_readlane((int)o.len, count - 1);
        break;
    }
    return found;
}

// What a launch has: both stages, or the second one alone with tiles of one kind.
enum { kBoth = 0, kNarrowAlone = 1, kWideAlone = 2 };

template <int kType, int kHead, int kStages, typename A>
__global__ void __launch_bounds__(kThreads, kHead == 256 ? 1 : 2) attention_kernel(const A a) {
    __shared__ __attribute__((aligned(16))) char lds[Shape<kType, kHead>::kAllLds];
    // The first stage's items come first: one launch has both run side by side at the seam, and items bound by the matrix cores are not slowed down
    // by others that keep memory busy, as they are where the two take turns.
    const uint32_t stage = kStages != kBoth || blockIdx.x >= a.items0 ? 1 : 0, item = blockIdx.x - (kStages == kBoth && stage ? a.items0 : 0);
    // The rows of a tile change last: workgroups that read the same keys are a multiple of the heads times ranges apart, and so on one die where that
    // is a multiple of eight (8 KV heads); where it is not (2 KV heads, 5 ranges), several dies read them (256 decodes: 465 MB fetched, 319 due).
    const uint32_t combos = stage ? a.combos[1] : a.combos[0], tile = divide(item, combos, stage ? a.combos_part[1] : a.combos_part[0]), combo = item - tile * combos;
    if (tile >= (stage ? a.tiles[1] : a.tiles[0])) return;
    uint32_t split = 0, kv_head = combo;
    while (kv_head >= a.kv_heads) kv_head -= a.kv_heads, split++;  // at most 64 times
    const bool wide = kStages == kBoth ? (stage ? a.wide[1] : a.wide[0]) != 0 : kStages == kWideAlone;
    const uint32_t rows_log = wide ? 7 : 5, tile_rows = 1u << rows_log;
    static_assert(kWideRows == 128 && kNarrowRows == 32, "");
    Item w;
    Owner o;
    if (stage == 0) {
        o = owner_of(a.n_groups, a.search[0], tile, a.share, rows_log, [&](uint32_t g) {
            const int32_t r0 = a.group_offsets[g], r1 = a.group_offsets[g + 1], len = a.prefix_lens[g];
            return Owner{g, token_of_request(a, clamp_u32(r0, a.n_requests)), token_of_request(a, clamp_u32(r1, a.n_requests)), clamp_u32(len, a.prefix_width << a.page_shift)};
        });
        w.table[0] = a.prefix_tables + o.index * a.prefix_width, w.len[0] = o.len;
        w.table[1] = nullptr, w.len[1] = 0;
    } else {
        const uint32_t lane = threadIdx.x & (kWave - 1);
        int32_t group_first = 0, group_len = 0;  // of the first 64 groups: read along with the requests
        const bool prefixed = kStages != kBoth && a.prefix_width != 0;
        if (prefixed) group_first = a.group_offsets[lane < a.n_groups ? lane : a.n_groups], group_len = a.prefix_lens[lane < a.n_groups ? lane : 0];
        o = owner_of(a.n_requests, a.search[1], tile, a.share, rows_log, [&](uint32_t r) {
            const int32_t t0 = a.q_offsets[r], t1 = a.q_offsets[r + 1], len = a.own_lens[r];
            return Owner{r, clamp_u32(t0, a.n_tokens), clamp_u32(t1, a.n_tokens), clamp_u32(len, a.own_width << a.page_shift)};
        });
        w.len[0] = 0, w.table[0] = nullptr;
        if (prefixed) {
            const int count = __popcll(__ballot(lane < a.n_groups && clamp_u32(group_first, a.n_requests) <= o.index));
            uint32_t g = count > 0 ? count - 1 : 0;
            w.len[0] = clamp_u32(__builtin_amdgcn_readlane(group_len, (int)g), a.prefix_width << a.page_shift);
            if (count == (int)kWave && a.n_groups > kWave) g = group_of(a, o.index), w.len[0] = prefix_len(a, g);
            w.table[0] = a.prefix_tables + g * a.prefix_width;
        }
        w.table[1] = a.own_tables + o.index * a.own_width, w.len[1] = o.len;
    }
    const uint32_t order = tile - tile_of(o.begin, a.share, rows_log, o.index), owned = ((o.end - o.begin) * a.share + tile_rows - 1) >> rows_log;
    if (o.end <= o.begin || order >= owned) return;
    // The last rows, which see most keys, first: what runs on alone at the end is short (a prompt of 2,048 tokens, 32 heads: 59 -> 54 us; 8 of them behind
    // 4,096: 1,392 -> 1,346).
    const uint32_t in_owner = owned - 1 - order;
    w.row0 = o.begin * a.share + in_owner * tile_rows;
    w.row_end = o.end * a.share;
    w.token0 = o.begin;
    w.hidden = w.len[1] - (o.end - o.begin);
    uint32_t units = units_of(w.len[0]) + units_of(w.len[1]);
    if constexpr (A::kWindow) {
        // units that the window of the tile's first token reaches, which goes back furthest, and the first tokens' before them
        const int32_t from = (int32_t)(w.len[0] + divide(w.row0, a.share, a.share_part) - w.token0 + w.hidden) + 1 - a.window;
        auto unit_of = [&](uint32_t place) { return place < w.len[0] ? place / kSplitKeys : units_of(w.len[0]) + (place - w.len[0]) / kSplitKeys; };
        w.window_unit = from <= 0 ? 0 : min(unit_of((uint32_t)from), units);
        const uint32_t sinks = min((uint32_t)a.sinks, w.len[0] + w.len[1]);
        w.sink_units = sinks == 0 ? 0 : min(unit_of(sinks - 1) + 1, w.window_unit);
        units -= w.window_unit - w.sink_units;
    }
    const uint32_t each = split_units(units, stage ? a.splits[1] : a.splits[0], stage ? a.least[1] : a.least[0]);
    w.unit0 = split * each, w.unit1 = w.unit0 + each < units ? w.unit0 + each : units;
    w.part = ((uint64_t)((stage ? a.splits[0] : 0) + split) * a.kv_heads + kv_head) * a.rows;
    if (a.joined && w.unit0 >= units) {  // not one of the ranges that there are
        if (threadIdx.x < tile_rows && w.row0 + threadIdx.x < w.row_end) a.part_ml[w.part + w.row0 + threadIdx.x] = make_float2(-__builtin_inff(), kNoPart);
        return;
    }
    if (wide) attend<kType, kHead, true>(a, w, kv_head, lds);
    else attend<kType, kHead, false>(a, w, kv_head, lds);
}

// ---------------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------------
static inline bool aligned_rows(const void* data, int64_t s0, int64_t s1, int64_t s2, int64_t bytes = 2) {
    return ((reinterpret_cast<uint64_t>(data) | (uint64_t)(s0 * bytes) | (uint64_t)(s1 * bytes) | (uint64_t)(s2 * bytes)) & 15) == 0;
}

constexpr float kLog2E = 1.44269504088896341f;  // scores are scaled by this too: weights are powers of two

static inline int check_attention(const lsm_attention_t* a, int64_t page_bytes = 2) {  // bytes of an element of the pages
    if (a == nullptr) return LSM_ERR_NULL;
    if (a->dtype != LSM_BF16 && a->dtype != LSM_FP16) return LSM_ERR_BAD_ARG;
    if (a->head_dim != 64 && a->head_dim != 128 && a->head_dim != 256) return LSM_ERR_BAD_ARG;
    if (a->page_tokens < LSM_MIN_PAGE_TOKENS || a->page_tokens > LSM_MAX_PAGE_TOKENS || (a->page_tokens & (a->page_tokens - 1)) != 0) return LSM_ERR_BAD_ARG;
    if (a->kv_heads == 0 || a->q.heads == 0 || a->q.heads != a->out.heads || a->q.heads % a->kv_heads != 0 || a->q.heads > 4096) return LSM_ERR_BAD_ARG;
    if (a->n_tokens >= 1u << 24 || a->n_tokens * a->q.heads >= 1ull << 31 || a->n_requests >= 1u << 24 || a->n_groups >= 1u << 24 || a->n_pages >= 1ull << 31) return LSM_ERR_BAD_ARG;
    if (a->prefix_width * a->page_tokens >= 1ull << 30 || a->own_width * a->page_tokens >= 1ull << 30 || a->prefix_width >= 1u << 30 || a->own_width >= 1u << 30) return LSM_ERR_BAD_ARG;
    if (a->reserved != 0 || !(a->scale > 0.f) || !(a->scale * kLog2E < __builtin_inff())) return LSM_ERR_BAD_ARG;
    if (a->n_tokens == 0) return LSM_OK;
    if (a->n_requests == 0) return LSM_ERR_BAD_ARG;
    if (a->q.data == nullptr || a->out.data == nullptr || a->q_offsets == nullptr || a->own_lens == nullptr) return LSM_ERR_NULL;
    if (a->own_width != 0 && a->own_tables == nullptr) return LSM_ERR_NULL;
    if (a->prefix_width != 0 && a->n_groups != 0 && (a->prefix_tables == nullptr || a->prefix_lens == nullptr || a->group_offsets == nullptr)) return LSM_ERR_NULL;
    if (a->n_pages != 0 && (a->k_pages.data == nullptr || a->v_pages.data == nullptr)) return LSM_ERR_NULL;
    if (!aligned_rows(a->q.data, a->q.token_stride, a->q.head_stride, 0) || !aligned_rows(a->out.data, a->out.token_stride, a->out.head_stride, 0) ||
        !aligned_rows(a->k_pages.data, a->k_pages.page_stride, a->k_pages.token_stride, a->k_pages.head_stride, page_bytes) ||
        !aligned_rows(a->v_pages.data, a->v_pages.page_stride, a->v_pages.token_stride, a->v_pages.head_stride, page_bytes)) return LSM_ERR_BAD_ARG;
    // the kernel has strides in bytes in 32 bits, and offsets inside a page too
    for (const lsm_pages_t* p : {&a->k_pages, &a->v_pages})
        if (p->page_stride < 0 || p->token_stride < 0 || p->head_stride < 0 || p->page_stride >= 1ll << 31 || p->token_stride >= 1 << 22) return LSM_ERR_BAD_ARG;
    const uint64_t words = reinterpret_cast<uint64_t>(a->lse) | reinterpret_cast<uint64_t>(a->group_offsets) | reinterpret_cast<uint64_t>(a->prefix_tables) |
                           reinterpret_cast<uint64_t>(a->prefix_lens) | reinterpret_cast<uint64_t>(a->q_offsets) | reinterpret_cast<uint64_t>(a->own_tables) |
                           reinterpret_cast<uint64_t>(a->own_lens);
    return words & 3 ? LSM_ERR_BAD_ARG : LSM_OK;
}

// How the work is cut; from sizes that the host knows (widths of tables stand for lengths).
// page_bytes: of an element of the pages; most_seen: of the keys of a request that any one tile of rows works on, where a window limits them.
static inline void plan_attention(const lsm_attention_t* a, AttentionArgs& p, uint64_t page_bytes = 2, uint64_t most_seen = ~0ull) {
    const uint64_t share = a->q.heads / a->kv_heads, rows = a->n_tokens * share;
    const uint64_t groups = a->prefix_width != 0 ? a->n_groups : 0;
    const uint64_t own_keys = a->own_width * a->page_tokens, prefix_keys = groups ? a->prefix_width * a->page_tokens : 0;
    p.share = (uint32_t)share, p.rows = (uint32_t)rows, p.kv_heads = (uint32_t)a->kv_heads;
    // One pass over prefix and own pages for each request, where nothing is shared or a request's rows fill tiles of 128 by themselves, and where
    // reading prefixes again and again is no more than 64 MB out of caches: two passes and the join of their parts cost more then (32 decodes behind
    // 4 prefixes of 1,500, 2 KV heads: 13.8 us so and 15.7 in two stages; 200 behind 4,000, 4 KV heads, 1.7 GB: 86 and 45).
    p.whole = groups == 0 || groups >= a->n_requests || rows / a->n_requests >= 300 || most_seen != ~0ull ||
              a->n_requests * a->kv_heads * (prefix_keys + own_keys) * a->head_dim * 2 * page_bytes <= 64ull << 20;
    for (int s = 0; s < 2; s++) {
        p.tiles[s] = 0, p.splits[s] = 0, p.wide[s] = 0, p.least[s] = 1;
        if (s == 0 && p.whole) continue;
        const uint64_t owners = s == 0 ? groups : a->n_requests, all_keys = s == 0 ? prefix_keys : own_keys + (p.whole ? prefix_keys : 0), keys = all_keys < most_seen ? all_keys : most_seen;
        p.wide[s] = rows / owners > 48;
        const uint64_t tile_rows = p.wide[s] ? kWideRows : kNarrowRows;
        p.tiles[s] = (uint32_t)(rows / tile_rows + owners);
        const uint64_t items = (rows / tile_rows > owners ? rows / tile_rows : owners) * a->kv_heads;  // about so many tiles have rows
        // Ranges of keys: enough for a workgroup on each compute unit (wide tiles; more of them write more parts: 200 decodes behind 4,000
        // 39.5 us with 256, 48 with 512), or two (narrow ones); narrow prefix tiles, whose time is the start and the end, 160 (64 decodes behind 8: 27.1, with 512 30).
        uint64_t splits = (p.wide[s] ? 256 : s == 1 ? 512 : 160) / items;
        p.least[s] = p.wide[s] ? 2 : 4;
        if (p.whole && !p.wide[s]) {
            // a short pass is over before its parts could be joined (4 decodes behind 512: 9.6 us in one range, 11.4 in five)
            if (keys <= 1024) splits = 1;
            // many ragged requests: ranges of about 1,024 keys each, so that the longest does not run on alone (96 of up to 8,000: 169 us, 204 uncut)
            else if (page_bytes == 2 && most_seen == ~0ull && items * splits >= 300 && keys > 2048) p.least[s] = 1024 / kSplitKeys, splits = keys / 1024;
            else if ((page_bytes != 2 || most_seen != ~0ull) && keys > 2048) {
                // Of 8 bits, or with a window: ranges of such a length that there are up to 768 where all requests are as long as the tables are wide, of 256 to
                // 1,024 keys (2,048 of 8 bits: as many bytes), whole tiles for all waves.  Requests of up to 8,000 tokens in 8 bits, by this rule / by the one above:
                // 1 of 2 KV heads 16 / 35 us, 16 of 2 heads 20 / 36, 16 of 8 heads 41 / 51, 48 of 2 heads 40 / 45, 96 of 4 heads 105 / 110.
                const uint64_t range = (items * keys / 768 + 255) / 256 * 256, longest = 2048 / page_bytes;
                p.least[s] = (uint32_t)((range < 256 ? 256 : range > longest ? longest : range) / kSplitKeys), splits = keys / (p.least[s] * kSplitKeys);
            }
        }
        const uint64_t most = keys / (p.least[s] * kSplitKeys);
        // A first stage with long ranges: 256 workgroups or a few more leave some compute units with two and the others with one, so more of them, and the
        // fewer the longer the second stage is (at 5 TB/s beside 1 PFLOP/s), which shares the compute units with them.  256 decodes behind 8,192 and
        // 16,384, 2 KV heads: 15 own tokens each 119 -> 90 us, 1,024 each 117 -> 93 with 410 of them; 2,047 each 127 with 256 or 410, 120 with 340.
        // Behind 4,096 and 8,192 with 2,047 each: 93 with 256, 101 with 340.  Own keys count as 16 bits in 8 too: by their bytes the first batch with 2,047 each would
        // have 410, 116 us for 113.
        if (s == 0 && p.wide[0]) {
            const bool alone = a->n_requests * own_keys * 200 < rows * prefix_keys;
            const uint64_t more = (alone ? 410 : 340) / (p.tiles[0] * a->kv_heads);
            if (more > splits && prefix_keys / more >= (alone ? 1024 : 2048)) splits = more;
        }
        if (splits > most) splits = most;
        if (splits > 64) splits = 64;
        p.splits[s] = splits > 1 ? (uint32_t)splits : 1;
    }
    p.share_part = part_of((uint32_t)share);
    for (int s = 0; s < 2; s++) {
        p.combos[s] = p.splits[s] * p.kv_heads, p.combos_part[s] = part_of(p.combos[s] ? p.combos[s] : 1);
    }
    p.items0 = p.tiles[0] * p.combos[0];
    p.joined = !(p.whole && p.splits[1] == 1);
}

// A launch has fewer than 2^32 threads; one of more is cut without an error.
static inline uint64_t join_blocks(const lsm_attention_t* a) {
    const uint64_t per_block = kWaves * kWave * 4 / a->head_dim;
    return (a->n_tokens * a->q.heads + per_block - 1) / per_block;
}
static inline bool fits_launches(const lsm_attention_t* a, const AttentionArgs& p) {
    constexpr uint64_t kMost = (1ull << 32) / kThreads - 1;
    return ((uint64_t)p.tiles[0] * p.splits[0] + (uint64_t)p.tiles[1] * p.splits[1]) * p.kv_heads <= kMost && (!p.joined || join_blocks(a) <= kMost);
}

static inline size_t part_bytes(const lsm_attention_t* a, const AttentionArgs& p) {
    if (!p.joined) return 0;
    return (size_t)(p.splits[0] + p.splits[1]) * a->n_tokens * a->q.heads * (a->head_dim * 4 + 8);
}

// What the kernels need to know besides the plan.
static inline void set_attention(const lsm_attention_t* a, AttentionArgs& p, void* workspace, uint64_t page_bytes = 2) {
    p.q = a->q.data, p.out = a->out.data, p.lse = a->lse, p.k = a->k_pages.data, p.v = a->v_pages.data;
    p.q_token = a->q.token_stride, p.q_head = a->q.head_stride, p.out_token = a->out.token_stride, p.out_head = a->out.head_stride;
    p.k_page = (uint32_t)a->k_pages.page_stride * (uint32_t)page_bytes, p.k_token = (uint32_t)a->k_pages.token_stride * (uint32_t)page_bytes, p.k_head = (uint64_t)a->k_pages.head_stride * page_bytes;
    p.v_page = (uint32_t)a->v_pages.page_stride * (uint32_t)page_bytes, p.v_token = (uint32_t)a->v_pages.token_stride * (uint32_t)page_bytes, p.v_head = (uint64_t)a->v_pages.head_stride * page_bytes;
    p.group_offsets = a->group_offsets, p.prefix_tables = a->prefix_tables, p.prefix_lens = a->prefix_lens;
    p.q_offsets = a->q_offsets, p.own_tables = a->own_tables, p.own_lens = a->own_lens;
    p.n_tokens = (uint32_t)a->n_tokens, p.n_requests = (uint32_t)a->n_requests, p.n_groups = (uint32_t)a->n_groups, p.n_pages = (uint32_t)a->n_pages;
    p.search[0] = search_step(a->n_groups), p.search[1] = search_step(a->n_requests);
    p.page_shift = (uint32_t)__builtin_ctzll(a->page_tokens);
    p.prefix_width = a->n_groups ? a->prefix_width : 0, p.own_width = a->own_width;
    p.scale = a->scale * kLog2E;
    p.part_out = static_cast<float*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + (size_t)(p.splits[0] + p.splits[1]) * a->n_tokens * a->q.heads * a->head_dim * 4);
}

// Joins the parts that an attention kernel left, if it did (p.joined).
void launch_join(const AttentionArgs& p, uint32_t dtype, uint32_t head, uint32_t joins, hipStream_t stream);

}  // namespace lsm
