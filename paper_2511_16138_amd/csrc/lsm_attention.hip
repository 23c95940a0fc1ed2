// lsm_prefix_attention: attention over a paged cache for batches whose requests share long prefixes.
//
// A row is one query head of one new token.  Rows of a KV head that see the same keys are packed into tiles, whatever request they
// belong to: behind a shared prefix these are the rows of the whole group, behind a request's own pages those of the request.
// A workgroup takes a tile of rows and a range of keys and goes over the keys once with a running maximum and sum; where a tile's
// keys are dealt to several workgroups (the prefix and the own pages always are, unless rows are packed by request anyway), each
// leaves its accumulator, maximum and sum, and a second kernel joins them in a fixed order.
//
// Measured, with the floor of bytes at a copy's 4.94 TB/s or of operations at a library product's 1.38 PFLOP/s:
//   96 decodes of up to 8,000 keys, 4 KV heads of 128     180 us, 4.9 TB/s     (178: memory)
//   64 decodes behind 8 prefixes of 512 - 1,536, 8 heads    30 us, 3.2 TB/s     (19: memory, then the way in and the join)
//   256 decodes behind 8,192 and 16,384, 2 heads           126 us, 0.53 PFLOP/s (65: the matrix cores on the prefixes, then memory on the own pages)
//   8 prompts of 1,024 - 2,048 behind 1,536 - 4,096        920 - 950 us, 1.01 PFLOP/s (686: matrix cores 51 % busy at 1.7 GHz, the softmax's vector instructions as long)
// The weights of the softmax are rounded to 16 bits for the second product, which the matrix cores take no other operands for at this rate; with that the
// error against 64 bits is 1.4 times that of a computation in 32 bits rounded once at the end (2.3e-3 and 1.7e-3 in bf16, 2.8e-4 and 2.1e-4 in fp16).
// In fp16, weights under 2^-14 lose bits as subnormals and those under 2^-25 are 0 in the product, though not in the sum: many keys that far below the
// maximum count for less (or more) than they should, by at most their number times 2^-25.
#include <hip/hip_runtime.h>

#include "lsm_cache.h"
#include "lsm_common.h"

namespace lsm {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int kType>
struct Half;
template <>
struct Half<LSM_BF16> {
    typedef __bf16 type;
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    static constexpr uint32_t kExponent = 0x7F80;
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Half<LSM_FP16> {
    typedef _Float16 type;
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    static constexpr uint32_t kExponent = 0x7C00;
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

constexpr uint32_t kThreads = 256, kWaves = kThreads / kWave;
constexpr uint32_t kWaveRows = 32;                      // rows of a wave: the columns of one product
constexpr uint32_t kWideRows = kWaveRows * kWaves;      // a wide tile: each wave has rows of its own, all go over the same keys
constexpr uint32_t kNarrowRows = kWaveRows;             // a narrow tile: all waves have the same rows, each goes over keys of its own
constexpr uint32_t kSplitKeys = 64;                     // ranges of keys are whole numbers of this

struct AttentionArgs {
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
    uint32_t joined;  // the parts are joined by another kernel
    float* part_out;  // [split of either stage][KV head][row][head_dim]
    float2* part_ml;  // [split of either stage][KV head][row]: maximum in units of the exponent of two, sum; kNoPart = there is no part
};
constexpr float kNoPart = -1.f;  // no sum of weights

// x / d for x < 2^31, given part_of(d): a division takes forty instructions, and a workgroup's first pass over its instructions is most of a short call.
inline uint32_t part_of(uint32_t d) { return 0xFFFFFFFFu / d; }
__device__ __forceinline__ uint32_t divide(uint32_t x, uint32_t d, uint32_t part) {
    const uint32_t q = __umulhi(x, part);  // or one too small
    return x - q * d >= d ? q + 1 : q;
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

// The last i < n with start(i) <= x, for start(0) <= x and start not descending; every lane of the wave calls and gets it.
template <typename F>
__device__ __forceinline__ uint32_t last_not_above(uint32_t n, uint64_t x, F start) {
    const uint32_t lane = threadIdx.x & (kWave - 1);
    uint32_t count = 0;
    for (uint32_t base = 0; base < n; base += kWave) {
        const uint32_t i = base + lane;
        const uint64_t ok = __ballot(i < n && start(i) <= x);
        count += (uint32_t)__popcll(ok);
        if (ok != ~0ull) break;
    }
    return count > 0 ? count - 1 : 0;
}
__device__ __forceinline__ uint32_t group_of(const AttentionArgs& a, uint32_t request) {
    return last_not_above(a.n_groups, request, [&](uint32_t g) { return (uint64_t)clamp_u32(a.group_offsets[g], a.n_requests); });
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
    // limit: how many of the tile's keys this lane's row sees.
    __device__ __forceinline__ void add_not_finite(const char* values, int32_t limit) {
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
                    if ((int32_t)row < limit && ((bits[j / 2] >> (j % 2 * 16 + 15)) & 1)) acc[i / 4][i % 4 * 4 + j] += (float)v.one[j];
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

template <int kType, int kHead, bool kWide>
__device__ __forceinline__ void attend(const AttentionArgs& a, const Item& w, uint32_t kv_head, char* lds) {
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
    const uint32_t units = a.n_pages == 0 ? 0 : units0 + units_of(seen);
    const uint32_t unit1 = w.unit1 < units ? w.unit1 : units;
    const uint32_t tile_end = unit1 * kPerUnit, step = kWide ? 1 : kWaves, second = units0 * kPerUnit;  // tiles from `second` on are of the second segment
    uint32_t t = w.unit0 * kPerUnit + (kWide ? 0 : wave);

    // Where the next tiles' tokens are, 16 of them a lane: addresses of keys and of values, and `there`: which of them have a page.  One load for 64 of these, and
    // no vector memory operations but the copies in between, which the waits below count.  Where there is no page any does: the scores of
    // keys that are not there are masked, and their values are zeroed in LDS.
    constexpr uint32_t kBlocks = kKeys / 16;  // lanes of a tile
    uint64_t k_at = 0, v_at = 0, there = 0, whole = 0;  // whole: which have a page and 16 tokens
    uint32_t first_tile = 0;                            // of lane 0
    auto find_pages = [&](uint32_t t) {
        const uint32_t u = t + lane / kBlocks * step;
        const bool own = u >= second;
        const uint32_t at = (u - (own ? second : 0)) * kKeys + lane % kBlocks * 16, len = own ? seen : w.len[0];
        uint32_t page = ~0u;
        if (u < tile_end && at < len) page = (uint32_t)(own ? w.table[1] : w.table[0])[at >> a.page_shift];
        there = __ballot(page < a.n_pages), whole = __ballot(page < a.n_pages && at + 16 <= len);
        if (page >= a.n_pages) page = 0;
        const uint32_t in_page = at & ((1u << a.page_shift) - 1);
        k_at = reinterpret_cast<uint64_t>(a.k) + kv_head * a.k_head + (uint64_t)page * a.k_page + in_page * a.k_token;
        v_at = reinterpret_cast<uint64_t>(a.v) + kv_head * a.v_head + (uint64_t)page * a.v_page + in_page * a.v_token;
        first_tile = t;
    };
    auto first_lane = [&](uint32_t t) { return (kWide ? t - first_tile : (t - first_tile) / kWaves) * kBlocks; };
    // Which keys of tile t there are.
    auto keys_there = [&](uint32_t t) -> uint64_t {
        const uint32_t first = first_lane(t), all = (1u << kBlocks) - 1;
        if (((uint32_t)(whole >> first) & all) == all) return kAllKeys;
        const bool own = t >= second;
        const uint32_t at = (t - (own ? second : 0)) * kKeys, len = own ? seen : w.len[0], left = at < len ? len - at : 0;
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
    for (uint32_t j = 0; j < kCopies; j++) {
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
    // values of keys that are not there: zeros, whatever the page holds
    auto zero_values = [&](uint64_t present, char* values) {
#pragma unroll 1
        for (uint32_t i = kWide ? threadIdx.x : lane; i < kKeys * X::kWords; i += kTeam * kWave)
            if (!((present >> (i / X::kWords)) & 1)) *reinterpret_cast<uint4*>(values + i * 16) = make_uint4(0, 0, 0, 0);
    };
    // A tile's values where some rows of the tile do not see all keys: an infinity or NaN among them would reach these rows too, as its product with a weight
    // of 0.  Such values are added to the rows that see them, and zeros take their places.
    const int32_t fewest_seen = (int32_t)(divide(w.row0, a.share, a.share_part) - w.token0 + w.hidden) + 1;  // of all rows
    auto keep_not_finite = [&](uint32_t t, char* values) {
        const int32_t before = (int32_t)((t - second) * kKeys);
        if (t < second || fewest_seen >= (int32_t)seen || fewest_seen >= before + kKeys) return;
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
        x.add_not_finite(values, sees - before);
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
        const bool own = t >= second;
        const int32_t before = (int32_t)((t - second) * kKeys);
        if (present != kAllKeys || (own && least_seen < before + kKeys)) X::mask(s, present, own ? sees - before : kKeys);
    };
    const uint32_t copies = lds_address(buffers);
    if (t < tile_end) find_pages(t);
    if (kWide) {
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
// little else to do than to wait for these); every lane of the wave calls.
template <typename F>
__device__ __forceinline__ Owner owner_of(uint32_t n, uint32_t tile, uint32_t share, uint32_t rows_log, F get) {
    const uint32_t lane = threadIdx.x & (kWave - 1);
    Owner found = {0, 0, 0, 0};
    for (uint32_t base = 0; base < n; base += kWave) {
        const uint32_t i = base + lane;
        const Owner o = get(i < n ? i : n - 1);
        const uint64_t ok = __ballot(i < n && tile_of(o.begin, share, rows_log, i) <= tile);
        const int count = __popcll(ok);
        if (count == 0) break;
        found.index = base + count - 1;
        found.begin = (uint32_t)__builtin_amdgcn_readlane((int)o.begin, count - 1);
        found.end = (uint32_t)__builtin_amdgcn_readlane((int)o.end, count - 1);
        found.len = (uint32_t)__builtin_amdgcn_readlane((int)o.len, count - 1);
        if (count < (int)kWave) break;
    }
    return found;
}

// What a launch has: both stages, or the second one alone with tiles of one kind.
enum { kBoth = 0, kNarrowAlone = 1, kWideAlone = 2 };

template <int kType, int kHead, int kStages>
__global__ void __launch_bounds__(kThreads, kHead == 256 ? 1 : 2) attention_kernel(const AttentionArgs a) {
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
        o = owner_of(a.n_groups, tile, a.share, rows_log, [&](uint32_t g) {
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
        o = owner_of(a.n_requests, tile, a.share, rows_log, [&](uint32_t r) {
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
    const uint32_t units = units_of(w.len[0]) + units_of(w.len[1]), each = split_units(units, stage ? a.splits[1] : a.splits[0], stage ? a.least[1] : a.least[0]);
    w.unit0 = split * each, w.unit1 = w.unit0 + each < units ? w.unit0 + each : units;
    w.part = ((uint64_t)((stage ? a.splits[0] : 0) + split) * a.kv_heads + kv_head) * a.rows;
    if (a.joined && w.unit0 >= units) {  // not one of the ranges that there are
        if (threadIdx.x < tile_rows && w.row0 + threadIdx.x < w.row_end) a.part_ml[w.part + w.row0 + threadIdx.x] = make_float2(-__builtin_inff(), kNoPart);
        return;
    }
    if (wide) attend<kType, kHead, true>(a, w, kv_head, lds);
    else attend<kType, kHead, false>(a, w, kv_head, lds);
}

// Joins a row's parts in the order of their numbers.  kHead / 4 lanes have a row; first each has the maxima and sums of some of its parts (at most 128 in
// all), then four columns of all of them.  A part whose weight is 0 is added like any other: it may hold an infinity or NaN, which a seen value put there.
template <int kType, int kHead>
__global__ void __launch_bounds__(kThreads) join_kernel(const AttentionArgs a) {
    typedef typename Half<kType>::type T;
    typedef T x4 __attribute__((ext_vector_type(4)));
    constexpr uint32_t kLanes = kHead / 4, kRows = kWave / kLanes, kMine = 128 / kLanes;  // lanes of a row, rows of a wave, parts of a lane
    const uint32_t lane = threadIdx.x & (kWave - 1), in_row = lane % kLanes, parts = a.splits[0] + a.splits[1];
    const uint64_t all = (uint64_t)a.rows * a.kv_heads;  // rows of a part, those of the first KV head first
    uint64_t at = ((uint64_t)blockIdx.x * kWaves + threadIdx.x / kWave) * kRows + lane / kLanes;
    const bool mine = at < all;
    if (!mine) at = all - 1;
    float2 ml[kMine];
    float most = -__builtin_inff();
#pragma unroll
    for (uint32_t i = 0; i < kMine; i++) {
        ml[i] = make_float2(-__builtin_inff(), kNoPart);
        if (i * kLanes + in_row < parts) ml[i] = a.part_ml[(i * kLanes + in_row) * all + at];
        most = fmaxf(most, ml[i].x);
    }
#pragma unroll
    for (uint32_t off = 1; off < kLanes; off <<= 1) most = fmaxf(most, __shfl_xor(most, (int)off, kWave));
    const float base = most == -__builtin_inff() ? 0.f : most;
    float sum = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < kMine; i++) {
        const bool none = ml[i].y == kNoPart;
        ml[i].x = none ? kNoPart : __builtin_amdgcn_exp2f(ml[i].x - base);
        if (!none) sum += ml[i].y * ml[i].x;
    }
#pragma unroll
    for (uint32_t off = 1; off < kLanes; off <<= 1) sum += __shfl_xor(sum, (int)off, kWave);
    const float* from = a.part_out + at * kHead + in_row * 4;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (uint32_t i = 0; i < kMine; i++) {
        if (i * kLanes >= parts) break;
        const uint32_t left = parts - i * kLanes < kLanes ? parts - i * kLanes : kLanes;
#pragma unroll 1
        for (uint32_t j = 0; j < left; j += 4) {
            float4 v[4];
            float by[4];
#pragma unroll
            for (uint32_t u = 0; u < 4; u++) {
                by[u] = j + u < left ? __shfl(ml[i].x, (int)(lane - in_row + j + u), kWave) : kNoPart;
                v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (by[u] != kNoPart) v[u] = *reinterpret_cast<const float4*>(from + (i * kLanes + j + u) * all * kHead);
            }
#pragma unroll
            for (uint32_t u = 0; u < 4; u++) o.x += v[u].x * by[u], o.y += v[u].y * by[u], o.z += v[u].z * by[u], o.w += v[u].w * by[u];
        }
    }
    if (!mine) return;
    const uint32_t kv_head = (uint32_t)at / a.rows, row = (uint32_t)at - kv_head * a.rows, token = divide(row, a.share, a.share_part), head = kv_head * a.share + (row - token * a.share);
    const float by = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    x4 r;
    r[0] = (T)(o.x * by), r[1] = (T)(o.y * by), r[2] = (T)(o.z * by), r[3] = (T)(o.w * by);
    *reinterpret_cast<x4*>(static_cast<T*>(a.out) + (int64_t)token * a.out_token + (int64_t)head * a.out_head + in_row * 4) = r;
    if (a.lse != nullptr && in_row == 0) a.lse[(uint64_t)token * a.share * a.kv_heads + head] = sum == 0.f ? -__builtin_inff() : (most + log2f(sum)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------------
static bool aligned_rows(const void* data, int64_t s0, int64_t s1, int64_t s2) {
    return ((reinterpret_cast<uint64_t>(data) | (uint64_t)(s0 * 2) | (uint64_t)(s1 * 2) | (uint64_t)(s2 * 2)) & 15) == 0;
}

constexpr float kLog2E = 1.44269504088896341f;  // scores are scaled by this too: weights are powers of two

static int check_attention(const lsm_attention_t* a) {
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
        !aligned_rows(a->k_pages.data, a->k_pages.page_stride, a->k_pages.token_stride, a->k_pages.head_stride) ||
        !aligned_rows(a->v_pages.data, a->v_pages.page_stride, a->v_pages.token_stride, a->v_pages.head_stride)) return LSM_ERR_BAD_ARG;
    // the kernel has strides in bytes in 32 bits, and offsets inside a page too
    for (const lsm_pages_t* p : {&a->k_pages, &a->v_pages})
        if (p->page_stride < 0 || p->token_stride < 0 || p->head_stride < 0 || p->page_stride >= 1ll << 31 || p->token_stride >= 1 << 22) return LSM_ERR_BAD_ARG;
    const uint64_t words = reinterpret_cast<uint64_t>(a->lse) | reinterpret_cast<uint64_t>(a->group_offsets) | reinterpret_cast<uint64_t>(a->prefix_tables) |
                           reinterpret_cast<uint64_t>(a->prefix_lens) | reinterpret_cast<uint64_t>(a->q_offsets) | reinterpret_cast<uint64_t>(a->own_tables) |
                           reinterpret_cast<uint64_t>(a->own_lens);
    return words & 3 ? LSM_ERR_BAD_ARG : LSM_OK;
}

// How the work is cut; from sizes that the host knows (widths of tables stand for lengths).
static void plan_attention(const lsm_attention_t* a, AttentionArgs& p) {
    const uint64_t share = a->q.heads / a->kv_heads, rows = a->n_tokens * share;
    const uint64_t groups = a->prefix_width != 0 ? a->n_groups : 0;
    const uint64_t own_keys = a->own_width * a->page_tokens, prefix_keys = groups ? a->prefix_width * a->page_tokens : 0;
    p.share = (uint32_t)share, p.rows = (uint32_t)rows, p.kv_heads = (uint32_t)a->kv_heads;
    // One pass over prefix and own pages for each request, where nothing is shared or a request's rows fill tiles of 128 by themselves, and where
    // reading prefixes again and again is no more than 64 MB out of caches: two passes and the join of their parts cost more then (32 decodes behind
    // 4 prefixes of 1,500, 2 KV heads: 13.8 us so and 15.7 in two stages; 200 behind 4,000, 4 KV heads, 1.7 GB: 86 and 45).
    p.whole = groups == 0 || groups >= a->n_requests || rows / a->n_requests >= 300 ||
              a->n_requests * a->kv_heads * (prefix_keys + own_keys) * a->head_dim * 4 <= 64ull << 20;
    for (int s = 0; s < 2; s++) {
        p.tiles[s] = 0, p.splits[s] = 0, p.wide[s] = 0, p.least[s] = 1;
        if (s == 0 && p.whole) continue;
        const uint64_t owners = s == 0 ? groups : a->n_requests, keys = s == 0 ? prefix_keys : own_keys + (p.whole ? prefix_keys : 0);
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
            else if (items * splits >= 300 && keys > 2048) p.least[s] = 1024 / kSplitKeys, splits = keys / 1024;
        }
        const uint64_t most = keys / (p.least[s] * kSplitKeys);
        // A first stage with long ranges: 256 workgroups or a few more leave some compute units with two and the others with one, so more of them, and the
        // fewer the longer the second stage is (at 5 TB/s beside 1 PFLOP/s), which shares the compute units with them.  256 decodes behind 8,192 and
        // 16,384, 2 KV heads: 15 own tokens each 119 -> 90 us, 1,024 each 117 -> 93 with 410 of them; 2,047 each 127 with 256 or 410, 120 with 340.
        // Behind 4,096 and 8,192 with 2,047 each: 93 with 256, 101 with 340.
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
static uint64_t join_blocks(const lsm_attention_t* a) {
    const uint64_t per_block = kWaves * kWave * 4 / a->head_dim;
    return (a->n_tokens * a->q.heads + per_block - 1) / per_block;
}
static bool fits_launches(const lsm_attention_t* a, const AttentionArgs& p) {
    constexpr uint64_t kMost = (1ull << 32) / kThreads - 1;
    return ((uint64_t)p.tiles[0] * p.splits[0] + (uint64_t)p.tiles[1] * p.splits[1]) * p.kv_heads <= kMost && (!p.joined || join_blocks(a) <= kMost);
}

static size_t part_bytes(const lsm_attention_t* a, const AttentionArgs& p) {
    if (!p.joined) return 0;
    return (size_t)(p.splits[0] + p.splits[1]) * a->n_tokens * a->q.heads * (a->head_dim * 4 + 8);
}

template <int kType, int kHead>
static void launch(const AttentionArgs& p, uint32_t blocks, uint32_t joins, hipStream_t stream) {
    if (!p.whole) hipLaunchKernelGGL((attention_kernel<kType, kHead, kBoth>), dim3(blocks), dim3(kThreads), 0, stream, p);
    else if (p.wide[1]) hipLaunchKernelGGL((attention_kernel<kType, kHead, kWideAlone>), dim3(blocks), dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((attention_kernel<kType, kHead, kNarrowAlone>), dim3(blocks), dim3(kThreads), 0, stream, p);
    if (!p.joined) return;
    hipLaunchKernelGGL((join_kernel<kType, kHead>), dim3(joins), dim3(kThreads), 0, stream, p);
}
template <int kType>
static void launch_type(const AttentionArgs& p, uint32_t head, uint32_t blocks, uint32_t joins, hipStream_t stream) {
    if (head == 64) launch<kType, 64>(p, blocks, joins, stream);
    else if (head == 128) launch<kType, 128>(p, blocks, joins, stream);
    else launch<kType, 256>(p, blocks, joins, stream);
}

}  // namespace lsm

using namespace lsm;

extern "C" size_t lsm_prefix_attention_workspace_bytes(const lsm_attention_t* a) {
    if (check_attention(a) != LSM_OK || a->n_tokens == 0) return 0;
    AttentionArgs p = {};
    plan_attention(a, p);
    return fits_launches(a, p) ? part_bytes(a, p) : 0;
}

extern "C" int lsm_prefix_attention(const lsm_attention_t* a, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_attention(a);
    if (rc != LSM_OK || a->n_tokens == 0) return rc;
    AttentionArgs p = {};
    plan_attention(a, p);
    if (!fits_launches(a, p)) return LSM_ERR_BAD_ARG;
    const size_t need = part_bytes(a, p);
    if (need != 0 && (workspace == nullptr || workspace_bytes < need || (reinterpret_cast<uint64_t>(workspace) & 255) != 0)) return LSM_ERR_WORKSPACE;
    const uint32_t blocks = p.items0 + p.tiles[1] * p.combos[1], joins = p.joined ? (uint32_t)join_blocks(a) : 0;
    p.q = a->q.data, p.out = a->out.data, p.lse = a->lse, p.k = a->k_pages.data, p.v = a->v_pages.data;
    p.q_token = a->q.token_stride, p.q_head = a->q.head_stride, p.out_token = a->out.token_stride, p.out_head = a->out.head_stride;
    p.k_page = (uint32_t)a->k_pages.page_stride * 2, p.k_token = (uint32_t)a->k_pages.token_stride * 2, p.k_head = (uint64_t)a->k_pages.head_stride * 2;
    p.v_page = (uint32_t)a->v_pages.page_stride * 2, p.v_token = (uint32_t)a->v_pages.token_stride * 2, p.v_head = (uint64_t)a->v_pages.head_stride * 2;
    p.group_offsets = a->group_offsets, p.prefix_tables = a->prefix_tables, p.prefix_lens = a->prefix_lens;
    p.q_offsets = a->q_offsets, p.own_tables = a->own_tables, p.own_lens = a->own_lens;
    p.n_tokens = (uint32_t)a->n_tokens, p.n_requests = (uint32_t)a->n_requests, p.n_groups = (uint32_t)a->n_groups, p.n_pages = (uint32_t)a->n_pages;
    p.page_shift = (uint32_t)__builtin_ctzll(a->page_tokens);
    p.prefix_width = a->n_groups ? a->prefix_width : 0, p.own_width = a->own_width;
    p.scale = a->scale * kLog2E;
    p.part_out = static_cast<float*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + (size_t)(p.splits[0] + p.splits[1]) * a->n_tokens * a->q.heads * a->head_dim * 4);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (a->dtype == LSM_BF16) launch_type<LSM_BF16>(p, a->head_dim, blocks, joins, s);
    else launch_type<LSM_FP16>(p, a->head_dim, blocks, joins, s);
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_HIP;
}
