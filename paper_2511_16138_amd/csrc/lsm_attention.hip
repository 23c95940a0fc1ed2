// lsm_prefix_attention: attention over a paged cache for batches whose requests share long prefixes.
//
// A row is one query head of one new token.  Rows of a KV head that see the same keys are packed into tiles, whatever request they
// belong to: behind a shared prefix these are the rows of the whole group, behind a request's own pages those of the request.
// A workgroup takes a tile of rows and a range of keys and goes over the keys once with a running maximum and sum; where a tile's
// keys are dealt to several workgroups (the prefix and the own pages always are, unless rows are packed by request anyway), each
// leaves its accumulator, maximum and sum, and a second kernel joins them in a fixed order.
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
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Half<LSM_FP16> {
    typedef _Float16 type;
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
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
    uint64_t k_page, k_token, k_head, v_page, v_token, v_head;  // bytes
    const int32_t *group_offsets, *prefix_tables, *prefix_lens, *q_offsets, *own_tables, *own_lens;
    uint32_t n_tokens, n_requests, n_groups, n_pages, page_shift, kv_heads, share, rows;
    uint64_t prefix_width, own_width;
    float scale;  // of the exponent of two
    // The plan.  Stage 0: rows packed by group over the prefix; stage 1: rows packed by request over its own pages, or over the
    // prefix and its own pages (`whole`).
    uint32_t whole, tiles[2], splits[2], wide[2];
    uint32_t joined;  // the parts are joined by another kernel
    float* part_out;  // [split of either stage][row][head_dim]
    float2* part_ml;  // [split of either stage][row]: maximum in units of the exponent of two, sum
};

// Keys in [0, length), in ranges of at least two splitting units; how many there are.
__device__ __forceinline__ uint32_t split_units(uint32_t units, uint32_t splits) {
    const uint32_t each = (units + splits - 1) / splits;
    return each < 2 ? 2 : each;
}
__device__ __forceinline__ uint32_t real_splits(uint32_t units, uint32_t splits) {
    const uint32_t each = split_units(units, splits);
    return (units + each - 1) / each;
}
__device__ __forceinline__ uint32_t units_of(uint32_t keys) { return (keys + kSplitKeys - 1) / kSplitKeys; }

__device__ __forceinline__ uint32_t clamp_u32(int32_t v, uint64_t most) { return v < 0 ? 0 : (uint64_t)v > most ? (uint32_t)most : (uint32_t)v; }
__device__ __forceinline__ uint32_t prefix_len(const AttentionArgs& a, uint32_t g) { return clamp_u32(a.prefix_lens[g], a.prefix_width << a.page_shift); }
__device__ __forceinline__ uint32_t own_len(const AttentionArgs& a, uint32_t r) { return clamp_u32(a.own_lens[r], a.own_width << a.page_shift); }
__device__ __forceinline__ uint32_t token_of_request(const AttentionArgs& a, uint32_t r) { return clamp_u32(a.q_offsets[r], a.n_tokens); }
__device__ __forceinline__ uint32_t token_of_group(const AttentionArgs& a, uint32_t g) { return token_of_request(a, clamp_u32(a.group_offsets[g], a.n_requests)); }

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
    uint32_t part;                 // which part it leaves
    uint32_t token0, hidden;       // own keys that token t sees: t - token0 + 1 + len[1] - (new tokens), as hidden = that for t = token0, minus 1, wrapped
};

// Copies 16 bytes a lane from global memory straight into LDS: lane i's from `from` + offset to `to` + 16 i.  No register is written, so the
// compiler, which would otherwise wait for all copies before any LDS read, need not know; whoever reads the tile waits by wait_loads.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // m0 is the compiler's own register; it keeps nothing there from one instruction to the next
__device__ __forceinline__ void copy_to_lds(const char* from, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(from), "s"(to) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }
// Until at most kLeft of this wave's vector memory operations are under way, and none of its LDS ones.
template <int kLeft>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLeft) : "memory");
}

// Order of the instructions around here: LDS reads of four products ahead of the first of them, so that they do not wait for LDS one by one.
// One of them for each of kProducts products.
template <int kProducts>
__device__ __forceinline__ void reads_ahead() {
    constexpr int kAhead = 4;
    __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
    for (int i = 0; i < kProducts - kAhead; i++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
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

    // The scores of a tile's keys, which are in LDS.
    __device__ __forceinline__ void score(const char* keys, Scores& s) const {
        const uint32_t lane = threadIdx.x & (kWave - 1), n = lane & 31, h = lane >> 5;
#pragma unroll
        for (int b = 0; b < kKeys / 32; b++) {
#pragma unroll
            for (int j = 0; j < 16; j++) s[b][j] = 0.f;
            const uint32_t row = b * 32 + n;
#pragma unroll
            for (uint32_t c = 0; c < kHead / 16; c++) {
                const x8 k = *reinterpret_cast<const x8*>(keys + row * kHead * 2 + key_word(row, 2 * c + h) * 16);
                s[b] = Half<kType>::mfma(k, query[c], s[b]);
            }
        }
        reads_ahead<kHead / 16 * (kKeys / 32)>();
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

    // Weights of the scores, and the accumulators brought to what they are relative to.
    __device__ __forceinline__ void weights(const Scores& s, Weights& p, float scale) {
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < kKeys / 32; b++)
#pragma unroll
            for (int j = 0; j < 16; j++) top = fmaxf(top, s[b][j]);
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
        float more = 0.f;
        const float base = most == -__builtin_inff() ? 0.f : -most * scale;  // a row that has seen nothing: all weights 0
#pragma unroll
        for (int b = 0; b < kKeys / 32; b++)
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                const f32x2 e = {__builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j], scale, base)), __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j + 1], scale, base))};
                const x2 w = __builtin_convertvector(e, x2);  // rounded to nearest, as the values are; the sum is of the weights before that
                sum += e[0], more += e[1];
                p[b * 2 + j / 8][j % 8] = w[0], p[b * 2 + j / 8][j % 8 + 1] = w[1];
            }
        sum += more;
    }

    // The left operand of product i of weigh: of columns i / kSteps * 32 .. + 31 the keys i % kSteps * 16 .. + 15.  16 lanes read a block of 4 keys x 16
    // columns, lane i of them gets column i.
    static constexpr uint32_t kSteps = kKeys / 16, kProducts = kHead / 32 * kSteps, kAhead = 4;
    static __device__ __forceinline__ x8 value_operand(const char* values, uint32_t i) {
        const uint32_t lane = threadIdx.x & (kWave - 1), h = lane >> 5, i16 = lane & 15, column = ((lane >> 4) & 1) * 16 + (i16 & 3) * 4;
        union {
            x8 all;
            s16x4 part[2];
        } u;
#pragma unroll
        for (uint32_t j = 0; j < 2; j++) {
            const uint32_t row = i % kSteps * 16 + 8 * j + 4 * h + (i16 >> 2), at = i / kSteps * 32 + column;
            const char* from = values + row * kHead * 2 + value_word(row, at >> 3) * 16 + (at & 4) * 2;
            u.part[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(from));
        }
        return u.all;
    }

    // The values, which are in LDS, by their weights.
    __device__ __forceinline__ void weigh(const char* values, const Weights& p) {
        x8 v[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; i++) v[i] = value_operand(values, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t i = 0; i < kProducts; i++) {
            acc[i / kSteps] = Half<kType>::mfma(v[i % kAhead], p[i % kSteps], acc[i / kSteps]);
            if (i + kAhead < kProducts) v[i % kAhead] = value_operand(values, i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// A wide tile's keys are copied by all waves together, a narrow one's by each wave for itself.
template <int kType, int kHead>
struct Shape {
    static constexpr int kWideKeys = kHead == 256 ? 32 : 64, kNarrowKeys = kHead == 64 ? 64 : 32;
    typedef Team<kType, kHead, kWaves, kWideKeys> Wide;
    typedef Team<kType, kHead, 1, kNarrowKeys> Narrow;
    static constexpr uint32_t kWideLds = Wide::kBytes * 2 * 2, kNarrowLds = Narrow::kBytes * 2 * kWaves;
    static constexpr uint32_t kLds = kWideLds > kNarrowLds ? kWideLds : kNarrowLds;
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
    const uint32_t token = row / a.share, head = kv_head * a.share + (row - token * a.share);
    {
        const T* from = static_cast<const T*>(a.q) + (int64_t)token * a.q_token + (int64_t)head * a.q_head + h * 8;
#pragma unroll
        for (uint32_t c = 0; c < kHead / 16; c++) {
            if (has_row) {
                x.query[c] = *reinterpret_cast<const x8*>(from + c * 16);
            } else {
#pragma unroll
                for (int j = 0; j < 8; j++) x.query[c][j] = (T)0.f;
            }
        }
    }
    const int32_t sees = (int32_t)(token - w.token0 + w.hidden) + 1;  // own keys this row sees
    // tiles of this range: of the first segment, then of the second as far as any row of the tile sees
    const uint32_t units0 = units_of(w.len[0]), tile_rows = kWide ? kWideRows : kNarrowRows;
    const uint32_t last_row = w.row_end - w.row0 < tile_rows ? w.row_end - 1 : w.row0 + tile_rows - 1;
    const uint32_t first_row = w.row0 + (kWide ? wave * 32 : 0);
    const int32_t most_seen = (int32_t)(last_row / a.share - w.token0 + w.hidden) + 1;
    const int32_t least_seen = (int32_t)(first_row / a.share - w.token0 + w.hidden) + 1;  // of the rows of this wave
    const uint32_t seen = most_seen < 0 ? 0 : (uint32_t)most_seen < w.len[1] ? (uint32_t)most_seen : w.len[1];
    const uint32_t units = a.n_pages == 0 ? 0 : units0 + units_of(seen);
    const uint32_t unit1 = w.unit1 < units ? w.unit1 : units;
    const uint32_t tile_end = unit1 * kPerUnit, step = kWide ? 1 : kWaves, second = units0 * kPerUnit;  // tiles from `second` on are of the second segment
    uint32_t t = w.unit0 * kPerUnit + (kWide ? 0 : wave);

    // The pages of the wave's next tiles, so many of each tile, a page a lane; `pages_there`: which of them there are.  One load for 64 of them, and
    // no vector memory operations but the copies in between, which the waits below count.
    const uint32_t page_mask = (1u << a.page_shift) - 1;
    const uint32_t shift = a.page_shift, page_log = shift >= (kKeys == 64 ? 6 : 5) ? 0 : (kKeys == 64 ? 6 : 5) - shift;  // log2 of the pages of a tile
    int32_t pages = -1;
    uint64_t pages_there = 0;
    uint32_t pages_first = 0;  // the tile of lane 0
    auto read_pages = [&](uint32_t t) {
        const uint32_t u = t + (lane >> page_log) * step;
        const bool own = u >= second;
        const uint32_t at = (u - (own ? second : 0)) * kKeys + ((lane & ((1u << page_log) - 1)) << shift);
        pages = -1;
        if (u < tile_end && at < (own ? seen : w.len[0])) pages = (own ? w.table[1] : w.table[0])[at >> shift];
        pages_there = __ballot((uint32_t)pages < a.n_pages);
        pages_first = t;
    };
    auto page_lane = [&](uint32_t t) { return (kWide ? t - pages_first : (t - pages_first) / step) << page_log; };
    auto next_pages = [&](uint32_t t) {
        if (page_lane(t) >= kWave) read_pages(t);
    };
    // Which keys of tile t there are.
    auto keys_there = [&](uint32_t t) -> uint64_t {
        const bool own = t >= second;
        const uint32_t at = (t - (own ? second : 0)) * kKeys, len = own ? seen : w.len[0], left = at < len ? len - at : 0;
        const uint64_t there = pages_there >> page_lane(t), full = (1ull << (1u << page_log)) - 1;  // at most 4 pages
        uint64_t keys = left >= (uint32_t)kKeys ? kAllKeys : (1ull << left) - 1;
        if ((there & full) != full) {
            for (uint32_t i = 0; i < (1u << page_log); i++)
                if (!((there >> i) & 1)) keys &= page_log == 0 ? 0 : ~(((1ull << (page_mask + 1)) - 1) << (i << shift));
        }
        return keys;
    };
    // One copy brings rows of one page, so the page is a scalar.  Where there is none any page does: the scores of keys that are not
    // there are masked, and their values are zeroed in LDS.
    const uint32_t in_load = lane / X::kWords, word = lane % X::kWords;
    auto copy = [&](uint32_t t, const void* from, uint64_t page_bytes, uint64_t token_bytes, uint64_t head_bytes, bool values, uint32_t to) {
        const uint32_t at = ((t - (t >= second ? second : 0)) * kKeys) & page_mask, first = page_lane(t);
        const char* base = static_cast<const char*>(from) + (uint64_t)kv_head * head_bytes + (uint64_t)at * token_bytes;
#pragma unroll
        for (uint32_t i = 0; i < X::kLoads; i++) {
            const uint32_t r0 = (i * kTeam + (kWide ? wave : 0)) * X::kRowsPerLoad, r = r0 + in_load;
            const uint32_t p = (uint32_t)__builtin_amdgcn_readlane(pages, (int)(first + (r0 >> shift))), held = p < a.n_pages ? p : 0;
            copy_to_lds(base + (uint64_t)held * page_bytes + (uint64_t)(r0 & page_mask) * token_bytes,
                        in_load * (uint32_t)token_bytes + (values ? X::value_word(r, word) : X::key_word(r, word)) * 16, to + r0 * kHead * 2);
        }
    };
    auto copy_keys = [&](uint32_t t, uint32_t to) { copy(t, a.k, a.k_page, a.k_token, a.k_head, false, to); };
    auto copy_values = [&](uint32_t t, uint32_t to) { copy(t, a.v, a.v_page, a.v_token, a.v_head, true, to); };
    // values of keys that are not there: zeros, whatever the page holds
    auto zero_values = [&](uint64_t present, char* values) {
        for (uint32_t i = kWide ? threadIdx.x : lane; i < kKeys * X::kWords; i += kTeam * kWave)
            if (!((present >> (i / X::kWords)) & 1)) *reinterpret_cast<uint4*>(values + i * 16) = make_uint4(0, 0, 0, 0);
    };
    auto scores_masked = [&](uint32_t t, uint64_t present, typename X::Scores& s) {
        const bool own = t >= second;
        const int32_t before = (int32_t)((t - second) * kKeys);
        if (present != kAllKeys || (own && least_seen < before + kKeys)) X::mask(s, present, own ? sees - before : kKeys);
    };
    const uint32_t copies = lds_address(buffers);
    if (t < tile_end) read_pages(t);
    if (kWide) {
        // Two buffers: a tile is asked for while the one before it is worked on.
        if (t < tile_end) {
            copy_keys(t, copies);
            copy_values(t, copies + X::kBytes);
            uint32_t buffer = 0;
            for (; t < tile_end; t++) {
                const uint64_t present = keys_there(t);
                char* keys = buffers + buffer;
                char* values = keys + X::kBytes;
                buffer ^= 2 * X::kBytes;
                wait_loads<0>();
                __builtin_amdgcn_s_barrier();  // the tile is there, and everybody is done with the one before it
                if (t + 1 < tile_end) {
                    next_pages(t + 1);
                    copy_keys(t + 1, copies + buffer);
                    copy_values(t + 1, copies + buffer + X::kBytes);
                }
                if (present != kAllKeys) {
                    zero_values(present, values);
                    wait_loads<63>();
                    __builtin_amdgcn_s_barrier();
                }
                typename X::Scores s;
                typename X::Weights p;
                x.score(keys, s);
                scores_masked(t, present, s);
                x.weights(s, p, a.scale);
                x.weigh(values, p);
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
                    next_pages(t + step);
                    copy_keys(t + step, copies);
                }
                scores_masked(t, present, s);
                x.weights(s, p, a.scale);
                if (more) wait_loads<X::kLoads>();  // but for the next keys
                else wait_loads<0>();
                if (present != kAllKeys) zero_values(present, values);
                x.weigh(values, p);
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
    const uint64_t place = (uint64_t)w.part * a.rows * a.kv_heads;  // rows of all KV heads: token by token, all heads of a token
    if (has_row && h == 0 && (kWide || wave == 0)) {
        const uint64_t at = (uint64_t)token * a.share * a.kv_heads + head;
        if (a.joined) a.part_ml[place + at] = make_float2(most, sum);
        else if (a.lse != nullptr) a.lse[at] = sum == 0.f ? -__builtin_inff() : (most + log2f(sum)) * 0.69314718055994531f;
    }
#pragma unroll
    for (uint32_t s = 0; s < kHead / 64; s++) {
#pragma unroll
        for (uint32_t d = 0; d < 2; d++)
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                const f32x16& v = x.acc[s * 2 + d];
                float4 o = make_float4(v[j * 4] * by, v[j * 4 + 1] * by, v[j * 4 + 2] * by, v[j * 4 + 3] * by);
                *reinterpret_cast<float4*>(slices + (wave * 32 + n) * S::kSlicePitch + d * 32 + j * 8 + h * 4) = o;
            }
        __syncthreads();
        // eight columns a thread
        for (uint32_t u = threadIdx.x; u < (kWide ? kWideRows : kNarrowRows) * 8; u += kThreads) {
            const uint32_t r = u >> 3, c = (u & 7) * 8;
            if (w.row0 + r >= w.row_end) break;
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; j++) o[j] = slices[r * S::kSlicePitch + c + j];
            if (!kWide) {
#pragma unroll
                for (uint32_t i = 1; i < kWaves; i++)
#pragma unroll
                    for (int j = 0; j < 8; j++) o[j] += slices[(i * 32 + r) * S::kSlicePitch + c + j];
            }
            const uint32_t tok = (w.row0 + r) / a.share, hd = kv_head * a.share + (w.row0 + r - tok * a.share);
            if (a.joined) {
                float* to = a.part_out + (place + (uint64_t)tok * a.share * a.kv_heads + hd) * kHead + s * 64 + c;
                *reinterpret_cast<float4*>(to) = make_float4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<float4*>(to + 4) = make_float4(o[4], o[5], o[6], o[7]);
            } else {
                x8 v;
#pragma unroll
                for (int j = 0; j < 8; j++) v[j] = (T)o[j];
                *reinterpret_cast<x8*>(static_cast<T*>(a.out) + (int64_t)tok * a.out_token + (int64_t)hd * a.out_head + s * 64 + c) = v;
            }
        }
        __syncthreads();
    }
}

template <int kType, int kHead>
__global__ void __launch_bounds__(kThreads, kHead == 256 ? 1 : 2) attention_kernel(const AttentionArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[Shape<kType, kHead>::kAllLds];
    uint32_t b = blockIdx.x;
    const uint32_t items0 = a.tiles[0] * a.splits[0] * a.kv_heads, stage = b >= items0 ? 1 : 0;
    if (stage) b -= items0;
    const uint32_t kv_head = b % a.kv_heads, tile = b / a.kv_heads % a.tiles[stage], split = b / a.kv_heads / a.tiles[stage];
    const bool wide = a.wide[stage] != 0;
    const uint32_t tile_rows = wide ? kWideRows : kNarrowRows;
    // Owner i of rows [offset(i), offset(i + 1)) has the tiles from offset(i) / tile_rows + i on: at least as many as it needs, at no one else's place
    Item w;
    uint32_t owner, begin, end;
    if (stage == 0) {
        owner = last_not_above(a.n_groups, tile, [&](uint32_t g) { return (uint64_t)token_of_group(a, g) * a.share / tile_rows + g; });
        begin = token_of_group(a, owner), end = token_of_group(a, owner + 1);
    } else {
        owner = last_not_above(a.n_requests, tile, [&](uint32_t r) { return (uint64_t)token_of_request(a, r) * a.share / tile_rows + r; });
        begin = token_of_request(a, owner), end = token_of_request(a, owner + 1);
    }
    const uint64_t row0 = (uint64_t)begin * a.share + (uint64_t)(tile - ((uint64_t)begin * a.share / tile_rows + owner)) * tile_rows;
    if (end <= begin || row0 >= (uint64_t)end * a.share) return;
    w.row0 = (uint32_t)row0;
    w.row_end = end * a.share;
    if (stage == 0) {
        w.table[0] = a.prefix_tables + owner * a.prefix_width, w.len[0] = prefix_len(a, owner);
        w.table[1] = nullptr, w.len[1] = 0;
    } else {
        w.len[0] = 0, w.table[0] = nullptr;
        if (a.whole && a.prefix_width != 0) {
            const uint32_t g = group_of(a, owner);
            w.table[0] = a.prefix_tables + g * a.prefix_width, w.len[0] = prefix_len(a, g);
        }
        w.table[1] = a.own_tables + owner * a.own_width, w.len[1] = own_len(a, owner);
    }
    w.token0 = begin;
    w.hidden = w.len[1] - (end - begin);
    const uint32_t units = units_of(w.len[0]) + units_of(w.len[1]), each = split_units(units, a.splits[stage]);
    w.unit0 = split * each, w.unit1 = w.unit0 + each < units ? w.unit0 + each : units;
    if (a.joined && w.unit0 >= units) return;  // not one of the ranges that there are
    w.part = (stage ? a.splits[0] : 0) + split;
    if (wide) attend<kType, kHead, true>(a, w, kv_head, lds);
    else attend<kType, kHead, false>(a, w, kv_head, lds);
}

// Joins a row's parts: those of its prefix, then those of its own pages, each in the order of the keys.  kHead / 4 lanes have a row.
template <int kType, int kHead>
__global__ void __launch_bounds__(kThreads) join_kernel(const AttentionArgs a) {
    typedef typename Half<kType>::type T;
    constexpr uint32_t kLanes = kHead / 4, kRows = kWave / kLanes;  // rows of a wave
    const uint32_t lane = threadIdx.x & (kWave - 1), heads = a.share * a.kv_heads;
    const uint64_t all = (uint64_t)a.n_tokens * heads;
    const uint64_t first = ((uint64_t)blockIdx.x * kWaves + threadIdx.x / kWave) * kRows;
    if (first >= all) return;
    uint64_t at = first + lane / kLanes;
    const bool mine = at < all;
    if (!mine) at = all - 1;
    const uint32_t token = (uint32_t)(at / heads), head = (uint32_t)(at - (uint64_t)token * heads), c = (lane % kLanes) * 4;
    // a wave's rows may belong to two tokens, and these to two requests
    const uint32_t token_a = (uint32_t)(first / heads);
    uint32_t request = last_not_above(a.n_requests, token_a, [&](uint32_t r) { return (uint64_t)token_of_request(a, r); });
    while (request + 1 < a.n_requests && token_of_request(a, request + 1) <= token) request++;
    uint32_t parts[2], from[2] = {0, a.splits[0]};
    uint32_t g = 0;
    if (a.prefix_width != 0) {
        const uint32_t first_request = (uint32_t)__builtin_amdgcn_readfirstlane((int)request);
        g = group_of(a, first_request);
        while (g + 1 < a.n_groups && clamp_u32(a.group_offsets[g + 1], a.n_requests) <= request) g++;
    }
    const uint32_t units0 = a.prefix_width != 0 ? units_of(prefix_len(a, g)) : 0, units1 = units_of(own_len(a, request));
    parts[0] = a.whole ? 0 : real_splits(units0, a.splits[0]);
    parts[1] = real_splits(units1 + (a.whole ? units0 : 0), a.splits[1]);
    float most = -__builtin_inff(), sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (uint32_t stage = 0; stage < 2; stage++)
        for (uint32_t i = 0; i < parts[stage]; i++) {
            const uint64_t place = (uint64_t)(from[stage] + i) * all + at;
            const float2 ml = a.part_ml[place];
            const float4 v = *reinterpret_cast<const float4*>(a.part_out + place * kHead + c);
            const float now = fmaxf(most, ml.x), base = now == -__builtin_inff() ? 0.f : now;
            const float old_by = __builtin_amdgcn_exp2f(most - base), new_by = __builtin_amdgcn_exp2f(ml.x - base);
            sum = sum * old_by + ml.y * new_by;
            o.x = o.x * old_by + v.x * new_by, o.y = o.y * old_by + v.y * new_by;
            o.z = o.z * old_by + v.z * new_by, o.w = o.w * old_by + v.w * new_by;
            most = now;
        }
    if (!mine) return;
    const float by = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    typedef T x4 __attribute__((ext_vector_type(4)));
    x4 r;
    r[0] = (T)(o.x * by), r[1] = (T)(o.y * by), r[2] = (T)(o.z * by), r[3] = (T)(o.w * by);
    *reinterpret_cast<x4*>(static_cast<T*>(a.out) + (int64_t)token * a.out_token + (int64_t)head * a.out_head + c) = r;
    if (a.lse != nullptr && lane % kLanes == 0) a.lse[at] = sum == 0.f ? -__builtin_inff() : (most + log2f(sum)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------------
static bool aligned_rows(const void* data, int64_t s0, int64_t s1, int64_t s2) {
    return ((reinterpret_cast<uint64_t>(data) | (uint64_t)(s0 * 2) | (uint64_t)(s1 * 2) | (uint64_t)(s2 * 2)) & 15) == 0;
}

static int check_attention(const lsm_attention_t* a) {
    if (a == nullptr) return LSM_ERR_NULL;
    if (a->dtype != LSM_BF16 && a->dtype != LSM_FP16) return LSM_ERR_BAD_ARG;
    if (a->head_dim != 64 && a->head_dim != 128 && a->head_dim != 256) return LSM_ERR_BAD_ARG;
    if (a->page_tokens < LSM_MIN_PAGE_TOKENS || a->page_tokens > LSM_MAX_PAGE_TOKENS || (a->page_tokens & (a->page_tokens - 1)) != 0) return LSM_ERR_BAD_ARG;
    if (a->kv_heads == 0 || a->q.heads == 0 || a->q.heads != a->out.heads || a->q.heads % a->kv_heads != 0 || a->q.heads > 4096) return LSM_ERR_BAD_ARG;
    if (a->n_tokens >= 1u << 24 || a->n_tokens * a->q.heads >= 1ull << 31 || a->n_requests >= 1u << 24 || a->n_groups >= 1u << 24 || a->n_pages >= 1ull << 31) return LSM_ERR_BAD_ARG;
    if (a->prefix_width * a->page_tokens >= 1ull << 30 || a->own_width * a->page_tokens >= 1ull << 30 || a->prefix_width >= 1u << 30 || a->own_width >= 1u << 30) return LSM_ERR_BAD_ARG;
    if (a->reserved != 0 || !(a->scale > 0.f) || a->scale > 3.0e38f) return LSM_ERR_BAD_ARG;
    if (a->n_tokens == 0) return LSM_OK;
    if (a->n_requests == 0) return LSM_ERR_BAD_ARG;
    if (a->q.data == nullptr || a->out.data == nullptr || a->q_offsets == nullptr || a->own_lens == nullptr) return LSM_ERR_NULL;
    if (a->own_width != 0 && a->own_tables == nullptr) return LSM_ERR_NULL;
    if (a->prefix_width != 0 && a->n_groups != 0 && (a->prefix_tables == nullptr || a->prefix_lens == nullptr || a->group_offsets == nullptr)) return LSM_ERR_NULL;
    if (a->n_pages != 0 && (a->k_pages.data == nullptr || a->v_pages.data == nullptr)) return LSM_ERR_NULL;
    if (!aligned_rows(a->q.data, a->q.token_stride, a->q.head_stride, 0) || !aligned_rows(a->out.data, a->out.token_stride, a->out.head_stride, 0) ||
        !aligned_rows(a->k_pages.data, a->k_pages.page_stride, a->k_pages.token_stride, a->k_pages.head_stride) ||
        !aligned_rows(a->v_pages.data, a->v_pages.page_stride, a->v_pages.token_stride, a->v_pages.head_stride)) return LSM_ERR_BAD_ARG;
    // a copy's lanes reach 16 rows from a scalar address by 32-bit offsets
    for (const lsm_pages_t* p : {&a->k_pages, &a->v_pages})
        if (p->page_stride < 0 || p->token_stride < 0 || p->head_stride < 0 || p->token_stride >= 1 << 26) return LSM_ERR_BAD_ARG;
    const uint64_t words = reinterpret_cast<uint64_t>(a->lse) | reinterpret_cast<uint64_t>(a->group_offsets) | reinterpret_cast<uint64_t>(a->prefix_tables) |
                           reinterpret_cast<uint64_t>(a->prefix_lens) | reinterpret_cast<uint64_t>(a->q_offsets) | reinterpret_cast<uint64_t>(a->own_tables) |
                           reinterpret_cast<uint64_t>(a->own_lens);
    return words & 3 ? LSM_ERR_BAD_ARG : LSM_OK;
}

// How the work is cut; from sizes that the host knows.
static void plan_attention(const lsm_attention_t* a, AttentionArgs& p) {
    const uint64_t share = a->q.heads / a->kv_heads, rows = a->n_tokens * share;
    const uint64_t groups = a->prefix_width != 0 ? a->n_groups : 0, mean = rows / a->n_requests;
    p.share = (uint32_t)share, p.rows = (uint32_t)rows, p.kv_heads = (uint32_t)a->kv_heads;
    p.whole = groups == 0 || groups >= a->n_requests || mean >= 96;
    const uint64_t own_keys = a->own_width * a->page_tokens, prefix_keys = groups ? a->prefix_width * a->page_tokens : 0;
    const uint64_t target = 512;  // workgroups wanted: two for each compute unit
    for (int s = 0; s < 2; s++) {
        p.tiles[s] = 0, p.splits[s] = 0, p.wide[s] = 0;
        if (s == 0 && p.whole) continue;
        const uint64_t owners = s == 0 ? groups : a->n_requests, keys = s == 0 ? prefix_keys : own_keys + (p.whole ? prefix_keys : 0);
        p.wide[s] = rows / owners > 48;
        const uint64_t tile_rows = p.wide[s] ? kWideRows : kNarrowRows;
        p.tiles[s] = (uint32_t)(rows / tile_rows + owners);
        const uint64_t real = rows / tile_rows > owners ? rows / tile_rows : owners;
        uint64_t splits = target / (real * a->kv_heads), most = (keys + 2 * kSplitKeys - 1) / (2 * kSplitKeys);
        if (splits > most) splits = most;
        if (splits > 64) splits = 64;
        p.splits[s] = splits > 1 ? (uint32_t)splits : 1;
    }
    p.joined = !(p.whole && p.splits[1] == 1);
}

static size_t part_bytes(const lsm_attention_t* a, const AttentionArgs& p) {
    if (!p.joined) return 0;
    return (size_t)(p.splits[0] + p.splits[1]) * a->n_tokens * a->q.heads * (a->head_dim * 4 + 8);
}

template <int kType, int kHead>
static void launch(const AttentionArgs& p, uint32_t blocks, hipStream_t stream) {
    hipLaunchKernelGGL((attention_kernel<kType, kHead>), dim3(blocks), dim3(kThreads), 0, stream, p);
    if (!p.joined) return;
    const uint64_t all = (uint64_t)p.n_tokens * p.share * p.kv_heads, per_block = kWaves * (kWave / (kHead / 4));
    hipLaunchKernelGGL((join_kernel<kType, kHead>), dim3((uint32_t)((all + per_block - 1) / per_block)), dim3(kThreads), 0, stream, p);
}
template <int kType>
static void launch_type(const AttentionArgs& p, uint32_t head, uint32_t blocks, hipStream_t stream) {
    if (head == 64) launch<kType, 64>(p, blocks, stream);
    else if (head == 128) launch<kType, 128>(p, blocks, stream);
    else launch<kType, 256>(p, blocks, stream);
}

}  // namespace lsm

using namespace lsm;

extern "C" size_t lsm_prefix_attention_workspace_bytes(const lsm_attention_t* a) {
    if (check_attention(a) != LSM_OK || a->n_tokens == 0) return 0;
    AttentionArgs p = {};
    plan_attention(a, p);
    return part_bytes(a, p);
}

extern "C" int lsm_prefix_attention(const lsm_attention_t* a, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_attention(a);
    if (rc != LSM_OK || a->n_tokens == 0) return rc;
    AttentionArgs p = {};
    plan_attention(a, p);
    const size_t need = part_bytes(a, p);
    if (need != 0 && (workspace == nullptr || workspace_bytes < need || (reinterpret_cast<uint64_t>(workspace) & 255) != 0)) return LSM_ERR_WORKSPACE;
    const uint64_t blocks = ((uint64_t)p.tiles[0] * p.splits[0] + (uint64_t)p.tiles[1] * p.splits[1]) * p.kv_heads;
    if (blocks >= 1ull << 31) return LSM_ERR_BAD_ARG;
    p.q = a->q.data, p.out = a->out.data, p.lse = a->lse, p.k = a->k_pages.data, p.v = a->v_pages.data;
    p.q_token = a->q.token_stride, p.q_head = a->q.head_stride, p.out_token = a->out.token_stride, p.out_head = a->out.head_stride;
    p.k_page = (uint64_t)a->k_pages.page_stride * 2, p.k_token = (uint64_t)a->k_pages.token_stride * 2, p.k_head = (uint64_t)a->k_pages.head_stride * 2;
    p.v_page = (uint64_t)a->v_pages.page_stride * 2, p.v_token = (uint64_t)a->v_pages.token_stride * 2, p.v_head = (uint64_t)a->v_pages.head_stride * 2;
    p.group_offsets = a->group_offsets, p.prefix_tables = a->prefix_tables, p.prefix_lens = a->prefix_lens;
    p.q_offsets = a->q_offsets, p.own_tables = a->own_tables, p.own_lens = a->own_lens;
    p.n_tokens = (uint32_t)a->n_tokens, p.n_requests = (uint32_t)a->n_requests, p.n_groups = (uint32_t)a->n_groups, p.n_pages = (uint32_t)a->n_pages;
    p.page_shift = (uint32_t)__builtin_ctzll(a->page_tokens);
    p.prefix_width = a->n_groups ? a->prefix_width : 0, p.own_width = a->own_width;
    p.scale = a->scale * 1.44269504088896341f;
    p.part_out = static_cast<float*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + (size_t)(p.splits[0] + p.splits[1]) * a->n_tokens * a->q.heads * a->head_dim * 4);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (a->dtype == LSM_BF16) launch_type<LSM_BF16>(p, a->head_dim, (uint32_t)blocks, s);
    else launch_type<LSM_FP16>(p, a->head_dim, (uint32_t)blocks, s);
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_HIP;
}
