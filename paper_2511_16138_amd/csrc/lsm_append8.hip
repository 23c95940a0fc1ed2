// lsm_kv_append8: keys and values of new tokens, normed and rotated, into pages of 8 bits with a scale for each block of 16 tokens and head.
#include <hip/hip_runtime.h>

#include "lsm_e4m3.h"
#include "lsm_pages.h"
#include "lsm_rotate.h"

namespace lsm {

struct Side {  // keys or values
    const void* in;
    uint8_t *pages, *scales;
    int64_t in_token, in_head;  // elements
    int64_t page, token, head;  // bytes, as all that follow
    int64_t scale_page, scale_block, scale_head;
};

struct Append8Args {
    RotateArgs rotate;  // the queries, and what belongs to keys as well: positions, table, sizes
    Side side[2];
    const void* weight;  // of the keys
    const int32_t *q_offsets, *own_tables, *own_lens;
    uint64_t own_width;
    uint32_t n_tokens, n_requests, n_pages, heads, page_blocks;
    uint32_t first_step;         // a power of 64: every so many requests there is one of the first 64 looked at
    uint32_t first_tile, tiles;  // of this launch
    uint32_t groups;             // workgroups of keys and values; those of the queries come after them
    uint32_t wide;               // bit 0: inputs' rows are 16-byte aligned, bit 1: pages' are aligned to a lane's bytes
    float most;
};

// A request's blocks have the tiles from its first token / 16 + 2 * its number on: at least as many as it reaches blocks, at no one else's place.
__device__ __forceinline__ uint32_t first_tile_of(uint32_t token, uint32_t request) { return token / LSM_SCALE_TOKENS + 2 * request; }

// x rounded to odd: to the float next to it that has the last bit set, where it is none itself.  What is rounded again, to fewer bits, comes out as if it had been
// rounded once.
__device__ __forceinline__ float to_odd(double x) {
    const float f = (float)x;
    const uint32_t bits = __float_as_uint(f);
    const double back = (double)f;
    const bool over = __builtin_fabs(back) > __builtin_fabs(x);  // an infinity that x does not have, too
    return back == x || x != x ? f : __uint_as_float((over ? bits - 1 : bits) | 1);
}

// 1 / sqrt(x) in 64 bits: an estimate and two steps of Newton's method; what has no such value is as the estimate has it (0: infinity, infinity: 0).
__device__ __forceinline__ double inverse_root(double x) {
    double y = __builtin_amdgcn_rsq(x);
    if (x > 0.0 && x < __builtin_inf()) {
        y = y * (1.5 - 0.5 * x * y * y);
        y = y * (1.5 - 0.5 * x * y * y);
    }
    return y;
}

// One wave has a block of 16 tokens of one head, keys or values: kLanes lanes of 16 bytes hold a row, and the rows wait in LDS until the largest magnitude is known, so
// every byte is read once and written once.  No other wave writes any of the block, nor its scale.
// Keys are normed and rotated in 64 bits: a code is the nearest one to the formula's value then, and not to one that 32 bits have moved across the border between
// two codes (one to three in a million).  That is about 20 instructions an element, and waves of 90 registers (fp16; 121 to 127 in bf16), 20 of them (16) on a compute unit, keep enough
// loads under way beside them: 16,384 tokens of 32 + 2 * 8 heads take 92.6 us in bf16 (78 at a copy's rate, 83 in 32 bits).  With the rows in registers a wave has 140 and more of
// these, and the same takes 105 to 136 us.
// kMode: 0 = pairs half the rotated part apart, a whole number of lanes; 1 = pairs of neighbours; both with aligned rows and weights of the elements' type; 2 = anything
// else; 3, 4 = as 0 and 1, with weights of 32 bits for elements of 16 (16,384 tokens: 107 us for 93 with 16 bits; by the way for anything 388).
template <int kType, int kLanes, int kMode>
__device__ __forceinline__ void append_block(const Append8Args& a, uint32_t wave, float* staged) {
    typedef typename Element<kType>::type T;
    constexpr int E = kEach<T>, kPairs = kMode >= 3 ? kMode - 3 : kMode;
    constexpr uint32_t kRows = kWave / kLanes, kSteps = LSM_SCALE_TOKENS / kRows;  // rows at a time
    static_assert(kRows * kSteps == LSM_SCALE_TOKENS, "");
    const uint32_t lane = threadIdx.x & (kWave - 1), sub = lane / kLanes, e0 = (lane & (kLanes - 1)) * E;
    const uint32_t tile = a.first_tile + wave / (2 * a.heads), combo = wave % (2 * a.heads);
    const bool keys = combo < a.heads;
    const uint32_t head = keys ? combo : combo - a.heads;
    if (tile >= a.first_tile + a.tiles) return;
    // Whose tile it is: of 64 requests that divide those in question the last whose first tile is not behind it, then among the requests up to the next of the 64, and so on.
    // (All requests one after the other, 64 at a time: decodes of 16,384 requests, 8 heads 5,750 us for 695, and 2^20 of them some 20 seconds.)
    uint32_t request = 0, t0, t1;
    int32_t len;
    for (uint32_t step = a.first_step;; step /= kWave) {
        const uint64_t i = request + (uint64_t)lane * step, at = i < a.n_requests ? i : a.n_requests - 1;
        const int32_t from = a.q_offsets[at], to = a.q_offsets[at + 1], length = a.own_lens[at];
        const uint32_t begin = from < 0 ? 0 : min((uint32_t)from, a.n_tokens), end = to < 0 ? 0 : min((uint32_t)to, a.n_tokens);
        const int count = __popcll(__ballot(i < a.n_requests && first_tile_of(begin, (uint32_t)at) <= tile));  // no more than there are such requests: offsets may descend
        if (count == 0) return;
        request += (uint32_t)(count - 1) * step;
        if (step > 1) continue;
        t0 = (uint32_t)__builtin_amdgcn_readlane((int)begin, count - 1), t1 = (uint32_t)__builtin_amdgcn_readlane((int)end, count - 1);
        len = __builtin_amdgcn_readlane(length, count - 1);
        break;
    }
    if (t1 <= t0 || len <= 0 || tile < first_tile_of(t0, request)) return;
    // its block, and the rows [row0, row1) of it that are new
    const int64_t start = (int64_t)len - (t1 - t0);  // place of the first new token; tokens before place 0 are not written
    const uint32_t block = (uint32_t)((start > 0 ? start : 0) / LSM_SCALE_TOKENS) + (tile - first_tile_of(t0, request));
    const int64_t place = (int64_t)block * LSM_SCALE_TOKENS;
    if (place >= len) return;
    const uint32_t row0 = start > place ? (uint32_t)(start - place) : 0, row1 = len - place < LSM_SCALE_TOKENS ? (uint32_t)(len - place) : LSM_SCALE_TOKENS;
    const uint32_t in_table = block / a.page_blocks, in_page = block - in_table * a.page_blocks;
    if (in_table >= a.own_width) return;
    const uint32_t page = (uint32_t)__builtin_amdgcn_readfirstlane(a.own_tables[request * a.own_width + in_table]);

    const Side& s = a.side[keys ? 0 : 1];
    const RotateArgs& r = a.rotate;
    const bool inside = e0 < r.head_dim;
    const int64_t first_token = (int64_t)t0 + place - start;  // of row 0
    const T* in = static_cast<const T*>(s.in) + first_token * s.in_token + (int64_t)head * s.in_head + e0;
    const uint32_t first_step = row0 / kRows, end_step = (row1 + kRows - 1) / kRows;  // steps with new rows
    auto is_new = [&](uint32_t row) { return row >= row0 && row < row1; };
    auto read_row = [&](uint32_t step) {
        const uint32_t row = step * kRows + sub;
        Lane<T> x;
        if (is_new(row) && inside) {
            x = load_lane<T>(in + (int64_t)row * s.in_token, kPairs != 2 || (a.wide & 1));
        } else {
#pragma unroll
            for (int j = 0; j < E; j++) x.v[j] = (T)0.f;
        }
        return x;
    };
    Lane<T> ahead = read_row(first_step);
    if (page >= a.n_pages) return;
    uint8_t* scale_at = s.scales + (int64_t)page * s.scale_page + (int64_t)in_page * s.scale_block + (int64_t)head * s.scale_head;
    const uint32_t old_scale = row0 > 0 ? *scale_at : 0;
    float top = 0.f;
    float* const mine = staged + sub * (kLanes * E) + e0;  // of row 0
    // to LDS, infinities as NaN and magnitudes cut to what the type holds
    auto keep = [&](uint32_t step, float (&y)[E]) {
#pragma unroll
        for (int j = 0; j < E; j++) {
            const float size = __builtin_fabsf(y[j]);
            const bool finite = size < __builtin_inff();
            y[j] = finite ? fminf(fmaxf(y[j], -a.most), a.most) : __builtin_nanf("");
            top = fmaxf(top, finite ? fminf(size, a.most) : 0.f);
        }
#pragma unroll
        for (int j = 0; j < E; j += 4) *reinterpret_cast<float4*>(mine + step * kRows * kLanes * E + j) = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
    };
    const bool normed = keys && a.weight != nullptr;
    if (normed || (keys && r.table != nullptr)) {
        const bool turns = r.table != nullptr && e0 < r.rot_dim;
        const uint32_t half = r.rot_dim >> 1;
        const bool by_lane = kPairs == 0 || (kPairs == 2 && !r.interleaved && half % E == 0), neighbours = kPairs == 1 || (kPairs == 2 && r.interleaved);
        const int other = turns && by_lane ? (int)(e0 < half ? lane + half / E : lane - half / E) : (int)lane;
        const double mean_by = 1.0 / (double)r.head_dim;
        constexpr bool kWhole = kType != LSM_FP32 && kMode < 2;  // weights of 16 bits, as the elements: 32 bits hold the bits of their products, and fp16's exponents
        float weight[E], weight_z[E];  // of this lane's elements, and of the others of their pairs
#pragma unroll
        for (int j = 0; j < E; j++) weight[j] = 1.f;
        if (normed && inside) {
            if (sizeof(T) == 4 || (kMode >= 2 && r.weight_fp32)) {
#pragma unroll
                for (int j = 0; j < E; j++) weight[j] = static_cast<const float*>(a.weight)[e0 + j];
            } else {
#pragma unroll
                for (int j = 0; j < E; j++) weight[j] = (float)static_cast<const T*>(a.weight)[e0 + j];
            }
        }
#pragma unroll
        for (int j = 0; j < E; j++) weight_z[j] = kWhole ? 1.f : neighbours ? weight[j ^ 1] : by_lane ? __shfl(weight[j], other, kWave) : 1.f;
        auto position_of = [&](uint32_t step) { return turns && is_new(step * kRows + sub) ? r.positions[first_token + step * kRows + sub] : 0; };
        int32_t position = position_of(first_step);
#pragma unroll 1
        for (uint32_t step = first_step; step < end_step; step++) {
            const Lane<T> raw = ahead;
            const int32_t p = position;
            const bool turn = turns && is_new(step * kRows + sub), known = p >= 0 && (uint64_t)p < r.n_positions;
            const float* angles = r.table + (known ? (uint64_t)p : 0) * r.rot_dim;
            float y[E], weighed[E], z[E], cosine[E], sine[E];
#pragma unroll
            for (int j = 0; j < E; j++) cosine[j] = 1.f, sine[j] = 0.f;
            if (turn) {
                if (kPairs == 1) {
                    typedef float few __attribute__((ext_vector_type(E / 2)));
                    const few c = *reinterpret_cast<const few*>(angles + e0 / 2), n = *reinterpret_cast<const few*>(angles + half + e0 / 2);
#pragma unroll
                    for (int j = 0; j < E; j++) cosine[j] = c[j / 2], sine[j] = j & 1 ? n[j / 2] : -n[j / 2];
                } else if (kPairs == 0) {
                    const uint32_t at = e0 < half ? e0 : e0 - half;
#pragma unroll
                    for (int j = 0; j < E; j += 4) {
                        const float4 c = *reinterpret_cast<const float4*>(angles + at + j), n = *reinterpret_cast<const float4*>(angles + half + at + j);
                        cosine[j] = c.x, cosine[j + 1] = c.y, cosine[j + 2] = c.z, cosine[j + 3] = c.w;
                        sine[j] = n.x, sine[j + 1] = n.y, sine[j + 2] = n.z, sine[j + 3] = n.w;
                    }
#pragma unroll
                    for (int j = 0; j < E; j++) sine[j] = e0 < half ? -sine[j] : sine[j];
                } else {
#pragma unroll 1
                    for (int j = 0; j < E; j++) {
                        const uint32_t e = e0 + j, at = r.interleaved ? e >> 1 : e < half ? e : e - half;
                        if (e >= r.rot_dim) break;
                        const float c = angles[at], n = (r.interleaved ? (e & 1) : e >= half) ? angles[half + at] : -angles[half + at];
#pragma unroll
                        for (int i = 0; i < E; i++) cosine[i] = i == j ? c : cosine[i], sine[i] = i == j ? n : sine[i];
                    }
                }
            }
            if (step + 1 < end_step) ahead = read_row(step + 1), position = position_of(step + 1);
#pragma unroll
            for (int j = 0; j < E; j++) y[j] = (float)raw.v[j];
            double by = 1.0;
            if (normed) {
                double sum = 0.0;
#pragma unroll
                for (int j = 0; j < E; j++) sum += (double)y[j] * (double)y[j];
#pragma unroll
                for (int off = 1; off < kLanes; off <<= 1) sum += __shfl_xor(sum, off, kWave);
                by = inverse_root(sum * mean_by + (double)r.eps);
            }
#pragma unroll
            for (int j = 0; j < E; j++) weighed[j] = kWhole ? y[j] * weight[j] : y[j];
            if constexpr (kWhole && kType == LSM_BF16) {
                // The product of two bfloat16 has 16 bits, but its exponent may leave the range of 32 bits, however ordinary it is once divided by the root: rows with
                // such products have them in 64 bits, and so have rows with zeros, which are not told apart.  (64 bits for all rows: 16,384 tokens 109 us for 92.6; without
                // the look 91.3.)
                float least = 1.f, largest = 0.f;
#pragma unroll
                for (int j = 0; j < E; j++) least = fminf(least, __builtin_fabsf(weighed[j])), largest = fmaxf(largest, __builtin_fabsf(weighed[j]));
                if (normed && __any(is_new(step * kRows + sub) && inside && !(least >= 0x1p-126f && largest < __builtin_inff()))) {
#pragma unroll
                    for (int j = 0; j < E; j++) {
                        double x = (double)y[j] * (double)weight[j];
                        const double pair = neighbours ? (double)y[j ^ 1] * (double)weight[j ^ 1] : by_lane ? __shfl(x, other, kWave) : 0.0;
                        if (turn && e0 + j < r.rot_dim) {
                            x = x * (double)cosine[j] + pair * (double)sine[j];
                            if (!known) x = __builtin_nan("");
                        }
                        z[j] = to_odd(x * by);
                    }
                    keep(step, z);
                    continue;
                }
            }
#pragma unroll
            for (int j = 0; j < E; j++) z[j] = neighbours ? weighed[j ^ 1] : by_lane ? __shfl(weighed[j], other, kWave) : 0.f;
            if (kPairs == 2 && turn && !neighbours && !by_lane) {  // the other element of the pair is in no whole lane: read again
                const T* row = in - e0 + (int64_t)(step * kRows + sub) * s.in_token;
#pragma unroll
                for (int j = 0; j < E; j++) {
                    const uint32_t e = e0 + j, pair = e < half ? e + half : e - half;
                    if (e < r.rot_dim) {
                        z[j] = (float)row[pair];
                        if (normed) weight_z[j] = sizeof(T) == 4 || r.weight_fp32 ? static_cast<const float*>(a.weight)[pair] : (float)static_cast<const T*>(a.weight)[pair];
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < E; j++) {
                double x = kWhole ? (double)weighed[j] : (double)y[j] * (double)weight[j];
                if (turn && e0 + j < r.rot_dim) {
                    x = x * (double)cosine[j] + (kWhole ? (double)z[j] : (double)z[j] * (double)weight_z[j]) * (double)sine[j];
                    if (!known) x = __builtin_nan("");
                }
                y[j] = to_odd(x * by);
            }
            keep(step, y);
        }
    } else {
#pragma unroll 2
        for (uint32_t step = first_step; step < end_step; step++) {
            const Lane<T> raw = ahead;
            if (step + 1 < end_step) ahead = read_row(step + 1);
            float y[E];
#pragma unroll
            for (int j = 0; j < E; j++) y[j] = (float)raw.v[j];
            keep(step, y);
        }
    }
    // the block's scale
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
    uint32_t scale = scale_for(top);
    if (row0 > 0 && old_scale > scale) scale = old_scale;
    uint8_t* rows = s.pages + (int64_t)page * s.page + (int64_t)(in_page * LSM_SCALE_TOKENS) * s.token + (int64_t)head * s.head + e0;
    if (row0 > 0 && scale != old_scale && inside) {
        const float by = power_of_two((int)old_scale - (int)scale);
#pragma unroll 1
        for (uint32_t row = sub; row < row0; row += kRows) {
            uint8_t* at = rows + (int64_t)row * s.token;
            Codes<E> c = load_codes<E>(at, kPairs != 2 || (a.wide & 2));
            float x[E];
            decode(c, x);
#pragma unroll
            for (int j = 0; j < E; j++) x[j] *= by;
            store_codes<E>(at, encode<E>(x), kPairs != 2 || (a.wide & 2));
        }
    }
    const float by = power_of_two(127 - (int)scale);
#pragma unroll 2
    for (uint32_t step = first_step; step < end_step; step++) {
        const uint32_t row = step * kRows + sub;
        float y[E];
#pragma unroll
        for (int j = 0; j < E; j += 4) {
            const float4 v = *reinterpret_cast<const float4*>(mine + step * kRows * kLanes * E + j);  // as this lane left it
            y[j] = v.x * by, y[j + 1] = v.y * by, y[j + 2] = v.z * by, y[j + 3] = v.w * by;
        }
        if (is_new(row) && inside) store_codes<E>(rows + (int64_t)row * s.token, encode<E>(y), kPairs != 2 || (a.wide & 2));
    }
    if (lane == 0) *scale_at = (uint8_t)scale;
}

template <int kType, int kLanes, int kMode>
__global__ void __launch_bounds__(256) append8_kernel(const Append8Args a) {
    constexpr uint32_t kStaged = LSM_SCALE_TOKENS * kLanes * kEach<typename Element<kType>::type>;
    __shared__ __attribute__((aligned(16))) float staged[4 * kStaged];
    const uint32_t in_group = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    // Workgroups of either kind by turns: those of the queries do little but move bytes, those of keys and values wait for chains of reads and compute
    // (16,384 tokens in 32 bits: 99 us with the queries last, 83 so).
    const uint32_t before = (uint32_t)((uint64_t)blockIdx.x * a.groups / gridDim.x), after = (uint32_t)((uint64_t)(blockIdx.x + 1) * a.groups / gridDim.x);
    if (after != before) {
        append_block<kType, kLanes, kMode>(a, before * 4 + in_group, staged + in_group * kStaged);
    } else {
        const uint32_t wave = (blockIdx.x - before) * 4 + in_group;
        if constexpr (kMode == 2) rotate_any<kType, kLanes>(a.rotate, wave);
        else rotate_aligned<kType, kLanes, kMode == 1 || kMode == 4>(a.rotate, wave);
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------------
static int set_side(Side& s, const lsm_rotation_t* how, const lsm_heads_t* in, const lsm_pages_t* pages, const lsm_scales_t* scales, bool any) {
    if (any && (in->data == nullptr || pages->data == nullptr || scales->data == nullptr)) return LSM_ERR_NULL;
    if (reinterpret_cast<uint64_t>(in->data) & (element_bytes(how->dtype) - 1)) return LSM_ERR_BAD_ARG;
    s = Side{in->data, static_cast<uint8_t*>(pages->data), scales->data, in->token_stride, in->head_stride, pages->page_stride, pages->token_stride, pages->head_stride,
             scales->page_stride, scales->block_stride, scales->head_stride};
    return LSM_OK;
}

template <int kType, int kLanes>
static void launch_lanes(const Append8Args& a, int mode, uint32_t blocks, hipStream_t stream) {
    if constexpr (kType != LSM_FP32) {
        if (mode == 3) hipLaunchKernelGGL((append8_kernel<kType, kLanes, 3>), dim3(blocks), dim3(256), 0, stream, a);
        if (mode == 4) hipLaunchKernelGGL((append8_kernel<kType, kLanes, 4>), dim3(blocks), dim3(256), 0, stream, a);
        if (mode >= 3) return;
    }
    if (mode == 0) hipLaunchKernelGGL((append8_kernel<kType, kLanes, 0>), dim3(blocks), dim3(256), 0, stream, a);
    else if (mode == 1) hipLaunchKernelGGL((append8_kernel<kType, kLanes, 1>), dim3(blocks), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((append8_kernel<kType, kLanes, 2>), dim3(blocks), dim3(256), 0, stream, a);
}
template <int kType>
static void launch_type(const Append8Args& a, uint32_t lanes, int mode, uint32_t blocks, hipStream_t stream) {
    if (lanes == 8) launch_lanes<kType, 8>(a, mode, blocks, stream);
    else if (lanes == 16) launch_lanes<kType, 16>(a, mode, blocks, stream);
    else if (kType != LSM_FP32 || lanes == 32) launch_lanes<kType, 32>(a, mode, blocks, stream);
    else launch_lanes<LSM_FP32, 64>(a, mode, blocks, stream);
}

}  // namespace lsm

using namespace lsm;

extern "C" int lsm_kv_append8(const lsm_rotation_t* how, const lsm_heads_t* k, const void* k_weight, const lsm_heads_t* v, const lsm_new_tokens_t* to,
                              const lsm_pages_t* k_pages, const lsm_scales_t* k_scales, const lsm_pages_t* v_pages, const lsm_scales_t* v_scales, const lsm_heads_t* q,
                              const void* q_weight, const lsm_heads_t* q_out, void* stream) {
    int rc = check_rotation(how);
    if (rc != LSM_OK) return rc;
    if (k == nullptr || v == nullptr || to == nullptr || k_pages == nullptr || k_scales == nullptr || v_pages == nullptr || v_scales == nullptr) return LSM_ERR_NULL;
    if (how->n_tokens >= 1u << 24 || to->n_requests >= 1u << 24 || to->n_pages >= 1ull << 31) return LSM_ERR_BAD_ARG;
    if (to->page_tokens == 0 || to->page_tokens % LSM_SCALE_TOKENS != 0 || to->page_tokens >= 1ull << 30 || to->own_width >= 1ull << 30 || to->own_width * to->page_tokens >= 1ull << 30) return LSM_ERR_BAD_ARG;
    if (k->heads != v->heads || k->heads > kMostHeads) return LSM_ERR_BAD_ARG;
    const bool any = how->n_tokens != 0 && to->n_requests != 0 && to->own_width != 0 && to->n_pages != 0 && k->heads != 0;  // anything to append
    if (any && (to->q_offsets == nullptr || to->own_tables == nullptr || to->own_lens == nullptr)) return LSM_ERR_NULL;
    if ((reinterpret_cast<uint64_t>(to->q_offsets) | reinterpret_cast<uint64_t>(to->own_tables) | reinterpret_cast<uint64_t>(to->own_lens)) & 3) return LSM_ERR_BAD_ARG;
    if (reinterpret_cast<uint64_t>(k_weight) & (element_bytes(how->weight_dtype) - 1)) return LSM_ERR_BAD_ARG;
    Append8Args a = {};
    RotateArgs& r = a.rotate;
    if ((rc = set_heads(r.part[0], how, q, q_weight, q_out)) != LSM_OK) return rc;
    if ((rc = set_side(a.side[0], how, k, k_pages, k_scales, any)) != LSM_OK) return rc;
    if ((rc = set_side(a.side[1], how, v, v_pages, v_scales, any)) != LSM_OK) return rc;
    const uint32_t lanes = set_rotation(r, how), each = 16 / element_bytes(how->dtype);
    if (r.part[0].heads != 0) set_slices(r, lanes);
    a.weight = k_weight;
    a.q_offsets = to->q_offsets, a.own_tables = to->own_tables, a.own_lens = to->own_lens, a.own_width = to->own_width;
    a.n_tokens = (uint32_t)how->n_tokens, a.n_requests = (uint32_t)to->n_requests, a.n_pages = (uint32_t)to->n_pages, a.heads = (uint32_t)k->heads;
    a.page_blocks = (uint32_t)(to->page_tokens / LSM_SCALE_TOKENS);
    for (a.first_step = 1; (uint64_t)a.first_step * kWave < to->n_requests;) a.first_step *= kWave;
    a.most = how->dtype == LSM_FP16 ? 61440.f : 0x1.ep127f;  // the largest of 4 significant bits; float32 holds those of bfloat16
    // aligned rows and pairs in whole lanes?
    a.wide = 3;
    for (int i = 0; i < 2; i++) {
        const Side& s = a.side[i];
        const int64_t si[2] = {s.in_token, s.in_head};
        if (!rows_aligned(s.in, si, 2, how->dtype)) a.wide &= ~1u;
        if ((reinterpret_cast<uint64_t>(s.pages) | (uint64_t)s.page | (uint64_t)s.token | (uint64_t)s.head) % each != 0) a.wide &= ~2u;
    }
    const bool aligned = a.wide == 3 && (reinterpret_cast<uint64_t>(r.table) & 15) == 0 && (r.part[0].heads == 0 || r.part[0].wide == 3);
    const int more = how->weight_dtype != how->dtype && k_weight != nullptr ? 3 : 0;
    const int mode = aligned && !r.interleaved && r.rot_dim % (2 * each) == 0 ? more : aligned && r.interleaved && r.rot_dim % each == 0 ? more + 1 : 2;
    // A launch has fewer than 2^32 threads (one of more is cut without an error): more tiles than that take several, the queries go with the first.
    const uint64_t tiles = any ? how->n_tokens / LSM_SCALE_TOKENS + 2 * to->n_requests : 0;
    const uint64_t query_groups = r.part[0].heads != 0 ? (how->n_tokens * r.slices + 3) / 4 : 0;
    const uint64_t most = any ? (kMostBlocks - query_groups) * 4 / (2 * k->heads) : 1;
    if (query_groups >= kMostBlocks / 2 || most == 0) return LSM_ERR_BAD_ARG;
    if (tiles == 0 && query_groups == 0) return LSM_OK;
    for (uint64_t first = 0; first < tiles || (first == 0 && query_groups != 0); first += most) {
        a.first_tile = (uint32_t)first, a.tiles = (uint32_t)(tiles - first < most ? tiles - first : most);
        a.groups = (uint32_t)(((uint64_t)a.tiles * 2 * a.heads + 3) / 4);
        const uint32_t blocks = a.groups + (first == 0 ? (uint32_t)query_groups : 0);
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (how->dtype == LSM_BF16) launch_type<LSM_BF16>(a, lanes, mode, blocks, s);
        else if (how->dtype == LSM_FP16) launch_type<LSM_FP16>(a, lanes, mode, blocks, s);
        else launch_type<LSM_FP32>(a, lanes, mode, blocks, s);
    }
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_HIP;
}
