// Norm of each head and position rotation: what the kernels of lsm_rotate.hip and lsm_append8.hip have in common.
#pragma once
#include <hip/hip_runtime.h>

#include "lsm_cache.h"
#include "lsm_common.h"

namespace lsm {

// ---------------------------------------------------------------------------------------------------------------------
// elements
// ---------------------------------------------------------------------------------------------------------------------
template <int kType>
struct Element;
template <>
struct Element<LSM_BF16> {
    typedef __bf16 type;
};
template <>
struct Element<LSM_FP16> {
    typedef _Float16 type;
};
template <>
struct Element<LSM_FP32> {
    typedef float type;
};

template <typename T>
constexpr int kEach = 16 / (int)sizeof(T);  // elements of a lane: 16 bytes

template <typename T>
struct Lane {
    typedef T vec __attribute__((ext_vector_type(kEach<T>)));
    vec v;
};

// A lane's elements as they are, in 16-byte words or one by one.
template <typename T>
__device__ __forceinline__ Lane<T> load_lane(const T* p, bool wide) {
    Lane<T> r;
    if (wide) {
        r.v = *reinterpret_cast<const typename Lane<T>::vec*>(p);
    } else {
#pragma unroll
        for (int j = 0; j < kEach<T>; j++) r.v[j] = p[j];
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void store_lane(T* p, const Lane<T>& r, bool wide) {
    if (wide) {
        *reinterpret_cast<typename Lane<T>::vec*>(p) = r.v;
    } else {
#pragma unroll
        for (int j = 0; j < kEach<T>; j++) p[j] = r.v[j];
    }
}

struct HeadsView {
    const void* in;
    void* out;
    const void* weight;
    int64_t in_token, in_head, out_token, out_head;  // elements
    uint32_t heads;
    uint32_t wide;  // bit 0: the input's rows are 16-byte aligned, bit 1: the output's
};

struct RotateArgs {
    HeadsView part[3];  // queries, keys, values; the outputs of keys and values are pages where `slots` is given
    const int32_t* positions;
    const float* table;
    const int64_t* slots;
    int64_t page_stride[3];
    uint64_t n_tokens, n_positions, n_slots, page_tokens;
    uint32_t page_shift;  // log2(page_tokens), or 64 where it is no power of two
    uint32_t head_dim, rot_dim, interleaved, weight_fp32;
    uint32_t slices, heads_per_slice;  // a token's heads are dealt to this many waves
    float eps;
};

// The rotation in its ordinary form: rows and table 16-byte aligned, and the other element of a pair in the lane itself
// (neighbouring elements) or a whole number of lanes away (halves apart).
//
// One wave takes heads_per_slice of a token's heads (queries, keys and values counted through), 64 / kLanes of them at a time:
// kLanes lanes of 16 bytes hold a head.  The angles belong to the token and the weights to all, so a lane reads them once and keeps
// them for all its heads; four heads' loads are under way before the first is worked on.  Bound by memory: every input is
// read once and every output written once.  Measured: 8,192 tokens of 40 heads of 128 in 37 us (4.6 TB/s; a copy 4.9), 16,384 of 48 into pages in 82 (5.0), 8 tokens
// of 34 heads in 3.5.  The loads ahead of slot, position and angles: 8,192 tokens 34 -> 40 us (inputs in the last-level cache).
// A wave waits for slot, position, angles and either weight one after the other, and asks for its first heads after that; where it has few heads that is a
// third of the time: 5,001 tokens of 24 heads of 64 in 9.0 us, 5.9 by their bytes.
template <int kType, int kLanes, bool kInterleaved>
__device__ __forceinline__ void rotate_aligned(const RotateArgs& a, uint32_t wave) {
    typedef typename Element<kType>::type T;
    constexpr int E = kEach<T>;
    constexpr uint32_t kHeads = kWave / kLanes;  // heads at a time
    constexpr uint32_t kAhead = 4;               // of these that are read before the first is worked on
    const uint32_t token = wave / a.slices;
    if (token >= a.n_tokens) return;
    const uint32_t lane = threadIdx.x & (kWave - 1), sub = lane / kLanes, e0 = (lane & (kLanes - 1)) * E;
    const uint32_t first = (wave - token * a.slices) * a.heads_per_slice;
    const uint32_t heads_q = a.part[0].heads, heads_qk = heads_q + a.part[1].heads, heads_all = heads_qk + a.part[2].heads;
    const uint32_t end = min(first + a.heads_per_slice, heads_all);
    const bool inside = e0 < a.head_dim, turns = e0 < a.rot_dim;
    const uint32_t half = a.rot_dim >> 1;
    const T* in[3];
    T* out[3];
    bool kept = true;
    uint64_t page = 0, row = token;
    if (a.slots != nullptr) {
        const int64_t slot = a.slots[token];
        kept = slot >= 0 && (uint64_t)slot < a.n_slots;
        const uint64_t at = kept ? (uint64_t)slot : 0;
        page = a.page_shift < 64 ? at >> a.page_shift : at / a.page_tokens;
        row = at - page * a.page_tokens;
    }
#pragma unroll
    for (int p = 0; p < 3; p++) {
        in[p] = static_cast<const T*>(a.part[p].in) + (int64_t)token * a.part[p].in_token;
        out[p] = static_cast<T*>(a.part[p].out) + (p == 0 ? (int64_t)token * a.part[p].out_token : (int64_t)page * a.page_stride[p] + (int64_t)row * a.part[p].out_token);
    }
    // the lane's angles: a' = a cos - b sin, b' = b cos + a sin, as own * cosine + other * sine
    float cosine[E], sine[E];
    if (turns) {
        const int32_t p = a.positions[token];
        const bool known = p >= 0 && (uint64_t)p < a.n_positions;
        const float* angles = a.table + (known ? (uint64_t)p : 0) * a.rot_dim;
        if (kInterleaved) {
            typedef float few __attribute__((ext_vector_type(E / 2)));
            const few c = *reinterpret_cast<const few*>(angles + e0 / 2), s = *reinterpret_cast<const few*>(angles + half + e0 / 2);
#pragma unroll
            for (int j = 0; j < E; j++) cosine[j] = c[j / 2], sine[j] = j & 1 ? s[j / 2] : -s[j / 2];
        } else {
            const uint32_t i = e0 < half ? e0 : e0 - half;
#pragma unroll
            for (int j = 0; j < E; j += 4) {
                const float4 c = *reinterpret_cast<const float4*>(angles + i + j), s = *reinterpret_cast<const float4*>(angles + half + i + j);
                cosine[j] = c.x, cosine[j + 1] = c.y, cosine[j + 2] = c.z, cosine[j + 3] = c.w;
                sine[j] = s.x, sine[j + 1] = s.y, sine[j + 2] = s.z, sine[j + 3] = s.w;
            }
#pragma unroll
            for (int j = 0; j < E; j++) sine[j] = e0 < half ? -sine[j] : sine[j];
        }
        if (!known) {
#pragma unroll
            for (int j = 0; j < E; j++) cosine[j] = __builtin_nanf("");
        }
    } else {
#pragma unroll
        for (int j = 0; j < E; j++) cosine[j] = 1.f, sine[j] = 0.f;
    }
    float weight[2][E];
#pragma unroll
    for (int p = 0; p < 2; p++) {
        const void* w = a.part[p].weight;
        if (w != nullptr && inside) {
            if (sizeof(T) == 4 || a.weight_fp32) {
#pragma unroll
                for (int j = 0; j < E; j++) weight[p][j] = static_cast<const float*>(w)[e0 + j];
            } else {
#pragma unroll
                for (int j = 0; j < E; j++) weight[p][j] = (float)static_cast<const T*>(w)[e0 + j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < E; j++) weight[p][j] = 1.f;
        }
    }
    const bool normed[2] = {a.part[0].weight != nullptr, a.part[1].weight != nullptr};
    const float mean_by = 1.f / (float)a.head_dim;
    // halves apart: the lane that has the other element of each of this lane's pairs
    const int other = turns ? (int)(e0 < half ? lane + half / E : lane - half / E) : (int)lane;
    for (uint32_t at = first; at < end; at += kHeads * kAhead) {
        Lane<T> raw[kAhead];
#pragma unroll
        for (uint32_t u = 0; u < kAhead; u++) {
            const uint32_t h = at + u * kHeads + sub;
            if (h < end && inside) {
                const T* from = h < heads_q ? in[0] + (int64_t)h * a.part[0].in_head
                                : h < heads_qk ? in[1] + (int64_t)(h - heads_q) * a.part[1].in_head
                                               : in[2] + (int64_t)(h - heads_qk) * a.part[2].in_head;
                raw[u] = load_lane<T>(from + e0, true);
            } else {
#pragma unroll
                for (int j = 0; j < E; j++) raw[u].v[j] = (T)0.f;
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < kAhead; u++) {
            if (at + u * kHeads >= end) break;
            const uint32_t h = at + u * kHeads + sub;
            const bool query = h < heads_q;
            float y[E];
#pragma unroll
            for (int j = 0; j < E; j++) y[j] = (float)raw[u].v[j];
            if (normed[0] || normed[1]) {
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < E; j++) sum += y[j] * y[j];
#pragma unroll
                for (int off = 1; off < kLanes; off <<= 1) sum += __shfl_xor(sum, off, kWave);
                const float by = __builtin_amdgcn_rsqf(sum * mean_by + a.eps);
                if (query ? normed[0] : normed[1]) {
#pragma unroll
                    for (int j = 0; j < E; j++) y[j] *= by * (query ? weight[0][j] : weight[1][j]);
                }
            }
            if (a.table != nullptr) {
                float z[E];
#pragma unroll
                for (int j = 0; j < E; j++) z[j] = kInterleaved ? y[j ^ 1] : __shfl(y[j], other, kWave);
                if (turns) {
#pragma unroll
                    for (int j = 0; j < E; j++) y[j] = y[j] * cosine[j] + z[j] * sine[j];
                }
            }
            if (h < end && inside) {
                Lane<T> done = raw[u];
                if (h < heads_qk) {
#pragma unroll
                    for (int j = 0; j < E; j++) done.v[j] = (T)y[j];
                }
                T* to = query ? out[0] + (int64_t)h * a.part[0].out_head
                        : h < heads_qk ? out[1] + (int64_t)(h - heads_q) * a.part[1].out_head
                                       : out[2] + (int64_t)(h - heads_qk) * a.part[2].out_head;
                if (query || kept) store_lane<T>(to + e0, done, true);
            }
        }
    }
}

// The same for any alignment and any rot_dim: elements one by one where rows are not aligned, and the other element of a pair read
// again where it is in no whole lane.
template <int kType, int kLanes>
__device__ __forceinline__ void rotate_any(const RotateArgs& a, uint64_t wave) {
    typedef typename Element<kType>::type T;
    constexpr int E = kEach<T>;
    constexpr uint32_t kHeads = kWave / kLanes, kAhead = 2;
    const uint64_t token = wave / a.slices;
    if (token >= a.n_tokens) return;
    const uint32_t lane = threadIdx.x & (kWave - 1), part_lane = lane & (kLanes - 1), sub = lane / kLanes;
    const uint32_t first = (uint32_t)(wave - token * a.slices) * a.heads_per_slice;
    const uint32_t heads_q = a.part[0].heads, heads_qk = heads_q + a.part[1].heads, heads_all = heads_qk + a.part[2].heads;
    const uint32_t end = min(first + a.heads_per_slice, heads_all);
    const uint32_t e0 = part_lane * E;
    const bool inside = e0 < a.head_dim;
    const uint32_t half = a.rot_dim >> 1;
    // the lane's angles
    float cosine[E], sine[E];
    const bool turns = a.table != nullptr && inside && e0 < a.rot_dim;
#pragma unroll
    for (int j = 0; j < E; j++) cosine[j] = 1.f, sine[j] = 0.f;
    if (turns) {
        const int32_t p = a.positions[token];
        const bool known = p >= 0 && (uint64_t)p < a.n_positions;
        const float* row = a.table + (known ? (uint64_t)p : 0) * a.rot_dim;
#pragma unroll
        for (int j = 0; j < E; j++) {
            const uint32_t e = e0 + j;
            if (e < a.rot_dim) {
                const uint32_t i = a.interleaved ? e >> 1 : (e < half ? e : e - half);
                const float s = row[half + i];
                cosine[j] = known ? row[i] : __builtin_nanf("");
                sine[j] = (a.interleaved ? (e & 1) : e >= half) ? s : -s;  // a' = a cos - b sin, b' = b cos + a sin
            }
        }
    }
    // halves apart: the other element of a pair is in the lane half / E further, or back, where that is whole; otherwise it is read again
    const bool by_lane = half % E == 0;
    const int other = e0 < half ? (int)(lane + half / E) : (int)(lane - half / E);
    uint64_t slot_row = 0, slot_page = 0;
    bool kept = true;
    if (a.slots != nullptr) {
        const int64_t slot = a.slots[token];
        kept = slot >= 0 && (uint64_t)slot < a.n_slots;
        if (kept) {
            slot_page = a.page_shift < 64 ? (uint64_t)slot >> a.page_shift : (uint64_t)slot / a.page_tokens;
            slot_row = (uint64_t)slot - slot_page * a.page_tokens;
        }
    }
    for (uint32_t at = first; at < end; at += kHeads * kAhead) {
        Lane<T> raw[kAhead];
        const T* from[kAhead];
        uint32_t which[kAhead], head[kAhead];
#pragma unroll
        for (uint32_t u = 0; u < kAhead; u++) {
            const uint32_t h = at + u * kHeads + sub;
            which[u] = h >= end ? 3 : h < heads_q ? 0 : h < heads_qk ? 1 : 2;
            head[u] = h - (which[u] == 0 ? 0 : which[u] == 1 ? heads_q : heads_qk);
            const HeadsView& v = a.part[which[u] < 3 ? which[u] : 0];
            from[u] = static_cast<const T*>(v.in) + (int64_t)token * v.in_token + (int64_t)head[u] * v.in_head + e0;
            if (which[u] < 3 && inside) {
                raw[u] = load_lane<T>(from[u], v.wide & 1);
            } else {
#pragma unroll
                for (int j = 0; j < E; j++) raw[u].v[j] = (T)0.f;
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < kAhead; u++) {
            const uint32_t w = which[u];
            const HeadsView& v = a.part[w < 3 ? w : 0];
            Lane<T> done = raw[u];
            float x[E], weight[E];
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < E; j++) x[j] = (float)raw[u].v[j], sum += x[j] * x[j];
#pragma unroll
            for (int off = 1; off < kLanes; off <<= 1) sum += __shfl_xor(sum, off, kWave);
            const bool normed = w < 2 && v.weight != nullptr;
            const float by = normed ? 1.f / sqrtf(sum / (float)a.head_dim + a.eps) : 1.f;
            if (normed && inside) {
#pragma unroll
                for (int j = 0; j < E; j++) weight[j] = a.weight_fp32 ? static_cast<const float*>(v.weight)[e0 + j] : (float)static_cast<const T*>(v.weight)[e0 + j];
            } else {
#pragma unroll
                for (int j = 0; j < E; j++) weight[j] = 1.f;
            }
            float y[E], z[E];
#pragma unroll
            for (int j = 0; j < E; j++) y[j] = x[j] * by * weight[j];
            if (a.table != nullptr) {
                if (a.interleaved) {
#pragma unroll
                    for (int j = 0; j < E; j++) z[j] = y[j ^ 1];
                } else if (by_lane) {
#pragma unroll
                    for (int j = 0; j < E; j++) z[j] = __shfl(y[j], other, kWave);
                } else {
#pragma unroll
                    for (int j = 0; j < E; j++) {
                        z[j] = 0.f;
                        const uint32_t e = e0 + j;
                        if (w < 2 && inside && e < a.rot_dim) {
                            const int to = e < half ? (int)half : -(int)half;
                            const float f = !normed ? 1.f : a.weight_fp32 ? static_cast<const float*>(v.weight)[(int)e + to] : (float)static_cast<const T*>(v.weight)[(int)e + to];
                            z[j] = (float)from[u][j + to] * by * f;
                        }
                    }
                }
            }
            if (w < 2) {
#pragma unroll
                for (int j = 0; j < E; j++) done.v[j] = (T)(turns && e0 + j < a.rot_dim ? y[j] * cosine[j] + z[j] * sine[j] : y[j]);
            }
            if (w < 3 && inside) {
                T* to = static_cast<T*>(v.out) + (int64_t)head[u] * v.out_head + e0;
                if (w > 0 && a.slots != nullptr) {
                    if (!kept) continue;
                    to += (int64_t)slot_page * a.page_stride[w] + (int64_t)slot_row * v.out_token;
                } else {
                    to += (int64_t)token * v.out_token;
                }
                store_lane<T>(to, done, v.wide & 2);
            }
        }
    }
}

static inline uint32_t element_bytes(uint32_t dtype) { return dtype == LSM_FP32 ? 4 : 2; }

static inline bool rows_aligned(const void* data, const int64_t* strides, int n, uint32_t dtype) {
    uint64_t bits = reinterpret_cast<uint64_t>(data);
    for (int i = 0; i < n; i++) bits |= (uint64_t)strides[i] * element_bytes(dtype);
    return (bits & 15) == 0;
}

static inline int check_rotation(const lsm_rotation_t* how) {
    if (how == nullptr) return LSM_ERR_NULL;
    if (how->dtype > LSM_FP32 || (how->weight_dtype != how->dtype && how->weight_dtype != LSM_FP32) || how->interleaved > 1) return LSM_ERR_BAD_ARG;
    if (how->head_dim == 0 || how->head_dim % 8 != 0 || how->head_dim > LSM_MAX_HEAD_DIM) return LSM_ERR_BAD_ARG;
    if (how->n_tokens >= 1ull << 31 || !(how->eps >= 0.f)) return LSM_ERR_BAD_ARG;
    if (how->table != nullptr) {
        if (how->rot_dim == 0 || how->rot_dim % 2 != 0 || how->rot_dim > how->head_dim || how->n_positions >= 1ull << 31) return LSM_ERR_BAD_ARG;
        if (how->n_positions == 0 && how->n_tokens != 0) return LSM_ERR_BAD_ARG;
        if (how->positions == nullptr && how->n_tokens != 0) return LSM_ERR_NULL;
        if ((reinterpret_cast<uint64_t>(how->table) | reinterpret_cast<uint64_t>(how->positions)) & 3) return LSM_ERR_BAD_ARG;
    }
    return LSM_OK;
}

constexpr uint64_t kMostHeads = 1u << 16;
constexpr uint64_t kMostBlocks = (1ull << 24) - 1;  // of 256 threads

// One of the parts with an output of its own: queries, or keys of lsm_rotate_heads.
static inline int set_heads(HeadsView& v, const lsm_rotation_t* how, const lsm_heads_t* in, const void* weight, const lsm_heads_t* out) {
    if (in == nullptr || in->heads == 0) return LSM_OK;
    if (out == nullptr) return LSM_ERR_NULL;
    if (in->heads > kMostHeads || out->heads != in->heads) return LSM_ERR_BAD_ARG;
    if (how->n_tokens != 0 && (in->data == nullptr || out->data == nullptr)) return LSM_ERR_NULL;
    const uint64_t mask = element_bytes(how->dtype) - 1;
    if ((reinterpret_cast<uint64_t>(in->data) | reinterpret_cast<uint64_t>(out->data)) & mask) return LSM_ERR_BAD_ARG;
    if (reinterpret_cast<uint64_t>(weight) & (element_bytes(how->weight_dtype) - 1)) return LSM_ERR_BAD_ARG;
    const int64_t si[2] = {in->token_stride, in->head_stride}, so[2] = {out->token_stride, out->head_stride};
    v = HeadsView{in->data, out->data, weight, in->token_stride, in->head_stride, out->token_stride, out->head_stride, (uint32_t)in->heads,
                  (rows_aligned(in->data, si, 2, how->dtype) ? 1u : 0u) | (rows_aligned(out->data, so, 2, how->dtype) ? 2u : 0u)};
    return LSM_OK;
}

// What a launch goes by besides its heads; the lanes that hold a head.
static inline uint32_t set_rotation(RotateArgs& a, const lsm_rotation_t* how) {
    a.positions = how->positions, a.table = how->table, a.n_positions = how->n_positions, a.n_tokens = how->n_tokens;
    a.head_dim = how->head_dim, a.rot_dim = how->table ? how->rot_dim : 0, a.interleaved = how->interleaved;
    a.weight_fp32 = how->weight_dtype == LSM_FP32, a.eps = how->eps;
    uint32_t lanes = 8;
    while (lanes * 16 < a.head_dim * element_bytes(how->dtype)) lanes *= 2;
    return lanes;
}

// How a token's heads are dealt to waves; there are some.
static inline void set_slices(RotateArgs& a, uint32_t lanes) {
    const uint32_t heads = a.part[0].heads + a.part[1].heads + a.part[2].heads, at_once = kWave / lanes, rounds = (heads + at_once - 1) / at_once;
    // few tokens: more waves per token, down to one round of heads each
    uint32_t slices = 1;
    while (slices < rounds && a.n_tokens * slices < 4096) slices *= 2;
    const uint32_t each = (rounds + slices - 1) / slices;
    a.heads_per_slice = each * at_once;
    a.slices = (heads + a.heads_per_slice - 1) / a.heads_per_slice;
}

}  // namespace lsm
