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

#include "lsm_attention.h"

namespace lsm {

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

template <int kType>
static void join_type(const AttentionArgs& p, uint32_t head, uint32_t joins, hipStream_t stream) {
    if (head == 64) hipLaunchKernelGGL((join_kernel<kType, 64>), dim3(joins), dim3(kThreads), 0, stream, p);
    else if (head == 128) hipLaunchKernelGGL((join_kernel<kType, 128>), dim3(joins), dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((join_kernel<kType, 256>), dim3(joins), dim3(kThreads), 0, stream, p);
}
void launch_join(const AttentionArgs& p, uint32_t dtype, uint32_t head, uint32_t joins, hipStream_t stream) {
    if (dtype == LSM_BF16) join_type<LSM_BF16>(p, head, joins, stream);
    else join_type<LSM_FP16>(p, head, joins, stream);
}

template <int kType, int kHead>
static void launch(const AttentionArgs& p, uint32_t blocks, hipStream_t stream) {
    if (!p.whole) hipLaunchKernelGGL((attention_kernel<kType, kHead, kBoth, AttentionArgs>), dim3(blocks), dim3(kThreads), 0, stream, p);
    else if (p.wide[1]) hipLaunchKernelGGL((attention_kernel<kType, kHead, kWideAlone, AttentionArgs>), dim3(blocks), dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((attention_kernel<kType, kHead, kNarrowAlone, AttentionArgs>), dim3(blocks), dim3(kThreads), 0, stream, p);
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
    const uint32_t blocks = p.items0 + p.tiles[1] * p.combos[1];
    set_attention(a, p, workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (a->dtype == LSM_BF16) launch_type<LSM_BF16>(p, a->head_dim, blocks, s);
    else launch_type<LSM_FP16>(p, a->head_dim, blocks, s);
    if (p.joined) launch_join(p, a->dtype, a->head_dim, (uint32_t)join_blocks(a), s);
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_HIP;
}
