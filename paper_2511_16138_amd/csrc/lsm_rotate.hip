// lsm_rope_table, lsm_rotate_heads, lsm_kv_append: norm of each head, position rotation, and the way into the pages of the cache.
#include <hip/hip_runtime.h>

#include "lsm_rotate.h"

namespace lsm {

template <int kType, int kLanes, bool kInterleaved>
__global__ void __launch_bounds__(256) rotate_kernel(const RotateArgs a) {
    rotate_aligned<kType, kLanes, kInterleaved>(a, (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * (blockDim.x / kWave) + threadIdx.x / kWave)));
}
template <int kType, int kLanes>
__global__ void __launch_bounds__(256) rotate_any_kernel(const RotateArgs a) {
    rotate_any<kType, kLanes>(a, (uint64_t)blockIdx.x * (blockDim.x / kWave) + threadIdx.x / kWave);
}

// Angles in 64 bits: at position 10^6 one in 32 bits is off by up to 0.03.
__global__ void __launch_bounds__(256) rope_table_kernel(float* table, uint64_t n, uint32_t half, double log_theta) {
    const uint64_t step = (uint64_t)gridDim.x * blockDim.x;
    for (uint64_t u = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; u < n * half; u += step) {
        const uint64_t p = u / half;
        const uint32_t i = (uint32_t)(u - p * half);
        double s, c;
        sincos((double)p * exp(-(double)i / (double)half * log_theta), &s, &c);
        table[p * 2 * half + i] = (float)c;
        table[p * 2 * half + half + i] = (float)s;
    }
}

// Keys or values that go to pages.
static int set_paged(RotateArgs& a, int part, const lsm_rotation_t* how, const lsm_heads_t* in, const void* weight, const lsm_pages_t* pages) {
    if (in == nullptr || pages == nullptr) return LSM_ERR_NULL;
    const lsm_heads_t out = {pages->data, pages->token_stride, pages->head_stride, in->heads};
    const int rc = set_heads(a.part[part], how, in, weight, &out);
    if (rc != LSM_OK) return rc;
    const int64_t so[3] = {pages->page_stride, pages->token_stride, pages->head_stride};
    a.part[part].wide = (a.part[part].wide & 1) | (rows_aligned(pages->data, so, 3, how->dtype) ? 2u : 0u);
    a.page_stride[part] = pages->page_stride;
    return LSM_OK;
}

template <int kType, int kLanes>
static void launch_lanes(const RotateArgs& a, uint32_t blocks, hipStream_t stream) {
    constexpr uint32_t each = kEach<typename Element<kType>::type>;
    const bool halves_apart = !a.interleaved && a.rot_dim % (2 * each) == 0, neighbours = a.interleaved && a.rot_dim % each == 0;
    bool wide = (reinterpret_cast<uint64_t>(a.table) & 15) == 0;
    for (const HeadsView& v : a.part) wide = wide && (v.heads == 0 || v.wide == 3);
    if (wide && halves_apart) hipLaunchKernelGGL((rotate_kernel<kType, kLanes, false>), dim3(blocks), dim3(256), 0, stream, a);
    else if (wide && neighbours) hipLaunchKernelGGL((rotate_kernel<kType, kLanes, true>), dim3(blocks), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((rotate_any_kernel<kType, kLanes>), dim3(blocks), dim3(256), 0, stream, a);
}
template <int kType>
static void launch_type(const RotateArgs& a, uint32_t lanes, uint32_t blocks, hipStream_t stream) {
    if (lanes == 8) launch_lanes<kType, 8>(a, blocks, stream);
    else if (lanes == 16) launch_lanes<kType, 16>(a, blocks, stream);
    else if (lanes == 32) launch_lanes<kType, 32>(a, blocks, stream);
    else launch_lanes<kType, 64>(a, blocks, stream);
}

static int launch_rotate(RotateArgs& a, const lsm_rotation_t* how, hipStream_t stream) {
    const uint32_t lanes = set_rotation(a, how);
    if (a.part[0].heads + a.part[1].heads + a.part[2].heads == 0 || a.n_tokens == 0) return LSM_OK;
    set_slices(a, lanes);
    // A launch has fewer than 2^32 threads (one of more is cut without an error): more tokens than that, 64 threads each, take several.
    const uint64_t all = a.n_tokens, most = kMostBlocks * 4 / a.slices;
    for (uint64_t first = 0; first < all; first += most) {
        a.n_tokens = all - first < most ? all - first : most;
        const uint32_t blocks = (uint32_t)((a.n_tokens * a.slices + 3) / 4);
        if (how->dtype == LSM_BF16) launch_type<LSM_BF16>(a, lanes, blocks, stream);
        else if (how->dtype == LSM_FP16) launch_type<LSM_FP16>(a, lanes, blocks, stream);
        else launch_type<LSM_FP32>(a, lanes, blocks, stream);
        for (int p = 0; p < 3; p++) {
            HeadsView& v = a.part[p];
            const int64_t step = (int64_t)a.n_tokens * element_bytes(how->dtype);
            v.in = static_cast<const char*>(v.in) + step * v.in_token;
            if (p == 0 || a.slots == nullptr) v.out = static_cast<char*>(v.out) + step * v.out_token;  // keys and values go to pages otherwise
        }
        if (a.positions != nullptr) a.positions += a.n_tokens;
        if (a.slots != nullptr) a.slots += a.n_tokens;
    }
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_HIP;
}

}  // namespace lsm

using namespace lsm;

extern "C" int lsm_rope_table(float* table, uint64_t n_positions, uint32_t rot_dim, double theta, void* stream) {
    if (rot_dim == 0 || rot_dim % 2 != 0 || rot_dim > LSM_MAX_HEAD_DIM || !(theta > 0.0) || !(theta < __builtin_inf()) || n_positions >= 1ull << 31) return LSM_ERR_BAD_ARG;
    if (n_positions == 0) return LSM_OK;
    if (table == nullptr) return LSM_ERR_NULL;
    if (reinterpret_cast<uint64_t>(table) & 3) return LSM_ERR_BAD_ARG;
    uint64_t blocks = (n_positions * (rot_dim / 2) + 255) / 256;
    if (blocks > 8192) blocks = 8192;
    hipLaunchKernelGGL(rope_table_kernel, dim3((uint32_t)blocks), dim3(256), 0, static_cast<hipStream_t>(stream), table, n_positions, rot_dim / 2, __builtin_log(theta));
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_HIP;
}

extern "C" int lsm_rotate_heads(const lsm_rotation_t* how, const lsm_heads_t* q, const void* q_weight, const lsm_heads_t* q_out,
                                const lsm_heads_t* k, const void* k_weight, const lsm_heads_t* k_out, void* stream) {
    int rc = check_rotation(how);
    if (rc != LSM_OK) return rc;
    RotateArgs a = {};
    if ((rc = set_heads(a.part[0], how, q, q_weight, q_out)) != LSM_OK) return rc;
    if ((rc = set_heads(a.part[1], how, k, k_weight, k_out)) != LSM_OK) return rc;
    return launch_rotate(a, how, static_cast<hipStream_t>(stream));
}

extern "C" int lsm_kv_append(const lsm_rotation_t* how, const lsm_heads_t* k, const void* k_weight, const lsm_heads_t* v, const int64_t* slots,
                             const lsm_pages_t* k_pages, const lsm_pages_t* v_pages, uint64_t n_pages, uint64_t page_tokens, const lsm_heads_t* q,
                             const void* q_weight, const lsm_heads_t* q_out, void* stream) {
    int rc = check_rotation(how);
    if (rc != LSM_OK) return rc;
    RotateArgs a = {};
    if (page_tokens == 0 || page_tokens >= 1ull << 31 || n_pages >= 1ull << 31) return LSM_ERR_BAD_ARG;
    if (slots == nullptr && how->n_tokens != 0) return LSM_ERR_NULL;
    if (reinterpret_cast<uint64_t>(slots) & 7) return LSM_ERR_BAD_ARG;
    if ((rc = set_heads(a.part[0], how, q, q_weight, q_out)) != LSM_OK) return rc;
    if ((rc = set_paged(a, 1, how, k, k_weight, k_pages)) != LSM_OK) return rc;
    if ((rc = set_paged(a, 2, how, v, nullptr, v_pages)) != LSM_OK) return rc;
    if (k->heads != v->heads) return LSM_ERR_BAD_ARG;
    a.slots = slots, a.page_tokens = page_tokens, a.n_slots = n_pages * page_tokens;
    a.page_shift = (page_tokens & (page_tokens - 1)) == 0 ? (uint32_t)__builtin_ctzll(page_tokens) : 64;
    return launch_rotate(a, how, static_cast<hipStream_t>(stream));
}
