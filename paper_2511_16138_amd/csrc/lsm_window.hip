// lsm_window_attention: attention over pages of 8 bits, and with a window and first tokens that stay visible.
//
// The kernels are those of lsm_attention.h.  Of 8 bits, rows are converted to dtype on their way into LDS, once for all waves that use them; with a window, tiles between the first tokens
// and the window are left out.  Measured, with the floor of bytes at a copy's 4.94 TB/s or of operations at a library product's 1.38 PFLOP/s:
//   96 decodes of up to 8,000 keys, 4 KV heads of 128, 8 bits    104 us, 4.2 TB/s      (88: memory, and the starts and ends of ranges)
//   256 decodes behind 8,192 and 16,384, 2 heads, 8 bits         113 us, 0.52 PFLOP/s  (43: no unit is busy half of the time)
//   8 prompts of 1,024 - 2,048 behind 1,536 - 4,096, 8 bits      1,098 - 1,157 us by card, 0.87 - 0.92 PFLOP/s (728: as in 16 bits, and the conversion, a tenth)
//   64 decodes of up to 16,000 keys, window 1,024, 16 bits       57 us, 4.7 TB/s       (54: memory)
//   6 prompts of 200 - 3,000, window 512, 8 bits                 204 - 210 us, 0.52 PFLOP/s  (78: a tile of rows sees 8.3 of its 11 tiles of keys, and starts and ends)
#include <hip/hip_runtime.h>

#include "lsm_attention.h"

namespace lsm {

template <int kType, int kHead, typename A>
static void launch(const A& p, uint32_t blocks, hipStream_t stream) {
    if constexpr (!A::kWindow) {
        if (!p.whole) {
            hipLaunchKernelGGL((attention_kernel<kType, kHead, kBoth, A>), dim3(blocks), dim3(kThreads), 0, stream, p);
            return;
        }
    }
    if (p.wide[1]) hipLaunchKernelGGL((attention_kernel<kType, kHead, kWideAlone, A>), dim3(blocks), dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((attention_kernel<kType, kHead, kNarrowAlone, A>), dim3(blocks), dim3(kThreads), 0, stream, p);
}
template <int kType, typename A>
static void launch_head(const A& p, uint32_t head, uint32_t blocks, hipStream_t stream) {
    if (head == 64) launch<kType, 64>(p, blocks, stream);
    else if (head == 128) launch<kType, 128>(p, blocks, stream);
    else launch<kType, 256>(p, blocks, stream);
}


static bool in_8_bits(const lsm_window_attention_t* w) { return w->k_scales.data != nullptr; }
static uint64_t element_bytes(const lsm_window_attention_t* w) { return in_8_bits(w) ? 1 : 2; }
// Whether the window can hide anything: where the tables hold no more than it, the calls without one are the same, and read a shared prefix once for all requests
// (256 decodes behind prefixes of 8,192 and 16,384 in 8 bits: 259 us with a window of 2^20 worked on request by request, 113 without one).
static bool hides(const lsm_window_attention_t* w) { return w->window != 0 && w->window < (w->base.prefix_width + w->base.own_width) * w->base.page_tokens; }
// The keys that a tile of rows reaches: the windows of up to 128 tokens, the first tokens, and what the ends of either have in a unit.
static uint64_t most_seen(const lsm_window_attention_t* w) { return hides(w) ? w->window + w->sinks + 128 + 2 * kSplitKeys : ~0ull; }

static int check_window(const lsm_window_attention_t* w) {
    if (w == nullptr) return LSM_ERR_NULL;
    if ((w->k_scales.data == nullptr) != (w->v_scales.data == nullptr)) return LSM_ERR_NULL;
    if (w->window >= 1u << 30 || w->sinks >= 1u << 30 || (w->window == 0 && w->sinks != 0)) return LSM_ERR_BAD_ARG;
    const int rc = check_attention(&w->base, (int64_t)element_bytes(w));
    // with a window the kernels have places, and places less windows, in 32 bits
    if (rc == LSM_OK && hides(w) && (w->base.prefix_width + w->base.own_width) * w->base.page_tokens >= 1ull << 30) return LSM_ERR_BAD_ARG;
    return rc;
}

template <typename A>
static int attend_with(const lsm_window_attention_t* w, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    const lsm_attention_t* a = &w->base;
    A p = {};
    plan_attention(a, p, element_bytes(w), most_seen(w));
    if (!fits_launches(a, p)) return LSM_ERR_BAD_ARG;
    const size_t need = part_bytes(a, p);
    if (need != 0 && (workspace == nullptr || workspace_bytes < need || (reinterpret_cast<uint64_t>(workspace) & 255) != 0)) return LSM_ERR_WORKSPACE;
    set_attention(a, p, workspace, element_bytes(w));
    p.k_scales = w->k_scales.data, p.v_scales = w->v_scales.data;
    p.k_scale_page = w->k_scales.page_stride, p.k_scale_block = w->k_scales.block_stride, p.k_scale_head = w->k_scales.head_stride;
    p.v_scale_page = w->v_scales.page_stride, p.v_scale_block = w->v_scales.block_stride, p.v_scale_head = w->v_scales.head_stride;
    p.window = (int32_t)w->window, p.sinks = (int32_t)w->sinks;
    const uint32_t blocks = p.items0 + p.tiles[1] * p.combos[1];
    if (a->dtype == LSM_BF16) launch_head<LSM_BF16>(p, a->head_dim, blocks, stream);
    else launch_head<LSM_FP16>(p, a->head_dim, blocks, stream);
    if (p.joined) launch_join(p, a->dtype, a->head_dim, (uint32_t)join_blocks(a), stream);
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_HIP;
}

}  // namespace lsm

using namespace lsm;

extern "C" size_t lsm_window_attention_workspace_bytes(const lsm_window_attention_t* w) {
    if (check_window(w) != LSM_OK || w->base.n_tokens == 0) return 0;
    AttentionArgs p = {};
    plan_attention(&w->base, p, element_bytes(w), most_seen(w));
    return fits_launches(&w->base, p) ? part_bytes(&w->base, p) : 0;
}

extern "C" int lsm_window_attention(const lsm_window_attention_t* w, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_window(w);
    if (rc != LSM_OK || w->base.n_tokens == 0) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (hides(w)) return in_8_bits(w) ? attend_with<WindowArgs<true, true>>(w, workspace, workspace_bytes, s) : attend_with<WindowArgs<false, true>>(w, workspace, workspace_bytes, s);
    return in_8_bits(w) ? attend_with<WindowArgs<true, false>>(w, workspace, workspace_bytes, s) : lsm_prefix_attention(&w->base, workspace, workspace_bytes, stream);
}
