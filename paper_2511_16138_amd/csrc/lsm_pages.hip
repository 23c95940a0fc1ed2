// lsm_copy_pages, lsm_compact_pages: pages copied within their buffers, and the live ones moved together.
#include <hip/hip_runtime.h>

#include "lsm_common.h"
#include "lsm_pages.h"

namespace lsm {

constexpr uint32_t kCopyThreads = 256, kCopyAhead = 4;
constexpr uint32_t kChunk = kCopyThreads * kCopyAhead * 16;  // bytes that a workgroup copies at a time
constexpr uint32_t kLaunchParts = 64;                        // buffers of a launch: one for each lane
constexpr uint32_t kCopyGroups = 4096;                       // workgroups of a launch at most: 16 on each compute unit; they take turns

struct Part {
    char* data;
    int64_t stride;
    uint64_t bytes;
    uint32_t first_chunk;  // chunks of a page are counted through its parts
    uint32_t wide;         // 16-byte words
};

struct CopyArgs {
    Part part[kLaunchParts];
    const int32_t *sources, *targets;
    const uint32_t* n_pairs;  // DEVICE; nullptr: `pairs` of them
    uint64_t pairs;
    uint32_t parts, chunks, n_pages;
};

// A workgroup copies chunk after chunk: a launch has enough of them for the chip, however many pairs there are, which the host need not know.
// Four words a lane are under way at a time.  Bound by memory: every byte is read once and written once.
__device__ __forceinline__ void copy_chunks(const CopyArgs& a, uint32_t group, uint32_t groups) {
    const uint32_t lane = threadIdx.x & (kWave - 1);
    const uint32_t first = lane < a.parts ? a.part[lane].first_chunk : ~0u;
    const uint64_t pairs = a.n_pairs != nullptr ? *a.n_pairs : a.pairs, all = pairs * a.chunks;
    for (uint64_t item = group; item < all; item += groups) {
        const uint64_t pair = item / a.chunks;
        const uint32_t chunk = (uint32_t)(item - pair * a.chunks);
        const uint32_t p = (uint32_t)__builtin_amdgcn_readfirstlane(__popcll(__ballot(first <= chunk)) - 1);
        const uint32_t from = (uint32_t)a.sources[pair], to = (uint32_t)a.targets[pair];
        if (from >= a.n_pages || to >= a.n_pages || from == to) continue;
        const Part& part = a.part[p];
        const uint64_t at = (uint64_t)(chunk - part.first_chunk) * kChunk, left = part.bytes - at;
        const char* in = part.data + (int64_t)from * part.stride + at;
        char* out = part.data + (int64_t)to * part.stride + at;
        if (part.wide) {
            uint4 v[kCopyAhead];
#pragma unroll
            for (uint32_t i = 0; i < kCopyAhead; i++) {
                const uint32_t b = (i * kCopyThreads + threadIdx.x) * 16;
                if (b < left) v[i] = *reinterpret_cast<const uint4*>(in + b);
            }
#pragma unroll
            for (uint32_t i = 0; i < kCopyAhead; i++) {
                const uint32_t b = (i * kCopyThreads + threadIdx.x) * 16;
                if (b < left) *reinterpret_cast<uint4*>(out + b) = v[i];
            }
        } else {
            const uint32_t end = left < kChunk ? (uint32_t)left : kChunk;
            for (uint32_t b = threadIdx.x; b < end; b += kCopyThreads) out[b] = in[b];
        }
    }
}

__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const CopyArgs a) { copy_chunks(a, blockIdx.x, gridDim.x); }

// ---------------------------------------------------------------------------------------------------------------------
// compaction
// ---------------------------------------------------------------------------------------------------------------------
struct Table {
    const int32_t *pages, *lens;
    int32_t* new_pages;
    uint64_t entries, width;
};
struct Tables {
    Table table[LSM_MAX_PAGE_TABLES];
    uint64_t page_tokens;
    uint32_t tables, n_pages;
};

// f(table, entry, page) for each entry of every table: page is what it holds, ~0 where it holds none.
template <typename F>
__device__ __forceinline__ void each_entry(const Tables& a, uint64_t thread, uint64_t threads, F f) {
    for (uint32_t t = 0; t < a.tables; t++) {
        const Table& table = a.table[t];
        for (uint64_t e = thread; e < table.entries; e += threads) {
            const uint64_t row = e / table.width, column = e - row * table.width;
            const int32_t len = table.lens[row];
            const uint32_t page = (uint32_t)table.pages[e];
            f(table, e, len > 0 && column * a.page_tokens < (uint64_t)len && page < a.n_pages ? page : ~0u);
        }
    }
}

constexpr uint32_t kPlanThreads = 1024;

struct PlanArgs {
    uint32_t* live;  // a bit a page
    int32_t *sources, *targets;
    uint32_t* n_moves;
    int32_t *moved, *n_live;
    uint32_t n_pages;
};

__global__ void __launch_bounds__(256) clear_kernel(uint32_t* live, uint32_t words) {
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < words; i += gridDim.x * 256) live[i] = 0;
}
__global__ void __launch_bounds__(256) mark_kernel(const Tables a, uint32_t* live) {
    each_entry(a, (uint64_t)blockIdx.x * 256 + threadIdx.x, (uint64_t)gridDim.x * 256, [&](const Table&, uint64_t, uint32_t page) {
        if (page != ~0u) atomicOr(&live[page >> 5], 1u << (page & 31));
    });
}

// The sum of x over the threads before this one, and over all.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t* lds, uint32_t& all) {
    const uint32_t lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    uint32_t sum = x;
#pragma unroll
    for (uint32_t off = 1; off < kWave; off <<= 1) {
        const uint32_t y = __shfl_up(sum, off, kWave);
        if (lane >= off) sum += y;
    }
    __syncthreads();
    if (lane == kWave - 1) lds[wave] = sum;
    __syncthreads();
    uint32_t before = 0;
    all = 0;
    for (uint32_t i = 0; i < kPlanThreads / kWave; i++) {
        if (i < wave) before += lds[i];
        all += lds[i];
    }
    return before + sum - x;
}

// One workgroup: counts the live pages, then numbers the free ones below that count and the live ones from it on, both in ascending order; the k-th of
// either make a move.
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanArgs a) {
    __shared__ uint32_t lds[kPlanThreads / kWave];
    const uint32_t words = (a.n_pages + 31) / 32, each = (words + kPlanThreads - 1) / kPlanThreads;
    const uint32_t begin = min(threadIdx.x * each, words), end = min(begin + each, words);
    uint32_t count = 0, n_live, n_holes, n_moves;
    for (uint32_t i = begin; i < end; i++) count += __popc(a.live[i]);
    sum_before(count, lds, n_live);
    auto below = [&](uint32_t word) {  // the bits of a word that are of pages below n_live
        const uint32_t first = word * 32;
        return first >= n_live ? 0 : n_live - first >= 32 ? ~0u : (1u << (n_live - first)) - 1;
    };
    uint32_t holes = 0, movers = 0;
    for (uint32_t i = begin; i < end; i++) {
        const uint32_t live = a.live[i], low = below(i);
        holes += __popc(~live & low), movers += __popc(live & ~low);
    }
    uint32_t hole = sum_before(holes, lds, n_holes), mover = sum_before(movers, lds, n_moves);
    for (uint32_t i = begin; i < end; i++) {
        const uint32_t live = a.live[i], low = below(i);
        for (uint32_t bits = ~live & low; bits != 0; bits &= bits - 1) a.targets[hole++] = (int32_t)(i * 32 + __builtin_ctz(bits));
        for (uint32_t bits = live & ~low; bits != 0; bits &= bits - 1) a.sources[mover++] = (int32_t)(i * 32 + __builtin_ctz(bits));
    }
    for (uint32_t p = threadIdx.x; p < a.n_pages; p += kPlanThreads) {
        const bool live = (a.live[p >> 5] >> (p & 31)) & 1;
        if (!live || p < n_live) a.moved[p] = live ? (int32_t)p : -1;
    }
    __syncthreads();  // the lists are written
    for (uint32_t i = threadIdx.x; i < n_moves; i += kPlanThreads) a.moved[a.sources[i]] = a.targets[i];
    if (threadIdx.x == 0) *a.n_moves = n_moves, *a.n_live = (int32_t)n_live;
}

// Sources are all at or above n_live and targets all below it, so pages move in any order.
__global__ void __launch_bounds__(kCopyThreads) move_kernel(const CopyArgs copies, const Tables tables, const int32_t* moved, uint32_t table_groups) {
    if (blockIdx.x < table_groups) {
        each_entry(tables, (uint64_t)blockIdx.x * kCopyThreads + threadIdx.x, (uint64_t)table_groups * kCopyThreads,
                   [&](const Table& t, uint64_t e, uint32_t page) { t.new_pages[e] = page == ~0u ? t.pages[e] : moved[page]; });
    } else {
        copy_chunks(copies, blockIdx.x - table_groups, gridDim.x - table_groups);
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------------
static int check_parts(const lsm_page_part_t* parts, uint64_t n_parts, uint64_t n_pages) {
    if (n_parts > LSM_MAX_PAGE_PARTS || n_pages >= 1ull << 30) return LSM_ERR_BAD_ARG;
    if (n_parts != 0 && parts == nullptr) return LSM_ERR_NULL;
    for (uint64_t i = 0; i < n_parts; i++) {
        if (parts[i].page_bytes >= 1ull << 36) return LSM_ERR_BAD_ARG;
        if (parts[i].data == nullptr && parts[i].page_bytes != 0 && n_pages != 0) return LSM_ERR_NULL;
    }
    return LSM_OK;
}

// The next buffers that fit a launch, from `at` on; false: there are none.
static bool next_parts(CopyArgs& a, const lsm_page_part_t* parts, uint64_t n_parts, uint64_t& at) {
    a.parts = 0, a.chunks = 0;
    for (; at < n_parts && a.parts < kLaunchParts; at++) {
        const lsm_page_part_t& p = parts[at];
        if (p.page_bytes == 0) continue;
        const uint64_t bits = reinterpret_cast<uint64_t>(p.data) | (uint64_t)p.page_stride | p.page_bytes;
        a.part[a.parts++] = Part{static_cast<char*>(p.data), p.page_stride, p.page_bytes, a.chunks, (bits & 15) == 0};
        a.chunks += (uint32_t)((p.page_bytes + kChunk - 1) / kChunk);
    }
    return a.parts != 0;
}
static uint32_t copy_groups(uint64_t pairs, uint32_t chunks) { return pairs < kCopyGroups && pairs * chunks < kCopyGroups ? (uint32_t)(pairs * chunks) : kCopyGroups; }

struct CompactWorkspace {
    uint64_t live, sources, targets, n_moves, bytes;
};
static CompactWorkspace compact_workspace(uint64_t n_pages) {
    auto up = [](uint64_t x) { return (x + 255) & ~255ull; };
    CompactWorkspace w = {};
    w.sources = up((n_pages + 31) / 32 * 4);
    w.targets = w.sources + up((n_pages / 2 + 1) * 4);  // moves are no more than live pages, nor than others
    w.n_moves = w.targets + up((n_pages / 2 + 1) * 4);
    w.bytes = w.n_moves + 256;
    return w;
}

}  // namespace lsm

using namespace lsm;

extern "C" int lsm_copy_pages(const lsm_page_part_t* parts, uint64_t n_parts, uint64_t n_pages, const int32_t* sources, const int32_t* targets, uint64_t n, void* stream) {
    const int rc = check_parts(parts, n_parts, n_pages);
    if (rc != LSM_OK) return rc;
    if (n >= 1ull << 31) return LSM_ERR_BAD_ARG;
    if (n == 0 || n_parts == 0 || n_pages == 0) return LSM_OK;
    if (sources == nullptr || targets == nullptr) return LSM_ERR_NULL;
    if ((reinterpret_cast<uint64_t>(sources) | reinterpret_cast<uint64_t>(targets)) & 3) return LSM_ERR_BAD_ARG;
    CopyArgs a = {};
    a.sources = sources, a.targets = targets, a.pairs = n, a.n_pages = (uint32_t)n_pages;
    for (uint64_t at = 0; next_parts(a, parts, n_parts, at);)
        hipLaunchKernelGGL(copy_kernel, dim3(copy_groups(n, a.chunks)), dim3(kCopyThreads), 0, static_cast<hipStream_t>(stream), a);
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_HIP;
}

extern "C" size_t lsm_compact_pages_workspace_bytes(uint64_t n_pages) { return n_pages >= 1ull << 30 ? 0 : compact_workspace(n_pages).bytes; }

extern "C" int lsm_compact_pages(const lsm_page_part_t* parts, uint64_t n_parts, uint64_t n_pages, uint64_t page_tokens, const lsm_page_table_t* tables, uint64_t n_tables, int32_t* moved,
                                 int32_t* n_live, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_parts(parts, n_parts, n_pages);
    if (rc != LSM_OK) return rc;
    if (n_tables > LSM_MAX_PAGE_TABLES || page_tokens == 0 || page_tokens >= 1ull << 31) return LSM_ERR_BAD_ARG;
    if (n_live == nullptr || (moved == nullptr && n_pages != 0) || (tables == nullptr && n_tables != 0)) return LSM_ERR_NULL;
    if ((reinterpret_cast<uint64_t>(moved) | reinterpret_cast<uint64_t>(n_live)) & 3) return LSM_ERR_BAD_ARG;
    Tables t = {};
    t.page_tokens = page_tokens, t.n_pages = (uint32_t)n_pages;
    uint64_t entries = 0;
    for (uint64_t i = 0; i < n_tables; i++) {
        const lsm_page_table_t& in = tables[i];
        if (in.rows >= 1ull << 31 || in.width >= 1ull << 31 || in.rows * in.width >= 1ull << 31) return LSM_ERR_BAD_ARG;
        if (in.rows * in.width == 0) continue;
        if (in.pages == nullptr || in.lens == nullptr || in.new_pages == nullptr) return LSM_ERR_NULL;
        if ((reinterpret_cast<uint64_t>(in.pages) | reinterpret_cast<uint64_t>(in.lens) | reinterpret_cast<uint64_t>(in.new_pages)) & 3) return LSM_ERR_BAD_ARG;
        t.table[t.tables++] = Table{in.pages, in.lens, in.new_pages, in.rows * in.width, in.width};
        entries += in.rows * in.width;
    }
    const CompactWorkspace w = compact_workspace(n_pages);
    if (workspace == nullptr || workspace_bytes < w.bytes || (reinterpret_cast<uint64_t>(workspace) & 255) != 0) return LSM_ERR_WORKSPACE;
    char* const base = static_cast<char*>(workspace);
    PlanArgs p = {reinterpret_cast<uint32_t*>(base), reinterpret_cast<int32_t*>(base + w.sources), reinterpret_cast<int32_t*>(base + w.targets),
                  reinterpret_cast<uint32_t*>(base + w.n_moves), moved, n_live, (uint32_t)n_pages};
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto groups = [](uint64_t threads, uint64_t most) { return (uint32_t)(threads == 0 ? 1 : threads > most * 256 ? most : (threads + 255) / 256); };
    const uint32_t words = (uint32_t)((n_pages + 31) / 32), table_groups = entries ? groups(entries, 1024) : 0;
    if (words) hipLaunchKernelGGL(clear_kernel, dim3(groups(words, 1024)), dim3(256), 0, s, p.live, words);
    if (entries) hipLaunchKernelGGL(mark_kernel, dim3(table_groups), dim3(256), 0, s, t, p.live);
    hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
    CopyArgs a = {};
    a.sources = p.sources, a.targets = p.targets, a.n_pairs = p.n_moves, a.n_pages = (uint32_t)n_pages;
    uint64_t at = 0;
    if (n_pages < 2) n_parts = 0;  // nothing can move
    const bool any = next_parts(a, parts, n_parts, at);
    if (any || table_groups != 0)
        hipLaunchKernelGGL(move_kernel, dim3(table_groups + (any ? copy_groups(n_pages / 2, a.chunks) : 0)), dim3(kCopyThreads), 0, s, a, t, moved, table_groups);
    while (next_parts(a, parts, n_parts, at)) hipLaunchKernelGGL(copy_kernel, dim3(copy_groups(n_pages / 2, a.chunks)), dim3(kCopyThreads), 0, s, a);
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_HIP;
}
