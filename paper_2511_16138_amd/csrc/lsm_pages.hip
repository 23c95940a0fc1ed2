// lsm_copy_pages, lsm_compact_pages: pages copied within their buffers, and the live ones moved together.
#include <hip/hip_runtime.h>

#include "lsm_common.h"
#include "lsm_pages.h"

namespace lsm {

constexpr uint32_t kCopyThreads = 256, kCopyAhead = 4;
constexpr uint32_t kChunk = kCopyThreads * 16;  // bytes that a workgroup copies at a time: a word a lane
constexpr uint32_t kLaunchParts = 64;           // buffers of a launch
// Workgroups of a launch, about: four on each compute unit, which take turns; more of them where there is more to do for each (1,000 pages of 32 buffers, 1 GB: 426 us
// with 1,024 of them, 414 with 16,384; 24 blocks of 320 kB 4.5 and 4.9).
constexpr uint64_t kLeastGroups = 1024, kMostGroups = 16384;

struct Part {
    char* data;
    int64_t stride;
    uint64_t bytes;
    uint32_t chunks;  // of a page
    uint32_t wide;    // 16-byte words
};

typedef uint32_t Word __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) Word GlobalWord;  // addresses that were numbers: in global memory
typedef __attribute__((address_space(1))) uint8_t GlobalByte;

struct CopyArgs {
    Part part[kLaunchParts];
    const int32_t *sources, *targets;
    const uint32_t* n_pairs;  // DEVICE, where the host does not know ...
    uint32_t pairs;           // ... this
    uint32_t parts, n_pages;
};

// A workgroup copies every groups-th chunk of a buffer's pages, four of them at a time: a launch has enough workgroups for the chip, however many pairs there
// are, which the host need not know.  Lanes 0 to 3 find a chunk each, in one go; its addresses are scalars then.  Bound by memory: every byte is read once and
// written once (1,000 pages of 1 MB in 32 buffers 415 us, 5.05 TB/s, a copy's rate; 24 blocks of 320 kB 5, of which a launch is 3).
__device__ __forceinline__ void copy_chunks(const CopyArgs& a, const Part& part, uint32_t pairs, uint32_t group, uint32_t groups) {
    const uint32_t chunks = part.chunks, lane = threadIdx.x & (kWave - 1), mine = lane & (kCopyAhead - 1);
    const uint32_t step = groups * kCopyAhead, more_pairs = step / chunks, more_chunks = step - more_pairs * chunks;
    uint32_t pair = (group + mine * groups) / chunks, chunk = group + mine * groups - pair * chunks;  // of this lane
    for (uint32_t first = group / chunks, first_chunk = group - first * chunks; first < pairs;) {
        uint64_t in = 0, out = 0;
        uint32_t size = 0;
        if (pair < pairs) {
            const uint32_t from = (uint32_t)a.sources[pair], to = (uint32_t)a.targets[pair];
            const uint64_t at = (uint64_t)chunk * kChunk, left = part.bytes - at;
            if (from < a.n_pages && to < a.n_pages && from != to) size = left < kChunk ? (uint32_t)left : kChunk;
            in = reinterpret_cast<uint64_t>(part.data) + (int64_t)from * part.stride + at, out = reinterpret_cast<uint64_t>(part.data) + (int64_t)to * part.stride + at;
        }
        auto scalar = [](uint64_t x, uint32_t i) {
            return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), (int)i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, (int)i);
        };
        auto size_of = [&](uint32_t i) { return (uint32_t)__builtin_amdgcn_readlane((int)size, (int)i); };
        if (part.wide) {
            const uint32_t b = threadIdx.x * 16;
            auto load = [&](uint32_t i) {
                Word v = {0, 0, 0, 0};
                if (b < size_of(i)) v = *reinterpret_cast<const GlobalWord*>(scalar(in, i) + b);
                return v;
            };
            auto store = [&](uint32_t i, const Word& v) {
                if (b < size_of(i)) *reinterpret_cast<GlobalWord*>(scalar(out, i) + b) = v;
            };
            const Word v0 = load(0), v1 = load(1), v2 = load(2), v3 = load(3);
            store(0, v0), store(1, v1), store(2, v2), store(3, v3);
        } else {
#pragma unroll 1
            for (uint32_t i = 0; i < kCopyAhead; i++) {
                const GlobalByte* from = reinterpret_cast<const GlobalByte*>(scalar(in, i));
                GlobalByte* to = reinterpret_cast<GlobalByte*>(scalar(out, i));
                const uint32_t end = size_of(i);
                for (uint32_t b = threadIdx.x; b < end; b += kCopyThreads) to[b] = from[b];
            }
        }
        pair += more_pairs, chunk += more_chunks;
        if (chunk >= chunks) chunk -= chunks, pair++;
        first += more_pairs, first_chunk += more_chunks;
        if (first_chunk >= chunks) first_chunk -= chunks, first++;
    }
}

__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const CopyArgs a) { copy_chunks(a, a.part[blockIdx.y], a.pairs, blockIdx.x, gridDim.x); }
__global__ void __launch_bounds__(kCopyThreads) copy_counted_kernel(const CopyArgs a) { copy_chunks(a, a.part[blockIdx.y], *a.n_pairs, blockIdx.x, gridDim.x); }

// ---------------------------------------------------------------------------------------------------------------------
// compaction
// ---------------------------------------------------------------------------------------------------------------------
struct Table {
    const int32_t *pages, *lens;
    int32_t* new_pages;
    uint32_t entries, width;
};
struct Tables {
    Table table[LSM_MAX_PAGE_TABLES];
    uint64_t page_tokens;
    uint32_t tables, n_pages;
};

// f(table, entry, page, held) for each entry of every table: page is what it holds, ~0 where that is no page (a hole, or behind the length).  A thread reads four entries at a time.
template <typename F>
__device__ __forceinline__ void each_entry(const Tables& a, uint32_t thread, uint32_t threads, F f) {
    for (uint32_t t = 0; t < a.tables; t++) {
        const Table& table = a.table[t];
        for (uint64_t first = thread; first < table.entries; first += 4ull * threads) {
            uint32_t page[4], column[4];
            int32_t len[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; i++) {
                const uint64_t at = first + (uint64_t)i * threads;
                const uint32_t e = at < table.entries ? (uint32_t)at : 0, row = e / table.width;
                column[i] = e - row * table.width;
                len[i] = table.lens[row], page[i] = (uint32_t)table.pages[e];
            }
#pragma unroll
            for (uint32_t i = 0; i < 4; i++) {
                const uint64_t e = first + (uint64_t)i * threads;
                if (e < table.entries) f(table, (uint32_t)e, len[i] > 0 && (uint64_t)column[i] * a.page_tokens < (uint64_t)len[i] && page[i] < a.n_pages ? page[i] : ~0u, (int32_t)page[i]);
            }
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
    each_entry(a, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256, [&](const Table&, uint32_t, uint32_t page, int32_t) {
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
// either make a move.  live: a bit a page, in LDS or in memory.
__device__ __forceinline__ void plan_moves(const PlanArgs& a, const uint32_t* live_bits, uint32_t* lds) {
    const uint32_t words = (a.n_pages + 31) / 32, each = (words + kPlanThreads - 1) / kPlanThreads;
    const uint32_t begin = min(threadIdx.x * each, words), end = min(begin + each, words);
    uint32_t count = 0, n_live, n_holes, n_moves;
    for (uint32_t i = begin; i < end; i++) count += __popc(live_bits[i]);
    sum_before(count, lds, n_live);
    auto below = [&](uint32_t word) {  // the bits of a word that are of pages below n_live
        const uint32_t first = word * 32;
        return first >= n_live ? 0 : n_live - first >= 32 ? ~0u : (1u << (n_live - first)) - 1;
    };
    uint32_t holes = 0, movers = 0;
    for (uint32_t i = begin; i < end; i++) {
        const uint32_t live = live_bits[i], low = below(i);
        holes += __popc(~live & low), movers += __popc(live & ~low);
    }
    uint32_t hole = sum_before(holes, lds, n_holes), mover = sum_before(movers, lds, n_moves);
    for (uint32_t i = begin; i < end; i++) {
        const uint32_t live = live_bits[i], low = below(i);
        for (uint32_t bits = ~live & low; bits != 0; bits &= bits - 1) a.targets[hole++] = (int32_t)(i * 32 + __builtin_ctz(bits));
        for (uint32_t bits = live & ~low; bits != 0; bits &= bits - 1) a.sources[mover++] = (int32_t)(i * 32 + __builtin_ctz(bits));
    }
    for (uint32_t p = threadIdx.x; p < a.n_pages; p += kPlanThreads) {
        const bool live = (live_bits[p >> 5] >> (p & 31)) & 1;
        if (!live || p < n_live) a.moved[p] = live ? (int32_t)p : -1;
    }
    __syncthreads();  // the lists are written
    for (uint32_t i = threadIdx.x; i < n_moves; i += kPlanThreads) a.moved[a.sources[i]] = a.targets[i];
    if (threadIdx.x == 0) *a.n_moves = n_moves, *a.n_live = (int32_t)n_live;
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanArgs a) {
    __shared__ uint32_t lds[kPlanThreads / kWave];
    plan_moves(a, a.live, lds);
}

// Short tables and a pool whose bits fit into LDS: one launch in place of three, and bits set there, where thousands of them in a few lines of
// memory wait for each other (a table of 61 x 66: 12 us).
constexpr uint32_t kShortEntries = 1 << 15, kShortPages = 1 << 19;
__global__ void __launch_bounds__(kPlanThreads) plan_short_kernel(const PlanArgs a, const Tables tables) {
    __shared__ uint32_t lds[kPlanThreads / kWave], live[kShortPages / 32];
    for (uint32_t i = threadIdx.x; i < (a.n_pages + 31) / 32; i += kPlanThreads) live[i] = 0;
    __syncthreads();
    each_entry(tables, threadIdx.x, kPlanThreads, [&](const Table&, uint32_t, uint32_t page, int32_t) {
        if (page != ~0u) atomicOr(&live[page >> 5], 1u << (page & 31));
    });
    __syncthreads();
    plan_moves(a, live, lds);
}

// Sources are all at or above n_live and targets all below it, so pages move in any order.  The last row of the grid rewrites the tables.
__global__ void __launch_bounds__(kCopyThreads) move_kernel(const CopyArgs copies, const Tables tables, const int32_t* moved) {
    if (blockIdx.y == copies.parts) {
        each_entry(tables, blockIdx.x * kCopyThreads + threadIdx.x, gridDim.x * kCopyThreads,
                   [&](const Table& t, uint32_t e, uint32_t page, int32_t held) { t.new_pages[e] = page == ~0u ? held : moved[page]; });
    } else {
        copy_chunks(copies, copies.part[blockIdx.y], *copies.n_pairs, blockIdx.x, gridDim.x);
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
    for (a.parts = 0; at < n_parts && a.parts < kLaunchParts; at++) {
        const lsm_page_part_t& p = parts[at];
        if (p.page_bytes == 0) continue;
        const uint64_t bits = reinterpret_cast<uint64_t>(p.data) | (uint64_t)p.page_stride | p.page_bytes;
        a.part[a.parts++] = Part{static_cast<char*>(p.data), p.page_stride, p.page_bytes, (uint32_t)((p.page_bytes + kChunk - 1) / kChunk), (bits & 15) == 0};
    }
    return a.parts != 0;
}
// Workgroups for each buffer of a launch, none of which has more chunks than the largest one.  pairs_known: `pairs` are to be copied; at most as many otherwise.
static uint32_t copy_groups(const CopyArgs& a, uint64_t pairs, bool pairs_known) {
    uint64_t chunks = 1, all = 0;
    for (uint32_t i = 0; i < a.parts; i++) chunks = a.part[i].chunks > chunks ? a.part[i].chunks : chunks, all += a.part[i].chunks;
    uint64_t groups = pairs_known ? pairs * all / 16 : 0;
    groups = groups < kLeastGroups ? kLeastGroups : groups > kMostGroups ? kMostGroups : groups;
    groups = (groups + a.parts - 1) / a.parts;
    return (uint32_t)(pairs * chunks < groups ? pairs * chunks : groups);
}

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
    a.sources = sources, a.targets = targets, a.pairs = (uint32_t)n, a.n_pages = (uint32_t)n_pages;
    for (uint64_t at = 0; next_parts(a, parts, n_parts, at);)
        hipLaunchKernelGGL(copy_kernel, dim3(copy_groups(a, n, true), a.parts), dim3(kCopyThreads), 0, static_cast<hipStream_t>(stream), a);
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
        t.table[t.tables++] = Table{in.pages, in.lens, in.new_pages, (uint32_t)(in.rows * in.width), (uint32_t)in.width};
        entries += in.rows * in.width;
    }
    const CompactWorkspace w = compact_workspace(n_pages);
    if (workspace == nullptr || workspace_bytes < w.bytes || (reinterpret_cast<uint64_t>(workspace) & 255) != 0) return LSM_ERR_WORKSPACE;
    char* const base = static_cast<char*>(workspace);
    PlanArgs p = {reinterpret_cast<uint32_t*>(base), reinterpret_cast<int32_t*>(base + w.sources), reinterpret_cast<int32_t*>(base + w.targets),
                  reinterpret_cast<uint32_t*>(base + w.n_moves), moved, n_live, (uint32_t)n_pages};
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto groups = [](uint64_t threads, uint64_t most) { return (uint32_t)(threads == 0 ? 1 : threads > most * 256 ? most : (threads + 255) / 256); };
    const uint32_t words = (uint32_t)((n_pages + 31) / 32);
    if (entries <= kShortEntries && n_pages <= kShortPages) {
        hipLaunchKernelGGL(plan_short_kernel, dim3(1), dim3(kPlanThreads), 0, s, p, t);
    } else {
        if (words) hipLaunchKernelGGL(clear_kernel, dim3(groups(words, 1024)), dim3(256), 0, s, p.live, words);
        if (entries) hipLaunchKernelGGL(mark_kernel, dim3(groups(entries, 1024)), dim3(256), 0, s, t, p.live);
        hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
    }
    CopyArgs a = {};
    a.sources = p.sources, a.targets = p.targets, a.n_pairs = p.n_moves, a.n_pages = (uint32_t)n_pages;
    uint64_t at = 0;
    if (n_pages < 2) n_parts = 0;  // nothing can move
    if (next_parts(a, parts, n_parts, at) || entries != 0) {
        const uint32_t for_tables = entries ? groups(entries, 1024) : 0, for_parts = a.parts ? copy_groups(a, n_pages / 2, false) : 0;
        hipLaunchKernelGGL(move_kernel, dim3(for_tables > for_parts ? for_tables : for_parts, a.parts + (entries ? 1 : 0)), dim3(kCopyThreads), 0, s, a, t, moved);
    }
    while (next_parts(a, parts, n_parts, at)) hipLaunchKernelGGL(copy_counted_kernel, dim3(copy_groups(a, n_pages / 2, false), a.parts), dim3(kCopyThreads), 0, s, a);
    return hipGetLastError() == hipSuccess ? LSM_OK : LSM_ERR_HIP;
}
