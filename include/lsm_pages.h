/*
 * lsm_pages.h -- C ABI of what a server does with the pages of lsm_cache.h beyond 16-bit append and attention (MI355X, gfx950).
 *
 *   lsm_kv_append8        keys and values of new tokens into pages held in 8 bits, normed and rotated on the way
 *   lsm_window_attention  lsm_prefix_attention over such pages, and with a window: a token sees the last few tokens and the first few
 *   lsm_copy_pages        pages copied, or forked, in any number of buffers at once
 *   lsm_compact_pages     the pages that some page table holds moved together, and the tables with them
 *
 * Conventions are those of lsm_cache.h.
 *
 * A cache in 8 bits: a key's or value's element is code * 2^e.  The code is one byte of type e4m3 (sign, 4 bits of exponent, 3 of mantissa:
 * magnitudes up to 448, 4 significant bits down to 2^-6, multiples of 2^-9 below; 0x7F and 0xFF are NaN, there is no infinity).  The
 * exponent belongs to a block of LSM_SCALE_TOKENS tokens of a page and a KV head, and is held as the byte e + 127; the byte 255 makes the whole block NaN.
 * A scale that is a power of two loses nothing against any other, the codes being of floating point: it moves the range that they
 * cover, not their steps.  Scaling is exact then, and a block's older codes outlive a larger scale but for their last bits under 2^-6.
 */
#ifndef LSM_PAGES_H
#define LSM_PAGES_H

#include "lsm_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    LSM_SCALE_TOKENS = 16,     /* tokens of a block with a scale: rows 16 i .. 16 i + 15 of a page                       */
    LSM_LEAST_SCALE = -100,    /* the smallest e that lsm_kv_append8 writes: magnitudes up to 2^-110 become 0             */
    LSM_MAX_PAGE_TABLES = 16,  /* tables of a call of lsm_compact_pages                                                  */
    LSM_MAX_PAGE_PARTS = 1024  /* buffers of a call of lsm_copy_pages or lsm_compact_pages                               */
};

/* Scales of one side (keys or values) of a layer's pages: the byte of head h of block b of page p is
 * data[p * page_stride + b * block_stride + h * head_stride]. */
typedef struct {
    uint8_t* data;       /* DEVICE */
    int64_t page_stride; /* in bytes */
    int64_t block_stride;
    int64_t head_stride;
} lsm_scales_t;

/* The new tokens of a batch and the pages that they belong to, as lsm_attention_t has them: request r has the new tokens
 * q_offsets[r] .. q_offsets[r + 1] - 1; they are the last of its own_lens[r] tokens, token i of which is in row i % page_tokens of page
 * own_tables[r * own_width + i / page_tokens]. */
typedef struct {
    const int32_t* q_offsets;  /* DEVICE, n_requests + 1                */
    const int32_t* own_tables; /* DEVICE, n_requests x own_width        */
    const int32_t* own_lens;   /* DEVICE, n_requests                    */
    uint64_t n_requests, own_width, n_pages, page_tokens;
} lsm_new_tokens_t;

/*
 * lsm_kv_append8 -- keys (normed and rotated as lsm_rotate_heads does) and values (as they are) of the new tokens into pages in 8 bits.
 * For every block of 16 tokens, KV head and side that a request's new tokens reach:
 *   e = the smallest whole number from LSM_LEAST_SCALE on with 448 * 2^e >= the largest finite magnitude among the new tokens
 *   if the block's first row is not new, the request goes on in it: e = max(e, the block's e so far), and where that is more
 *     than it was, the codes of the rows before the first new one become those of their values divided by 2^e
 *   new codes = values / 2^e, rounded once, to nearest, ties to even; infinities and NaN become NaN
 * Magnitudes beyond the largest number of 4 significant bits that dtype holds (61440 in LSM_FP16) become that (so that no finite value is infinite when it is read).
 * Keys are computed as if in 64 bits, so that each code is the nearest one to the formula's value.
 * Rows behind the new ones keep their bytes.  Tokens that no request has, or whose place is below 0, beyond the table or in a page outside
 * [0, n_pages), are not written.  A block belongs to one request: two that write the same one leave bytes and scale of either.
 * The queries of all n_tokens tokens are normed and rotated in the same launch if q is given.
 * k, v: the same number of heads; how->dtype is theirs and the queries'.  page_tokens: a multiple of LSM_SCALE_TOKENS.
 * n_requests is below 2^24, own_width * page_tokens below 2^30, n_tokens below 2^24.
 * Errors: LSM_ERR_NULL, LSM_ERR_BAD_ARG, LSM_ERR_HIP.
 */
int lsm_kv_append8(const lsm_rotation_t* how, const lsm_heads_t* k, const void* k_weight, const lsm_heads_t* v, const lsm_new_tokens_t* to,
                   const lsm_pages_t* k_pages, const lsm_scales_t* k_scales, const lsm_pages_t* v_pages, const lsm_scales_t* v_scales,
                   const lsm_heads_t* q, const void* q_weight, const lsm_heads_t* q_out, void* stream);

/*
 * lsm_window_attention -- lsm_prefix_attention (its limits and guarantees hold here too), with
 *   window > 0: the token at place p of its request's sequence (the group's prefix, then the request's own tokens, holes and all) sees
 *     of what it would see otherwise the tokens at places i < sinks and i > p - window.  window = 0: all of it; sinks has to be 0 then.
 *   scales given (both sides): the pages hold 8 bits, their strides count bytes, and all rows are 16-byte aligned (data 16-byte
 *     aligned, strides multiples of 16).  A value is rounded to base.dtype where that does not hold it (LSM_FP16: below 2^-14, and beyond 65504, which
 *     becomes infinite; LSM_BF16: below 2^-126, which becomes 0, and from 2^128 on).
 * With a window that is shorter than the tables ((prefix_width + own_width) * page_tokens) every request is worked on by itself: a prefix is read again
 * for each request whose window reaches it.
 * workspace: as for lsm_prefix_attention, of lsm_window_attention_workspace_bytes(a) bytes.  window, sinks and, with such a window,
 * (prefix_width + own_width) * page_tokens are below 2^30.
 * Errors: LSM_ERR_NULL, LSM_ERR_BAD_ARG, LSM_ERR_WORKSPACE, LSM_ERR_HIP.
 */
typedef struct {
    lsm_attention_t base;
    lsm_scales_t k_scales, v_scales; /* data NULL (both): pages of base.dtype */
    uint64_t window, sinks;
} lsm_window_attention_t;

size_t lsm_window_attention_workspace_bytes(const lsm_window_attention_t* a);
int lsm_window_attention(const lsm_window_attention_t* a, void* workspace, size_t workspace_bytes, void* stream);

/* A buffer of pages: page p is the page_bytes bytes from data + p * page_stride on. */
typedef struct {
    void* data;          /* DEVICE */
    int64_t page_stride; /* in bytes */
    uint64_t page_bytes;
} lsm_page_part_t;

/*
 * lsm_copy_pages -- page targets[i] becomes a copy of page sources[i], i < n, in every one of n_parts buffers.  One source may have many
 * targets (a fork).  A pair with either number outside [0, n_pages), or with both the same, copies nothing.  A page that is a target twice, or a target and
 * the source of another pair, ends up with 16-byte pieces (single bytes where buffers are not 16-byte aligned) of any of the pages in question.
 * parts: HOST, read before the call returns; buffers do not overlap, nor a buffer's pages.  sources, targets: DEVICE.
 * Buffers whose data, stride and size are multiples of 16 are copied in 16-byte words, others by bytes.
 * n is below 2^31.  Errors: LSM_ERR_NULL, LSM_ERR_BAD_ARG, LSM_ERR_HIP.
 */
int lsm_copy_pages(const lsm_page_part_t* parts, uint64_t n_parts, uint64_t n_pages, const int32_t* sources, const int32_t* targets, uint64_t n,
                   void* stream);

/* A page table: entry j of row r, pages[r * width + j], holds a page if j * page_tokens < lens[r].  new_pages: the same with the new numbers;
 * may be `pages` itself, may not overlap it otherwise. */
typedef struct {
    const int32_t* pages; /* DEVICE, rows x width */
    const int32_t* lens;  /* DEVICE, rows         */
    int32_t* new_pages;   /* DEVICE, rows x width */
    uint64_t rows, width;
} lsm_page_table_t;

/*
 * lsm_compact_pages -- a page is live if some table holds it; nothing has to be said of pages that nobody holds any more.  With n_live the number of
 * live pages, those below n_live stay where they are; the k-th live page from n_live on (k = 0, 1, ..) moves to the k-th page below n_live that
 * is not live.  Pages 0 .. n_live - 1 are live then and the others free, with as few moves as that takes.
 *   moved[p]  the new number of page p, -1 where it was not live
 *   n_live    one number
 *   the pages' bytes in all n_parts buffers, and the tables: entries that hold a page get its new number, others stay as they are.
 * A held number outside [0, n_pages) is a hole: it holds no page.  Which tables are given decides: a cache that keeps blocks for later has to say so, with a
 * table of its own.  n_parts may be 0, and so may n_tables (nothing is live then).
 * parts, tables: HOST, read before the call returns.  workspace: DEVICE, 256-byte aligned, lsm_compact_pages_workspace_bytes(n_pages) bytes;
 * contents on entry are irrelevant.  n_pages is below 2^30, rows * width of a table below 2^31, page_tokens above 0 and below 2^31.
 * Errors: LSM_ERR_NULL, LSM_ERR_BAD_ARG, LSM_ERR_WORKSPACE, LSM_ERR_HIP.
 */
size_t lsm_compact_pages_workspace_bytes(uint64_t n_pages);
int lsm_compact_pages(const lsm_page_part_t* parts, uint64_t n_parts, uint64_t n_pages, uint64_t page_tokens, const lsm_page_table_t* tables,
                      uint64_t n_tables, int32_t* moved, int32_t* n_live, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
