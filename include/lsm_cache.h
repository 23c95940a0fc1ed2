/*
 * lsm_cache.h -- C ABI of the paged KV cache behind the key index (MI355X, gfx950).
 *
 * lsm_probe answers a batch of requests with their longest cached prefixes: value pointers to 16-token blocks of keys and
 * values, many requests behind few shared prefixes.  The calls here work on those blocks once they lie in device memory as
 * the pages of a cache:
 *
 *   lsm_rope_table        cosines and sines of the position rotation, made once
 *   lsm_rotate_heads      norm of queries and keys for each head, and the position rotation, in one pass
 *   lsm_kv_append         keys and values of new tokens into pages, normed and rotated on the way
 *   lsm_prefix_attention  attention of a batch whose requests share long prefixes: a prefix's keys and values are read once
 *                         for all requests behind it, and every request has pages of its own after it
 *
 * Conventions are those of lsm_index.h: DEVICE pointers, work enqueued on `stream`, 0 or a negative lsm_status, argument errors
 * found on the host before anything is launched, no allocation, no state between calls.  All of them may be captured into a
 * graph.  What the host cannot see (positions, slots, page numbers, lengths) is checked by the kernels: a value out of range
 * never makes them read or write outside the buffers described; what it does instead is said at each call.
 * Sums, norms, the running maximum and sum of the softmax and the accumulators are held in 32 bits.
 */
#ifndef LSM_CACHE_H
#define LSM_CACHE_H

#include "lsm_index.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { LSM_BF16 = 0, LSM_FP16 = 1, LSM_FP32 = 2 } lsm_dtype;

enum {
    LSM_MAX_HEAD_DIM = 256,   /* elements of a head                                                              */
    LSM_MIN_PAGE_TOKENS = 16, /* tokens of a page of lsm_prefix_attention: a power of two from here ...          */
    LSM_MAX_PAGE_TOKENS = 256 /* ... to here                                                                     */
};

/* Heads of n_tokens tokens: element d of head h of token t is data[t * token_stride + h * head_stride + d]. */
typedef struct {
    void* data;           /* DEVICE; NULL = none                                            */
    int64_t token_stride; /* in elements                                                    */
    int64_t head_stride;
    uint64_t heads;
} lsm_heads_t;

/* One side (keys or values) of a layer's pages: element d of head h of token i of page p is
 * data[p * page_stride + i * token_stride + h * head_stride + d].  A layer of a block that holds all layers' keys
 * and values is described by its strides; nothing has to be copied together. */
typedef struct {
    void* data;          /* DEVICE */
    int64_t page_stride; /* in elements */
    int64_t token_stride;
    int64_t head_stride;
} lsm_pages_t;

/*
 * What lsm_rotate_heads and lsm_kv_append do to a head x of a token at position p:
 *   norm (where a weight w is given):  y = x / sqrt(mean(x^2) + eps) * w;   otherwise y = x
 *   rotation (where a table is given): pairs (a, b) of the first rot_dim elements, pair i by the angle whose cosine and
 *     sine are table[p][i] and table[p][rot_dim / 2 + i]:  a' = a cos - b sin,  b' = b cos + a sin
 *     pair i = elements (i, i + rot_dim / 2), or (2 i, 2 i + 1) with `interleaved`; elements from rot_dim on stay y
 * in 32 bits, rounded once.  A position outside [0, n_positions) has no angle: what would be rotated by it becomes NaN.
 */
typedef struct {
    const int32_t* positions; /* DEVICE, n_tokens values; may be NULL without a table       */
    const float* table;       /* DEVICE, n_positions x rot_dim (lsm_rope_table); NULL = no rotation */
    uint64_t n_positions;
    uint64_t n_tokens;
    uint32_t rot_dim;         /* even, <= head_dim                                          */
    uint32_t head_dim;        /* a multiple of 8, <= LSM_MAX_HEAD_DIM                       */
    uint32_t dtype;           /* lsm_dtype of queries, keys, values and pages               */
    uint32_t weight_dtype;    /* lsm_dtype of the weights: dtype or LSM_FP32                */
    uint32_t interleaved;     /* 0 or 1                                                     */
    float eps;
} lsm_rotation_t;

/*
 * lsm_rope_table -- table[p][i] = cos(p theta^(-2i / rot_dim)), table[p][rot_dim / 2 + i] = the sine, for p < n_positions
 * and i < rot_dim / 2; angles, cosines and sines in 64 bits (an angle of 10^5 held in 32 bits is off by 4e-3), rounded once.
 * Errors: LSM_ERR_NULL, LSM_ERR_BAD_ARG (rot_dim odd, 0 or > LSM_MAX_HEAD_DIM, theta not above 0 or infinite), LSM_ERR_HIP.
 */
int lsm_rope_table(float* table, uint64_t n_positions, uint32_t rot_dim, double theta, void* stream);

/*
 * lsm_rotate_heads -- norm and rotation of the queries and keys of n_tokens tokens in one launch.  q or k may be NULL; so
 * may the weights (head_dim values each: no norm).  q_out, k_out: same number of heads; either the input itself (same data,
 * same strides) or not overlapping it.  Rows that are 16-byte aligned are read and written in 16-byte words, others by
 * elements.  Errors: LSM_ERR_NULL, LSM_ERR_BAD_ARG, LSM_ERR_HIP.
 */
int lsm_rotate_heads(const lsm_rotation_t* how, const lsm_heads_t* q, const void* q_weight, const lsm_heads_t* q_out,
                     const lsm_heads_t* k, const void* k_weight, const lsm_heads_t* k_out, void* stream);

/*
 * lsm_kv_append -- keys (normed and rotated) and values (as they are) of token t go to slot slots[t] of the cache: page
 * slots[t] / page_tokens, row slots[t] % page_tokens.  A slot below 0 or not below n_pages * page_tokens writes nothing
 * (padding, tokens that are cached already).  Two tokens with one slot: either may win, for every 16 bytes, or
 * every element where rows are not 16-byte aligned.  The queries of the same tokens, skipped or not, are normed and rotated
 * in the same launch if q is given, as lsm_rotate_heads does.  Tokens beyond 2^26 take several launches, there and here.
 * slots: DEVICE, n_tokens int64.  k, v: the same number of heads.  page_tokens: any number above 0.
 * Errors: LSM_ERR_NULL, LSM_ERR_BAD_ARG, LSM_ERR_HIP.
 */
int lsm_kv_append(const lsm_rotation_t* how, const lsm_heads_t* k, const void* k_weight, const lsm_heads_t* v,
                  const int64_t* slots, const lsm_pages_t* k_pages, const lsm_pages_t* v_pages, uint64_t n_pages,
                  uint64_t page_tokens, const lsm_heads_t* q, const void* q_weight, const lsm_heads_t* q_out, void* stream);

/*
 * lsm_prefix_attention -- attention of n_requests requests in n_groups groups.  Requests group_offsets[g] ..
 * group_offsets[g + 1] - 1 share the prefix of group g (group_offsets[0] = 0, group_offsets[n_groups] = n_requests, not
 * descending); request r has the new tokens q_offsets[r] .. q_offsets[r + 1] - 1 (likewise, to n_tokens).
 * Token j of the q_len new tokens of request r sees
 *   all prefix_lens[g] tokens of its group's prefix: token i is in row i % page_tokens of page
 *     prefix_tables[g * prefix_width + i / page_tokens]
 *   and the first own_lens[r] - q_len + j + 1 tokens of its own pages (own_tables, the same way): the new tokens are the
 *     last of them, their keys and values are in the pages already.
 * With s_i = scale * (q . k_i) over those:  out = sum_i exp(s_i) v_i / sum_i exp(s_i),  lse = log sum_i exp(s_i).
 * A token that sees nothing has out = 0 and lse = -infinity.  Query head h reads KV head h / (q.heads / kv_heads).
 * Lengths are cut to [0, width * page_tokens]; the tokens of a page number outside [0, n_pages) are not seen (holes).
 * Rows behind a length, and pages that no length reaches, are never used, whatever they hold; keys and values that are not
 * finite reach the tokens that see them and no others.
 * Offsets that descend or leave their range give an unspecified, in-bounds result.
 * scale: above 0, and scale log2(e) finite.  n_tokens, n_requests and n_groups are below 2^24, n_tokens * q.heads below 2^31,
 * widths times page_tokens below 2^30; a batch is one launch of fewer than 2^24 workgroups (about 1.8 million decodes of
 * 8 KV heads).
 * dtype: LSM_BF16 or LSM_FP16; head_dim: 64, 128 or 256.  The weights of the softmax are rounded to dtype for the product
 * with the values, as the values are; in LSM_FP16 those under 2^-14 lose bits as subnormals, so that n keys far below the
 * largest score are off by up to n 2^-25 of its weight.
 * All rows 16-byte aligned: data 16-byte aligned, strides multiples of 8.
 * workspace: DEVICE, 256-byte aligned, lsm_prefix_attention_workspace_bytes(a) bytes; contents on entry are irrelevant.
 * Results are the same bits from call to call.  Errors: LSM_ERR_NULL, LSM_ERR_BAD_ARG, LSM_ERR_WORKSPACE, LSM_ERR_HIP.
 */
typedef struct {
    lsm_heads_t q;
    lsm_heads_t out; /* may not overlap q */
    float* lse;      /* DEVICE, n_tokens x q.heads; NULL = none */
    lsm_pages_t k_pages, v_pages;
    const int32_t* group_offsets; /* DEVICE, n_groups + 1                */
    const int32_t* prefix_tables; /* DEVICE, n_groups x prefix_width     */
    const int32_t* prefix_lens;   /* DEVICE, n_groups                    */
    const int32_t* q_offsets;     /* DEVICE, n_requests + 1              */
    const int32_t* own_tables;    /* DEVICE, n_requests x own_width      */
    const int32_t* own_lens;      /* DEVICE, n_requests                  */
    uint64_t n_tokens, n_requests, n_groups, prefix_width, own_width, n_pages, page_tokens, kv_heads;
    uint32_t head_dim;
    uint32_t dtype;
    float scale;
    uint32_t reserved; /* 0 */
} lsm_attention_t;

size_t lsm_prefix_attention_workspace_bytes(const lsm_attention_t* a);
int lsm_prefix_attention(const lsm_attention_t* a, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
