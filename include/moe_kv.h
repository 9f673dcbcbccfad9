/*
 * moe_kv.h -- C ABI of the attention half of a decode step on MI355X (gfx950): a paged key/value cache held in
 * 8 bits, the pages of a step's tokens, the store of rotated keys and values, and attention over the cache.
 *
 * A step is a ragged batch of requests.  Request r has ctx_len[r] tokens in the cache and brings new_len[r] new ones (one
 * token, a few drafted ones, a prompt or a part of one); the new tokens of all requests are packed row after row,
 * request after request.  Per step, once:      moe_kv_plan    block tables, slots, and how attention is shared out
 * and then per layer, with the layer's cache:  moe_kv_write   norm, rotation, store of keys and values
 *                                              moe_kv_attend  attention of the new tokens over all that is cached
 * No call reads a length on the host, waits or allocates: all of them can be captured into a HIP graph that later runs
 * with other lengths of the same bounds.  The conventions are those of moe_offload.h (status codes, moe_last_error, caller-owned memory and
 * streams); a call is ordered by the stream that it is given and by nothing else.
 *
 * The cache of a layer.  A page holds `page` consecutive tokens of one request.  For every page and kv head there is a
 * run of page * head_dim codes, in tiles of 16 x 16 bytes, and one fp32 scale, for keys and for values each:
 *   k: [n_pages][kv_heads][page/16][head_dim/16][16 tokens][16 dims]
 *   v: [n_pages][kv_heads][page/16][head_dim/16][16 dims][16 tokens]
 *   value = code * scale[page][kv head]
 * Codes are finite: the store clamps numbers to +-65504 (fp16 rows) or +-2^100 (bf16 rows), infinities with them, and takes NaN for 0, for
 * a single NaN would otherwise reach every token of its page.  A scale is not negative and 2^100 at most; of scales below
 * 2^-96, the store's least, attention takes 2^-96.
 *
 * Whose pages these are.  A page that gets tokens belongs to one request: two whose tables name the same begun page would both rewrite
 * it.  Full pages that several requests read may be in several tables; before a request is released, its entries of pages that
 * others still read become -1.  Tokens are taken back by lowering ctx_len as long as ceil(ctx_len/page) stays as it is; beyond that the next plan takes a new
 * page off the stack over the table's entry, and the old page is the caller's to push onto the stack first, as are pages that a window has
 * left behind (whose entries become -1).  A page's scale does not fall when tokens are taken back.
 */
#ifndef MOE_KV_H
#define MOE_KV_H

#include "moe_offload.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MOE_KV_MAX_REQUESTS 4096
#define MOE_KV_MAX_TOKENS   1048576   /* rows of a step */

enum { MOE_KV_E4M3 = 0, MOE_KV_INT8 = 1 };   /* codes: OCP fp8 e4m3 (largest 448), two's complement (largest 127) */
enum { MOE_KV_F16 = 0, MOE_KV_BF16 = 1 };    /* 16-bit types of rows                                              */

/* Why a request of a step gets nothing (moe_kv_lists_t.status). */
enum {
    MOE_KV_SERVED    = 0,
    MOE_KV_NO_PAGES  = 1,   /* the free pages do not reach for it and those before it                            */
    MOE_KV_TOO_LONG  = 2,   /* ctx_len + new_len needs more than max_blocks pages                                */
    MOE_KV_BAD_SIZE  = 3    /* a negative length, or rows beyond n_tokens                                        */
};

typedef struct {
    int32_t n_pages;          /* n_pages * page < 2^31 and n_pages * kv_heads * page / 16 < 2^32                 */
    int32_t page;             /* tokens per page: 16, 32, 64 or 128                                              */
    int32_t kv_heads;         /* 1..256                                                                          */
    int32_t head_dim;         /* 64, 128 or 256                                                                  */
    int32_t format;           /* MOE_KV_E4M3 or MOE_KV_INT8                                                      */
    int32_t reserved;         /* 0                                                                               */
    void *k, *v;              /* dev, 16-byte aligned                                                            */
    float *k_scale, *v_scale; /* dev [n_pages][kv_heads]                                                         */
} moe_kv_cache_t;

/* What the host knows of a step: bounds, not lengths. */
typedef struct {
    int32_t n_requests;       /* 1..MOE_KV_MAX_REQUESTS                                                          */
    int32_t n_tokens;         /* rows of the batch, 1..MOE_KV_MAX_TOKENS; rows past the last request's are left alone */
    int32_t max_new;          /* no request brings more rows than this (those that do are BAD_SIZE)              */
    int32_t max_blocks;       /* width of the block table; max_blocks * page <= 2^24 - 32 tokens of a request    */
    int32_t n_pages, page, kv_heads, head_dim;   /* as the caches that the step runs on                          */
    int32_t q_heads;          /* a multiple of kv_heads; query head h reads kv head h / (q_heads / kv_heads)     */
    int32_t causal;           /* 1: a token sees the tokens up to itself; 0: all of its request                  */
    int32_t window;           /* w > 0: a token sees nothing more than w - 1 positions before it; 0: no limit    */
    int32_t reserved;         /* 0                                                                               */
} moe_kv_step_t;

/* Device arrays of int32.  No output may lie in an input; every pointer is required. */
typedef struct {
    const int32_t *ctx_len;     /* [n_requests] tokens in the cache                                              */
    const int32_t *new_len;     /* [n_requests] tokens that this step adds                                       */
    int32_t *block_table;       /* [n_requests][max_blocks]: page of tokens [b page, (b+1) page).  Entries up to
                                   ceil(ctx_len/page) are read, those of the pages a step adds are written       */
    const int32_t *free_pages;  /* a stack of at most n_pages free pages, its top at [*free_count - 1]; the first min(*free_count,
                                   n_pages) entries may be read (moe_kv_plan_within: no more than free_capacity)  */
    const int32_t *free_count;
    int32_t *row_start;         /* out [n_requests + 1]: first row of each request                               */
    int32_t *positions;         /* out [n_tokens]: position of a row's token in its request, -1 for none         */
    int32_t *slots;             /* out [n_tokens]: page * page size + offset, -1 for none                        */
    int32_t *kv_len;            /* out [n_requests]: ctx_len + new_len, or ctx_len where status is not 0         */
    int32_t *status;            /* out [n_requests]                                                              */
    int32_t *free_left;         /* out [1]: free pages that remain on the stack                                  */
} moe_kv_lists_t;

/* Device bytes of a step's plan, and of the scratch that moe_kv_attend needs (one per stream; layers share it; 0 is a
 * possible answer).  Both 0 for a bad step. */
uint64_t moe_kv_plan_bytes(const moe_kv_step_t *step);
uint64_t moe_kv_scratch_bytes(const moe_kv_step_t *step);

/* Pages of a step's new tokens.  Requests are served in order: one gets its pages if it needs none or if the pages that
 * it and the requests before it need (those that were turned down for want of pages included) are not more than the free
 * ones; they are taken off the stack's top, in order.  A request with a status gets nothing: its rows have no slot and attend
 * to nothing (those of a BAD_SIZE request are left alone).  A slot is -1, too, where the table or the stack names a page that does not exist.
 * plan_dev: moe_kv_plan_bytes, 256-byte aligned: what moe_kv_write and moe_kv_attend read, with the step that it was made for.  One
 * moe_kv_attend at a time uses a plan (it counts the parts that are done there). */
int32_t moe_kv_plan(const moe_kv_step_t *step, const moe_kv_lists_t *lists, void *plan_dev, void *stream);
/* The same with a stack that has room for free_capacity entries: a *free_count above it counts as free_capacity. */
int32_t moe_kv_plan_within(const moe_kv_step_t *step, const moe_kv_lists_t *lists, int32_t free_capacity, void *plan_dev, void *stream);

/* Give back all pages of `n` requests (ids in `requests`, dev; out of range or repeated ones do nothing more), in the order given: their
 * pages go onto the stack, ctx_len[r] becomes 0.  Pages that are no page of the cache, and those that find the
 * stack's `capacity` entries full, are dropped.  Not between a step's plan and the copying of its kv_len and free_left over ctx_len and
 * free_count, which would undo it.  Requests are taken one after the other. */
int32_t moe_kv_release(const int32_t *requests, int32_t n, int32_t n_requests, int32_t n_pages, int32_t page, int32_t max_blocks,
                       int32_t *ctx_len, const int32_t *block_table, int32_t *free_pages, int32_t capacity,
                       int32_t *free_count, void *stream);

/* The rows of a step.  q [n_tokens][q_heads][head_dim], k and v [n_tokens][kv_heads][head_dim]: heads follow each other, rows
 * are *_stride elements apart.  Any alignment; 16-byte aligned pointers with strides that are multiples of 8 are faster. */
typedef struct {
    int32_t dtype;              /* MOE_KV_F16 or MOE_KV_BF16, of q, k, v, q_out and the gains                    */
    int32_t rot_dim;            /* first dims of a head that are rotated, a multiple of 16, 0..head_dim          */
    int32_t interleaved;        /* rotated pairs: 0 (i, i + rot_dim/2), 1 (2i, 2i + 1)                           */
    float eps;                  /* > 0: RMSNorm of every query and key head with this eps; 0: none               */
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const void *q_gamma, *k_gamma;   /* [head_dim] gains of the norms, NULL: 1                                   */
    const float *inv_freq;      /* [rot_dim/2]: a pair turns by position * inv_freq[i], in fp64                  */
    void *q_out;                /* normed and rotated queries, rounded once; may be q (with its stride)          */
    int64_t q_out_stride;
} moe_kv_rows_t;

/* Norm and rotation of queries and keys in fp32, queries to q_out, keys and values as 8-bit codes to the cache.
 * A page's scale is the smallest power of two, 2^-96 at least, that keeps every number of the page within the format's largest code, and
 * at least what it was if tokens of the page are in the cache already.  Where it grows, their codes are rounded again: with a power of two
 * e4m3 codes stay exact but for those that become subnormal, int8 codes move by less than one step of the final scale
 * in all the growths of a page together. */
int32_t moe_kv_write(const moe_kv_cache_t *cache, const moe_kv_step_t *step, const void *plan_dev, const moe_kv_rows_t *rows,
                     void *stream);

typedef struct {
    int32_t dtype;              /* MOE_KV_F16 or MOE_KV_BF16, of q and out                                       */
    float scale;                /* of the scores, > 0                                                            */
    const void *q;              /* [n_tokens][q_heads][head_dim], rows q_stride elements apart                   */
    int64_t q_stride;
    void *out;                  /* same form; must not be q                                                      */
    int64_t out_stride;
    float *lse;                 /* nullable [n_tokens][q_heads]: natural log of the sum of the exponentials      */
} moe_kv_query_t;

/* Attention of a step's rows: out = sum_j softmax(scale * q.k_j) v_j over the cached tokens that the row sees.  A row that sees none gets
 * 0 and lse -inf.  Table entries outside the cache are skipped as if they were masked.  Deterministic: how the work is split follows from the lengths alone.
 * Scores, maxima, sums and outputs are held in fp32, codes are exact.  Rounded to fewer bits are: the weights that values are multiplied with, to fp16
 * (2^-11 of a weight at most; with fp16 outputs the distance from 64 bits is 1.3 times that of fp32 weights, with bf16 outputs the same), and bf16
 * queries, to fp16 after a power of two is taken off each row (what is 2^38 below a row's largest is dropped).  Both let the matrix units
 * work on 16-bit operands. */
int32_t moe_kv_attend(const moe_kv_cache_t *cache, const moe_kv_step_t *step, const void *plan_dev, const int32_t *block_table,
                      const moe_kv_query_t *query, void *scratch, uint64_t scratch_bytes, void *stream);

/* The values that cached tokens stand for, rounded to dtype: k_out, v_out [n][kv_heads][head_dim], 16-byte aligned; a slot
 * outside the cache gives zeros. */
int32_t moe_kv_gather(const moe_kv_cache_t *cache, const int32_t *slots, int32_t n, int32_t dtype, void *k_out, void *v_out,
                      void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_KV_H */
