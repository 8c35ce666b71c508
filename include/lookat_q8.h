/*
 * lookat_q8.h - C ABI of the 8-bit paged cache (part of liblookat.so): the scalar-quantised counterpart of the code cache.
 *
 * The paper compares its product-quantised keys with symmetric 8-bit quantisation that is dequantised before the
 * product (Section 3.2, Section 4.1 "Baselines").  This is that cache in a form that can be served from: keys and
 * values in 8 bits with one scale per block of tokens and KV head, the blocks being pages that rows of any length own
 * through a table; attention that reads the 8-bit numbers as they are; and the upkeep of the pages (room for new tokens
 * with copy on write, forks of rows, compaction) on the device, without a host synchronisation.
 *
 * THE CACHE.  A page holds `page` tokens of every KV head; a block is one page of one KV head.  Its stored numbers n
 * stand for  n * amax / R,  amax the block's largest magnitude, R = 127 for int8 and 448 for e4m3.  amax is kept rather
 * than amax / R because it is an fp16 value: every quotient below then rounds as the real quotient does.
 *   Row b of a batch owns the pages tables[b][0 .. ceil(seq_lens[b] / page)), token t lying in page
 * tables[b][t / page] at place t % page.  Entries behind those are not read.  In all calls seq_lens already counts the
 * tokens of the running step: lookat_pages_extend raises it, lookat_q8_append fills the last n_new[b] tokens and
 * lookat_attend_q8 lets its L_q queries stand at the last L_q positions.
 *   A context serves one attention shape (its n_q_heads, n_kv_heads, d_k, d_v and scale; its codebook shape plays no
 * part here); d_k and d_v are multiples of 16 up to 256, else LOOKAT_ERR_UNSUPPORTED.  The pages_* calls use a context's
 * stream and device only.
 *
 * DEVICE-SIDE FINDINGS.  Lengths and tables live on the device, so the host cannot refuse them.  Kernels check each
 * entry before they use it: a length is taken as at least 0 and at most max_pages * page; the tokens of a page outside
 * 0..n_pages-1 are left out (not attended, not stored).  The finding is recorded in the context's status word and
 * lookat_last_error reports it once after the caller has synchronised, one kind of finding per call.  Nothing out of range is
 * read or written.
 *
 * WORKSPACE.  The context's scratch grows on demand; a call that would have to allocate while its stream is being
 * captured returns LOOKAT_ERR_INVALID_ARG (make one call of the same size before the capture).  Scratch that a graph
 * was captured with stays valid until the context is destroyed.  All calls of a context use the same scratch: run graphs
 * captured from one context one after another, and use a context per stream for work that overlaps.
 */
#ifndef LOOKAT_Q8_H
#define LOOKAT_Q8_H

#include "lookat.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    LOOKAT_Q8_INT8 = 0,    /* int8, R = 127 */
    LOOKAT_Q8_E4M3 = 1     /* 8-bit float, 4 exponent and 3 fraction bits, R = 448 */
};

/* The arrays of a cache (device memory of the caller, 16-byte aligned). */
typedef struct lookat_q8_cache {
    void *k;               /* 8-bit [n_pages][H_kv][page][d_k] */
    float *k_amax;         /* fp32 [n_pages][H_kv] */
    void *v;               /* 8-bit [n_pages][H_kv][page][d_v] */
    float *v_amax;         /* fp32 [n_pages][H_kv] */
    int32_t n_pages;
    int32_t page;          /* tokens per page: 16, 32, 64 or 128 */
    int32_t format;        /* LOOKAT_Q8_INT8 or LOOKAT_Q8_E4M3 */
} lookat_q8_cache;

/*
 * Quantises the newest tokens of every row into its pages.
 *
 *   k_new, v_new  fp16 [B][H_kv][n][d_k], [B][H_kv][n][d_v]; of row b the first n_new[b] tokens count
 *   tables        int32 [B][max_pages]
 *   seq_lens      int32 [B], lengths that count the new tokens: they go to positions seq_lens[b] - n_new[b] ...
 *   n_new         NULL (n for every row) or int32 [B], up to n; negative counts are taken as 0, as lookat_pages_extend does
 * Per block, with x the new tokens in it (NaN taken as 0, infinities as +-65504):
 *   amax' = max(amax if the block holds earlier tokens of the row, else 0; |x|)
 *   new numbers     n = round(R x / amax')        earlier ones, where amax has grown:  n = round(n amax / amax')
 * rounded to the nearest number, ties to even, as in real arithmetic; amax' = 0 gives n = 0.  Places behind the row's
 * last token are left as they were.  A page that a call writes belongs to one row (lookat_pages_extend sees to it).
 * Requires 1 <= n <= 2^20.
 */
lookat_status lookat_q8_append(lookat_ctx *ctx, const lookat_q8_cache *cache, const void *k_new, const void *v_new, int32_t B,
                               int32_t n, const int32_t *tables, int32_t max_pages, const int32_t *seq_lens,
                               const int32_t *n_new);

/*
 * Attention over the cache: for query i of L_q, at position p = seq_lens[b] - L_q + i,
 *   s_t = q . k_t * scale,  alpha = softmax of s over the tokens t = 0..p,  o = sum_t alpha_t v_t.
 * One generated token (L_q = 1), a few draft tokens, or a prompt or a piece of it.  A query without a token to attend
 * (p < 0, an empty row) gives zeros.  What lies behind a row's last token may be anything; the row's own numbers and
 * scales are finite (lookat_q8_append writes no others: a NaN among the values reaches every query of the row).
 *
 *   q          fp16 [B][H_q][L_q][d_k]
 *   tables     int32 [B][max_pages];  seq_lens  int32 [B]
 *   out        [B][H_q][L_q][d_v], fp32, or fp16 with out_fp16 = 1
 * Scores, softmax statistics and sums are fp32.  The weights of the sum are two fp16 numbers each: 22 bits for a token
 * whose weight times its block's amax is at least 2^-13 of the row's largest such product, fewer below, none below 2^-35.
 * With out_fp16 those of prompts (more than 16 queries times heads of a group) are one fp16 number: 11 bits down to 2^-21.
 * Requires 1 <= B <= 65535, 1 <= L_q <= 2^20, H_q * L_q <= 2^30.
 * Returns LOOKAT_ERR_TIMEOUT once if an earlier attention kernel of the context gave up a bounded wait (its output is not
 * valid).
 */
lookat_status lookat_attend_q8(lookat_ctx *ctx, const lookat_q8_cache *cache, const void *q, int32_t B, int32_t L_q,
                               const int32_t *tables, int32_t max_pages, const int32_t *seq_lens, void *out, int32_t out_fp16);

/* The pages of a batch (device arrays).  refs[p] counts who holds page p: table entries of live rows, and whatever the
 * caller adds for holders of its own.  free_list[0 .. *n_free) is a stack of the pages with refs 0; what lies above it is
 * not changed. */
typedef struct lookat_page_state {
    int32_t *tables;       /* [B][max_pages] */
    int32_t *seq_lens;     /* [B] */
    int32_t *refs;         /* [n_pages] */
    int32_t *free_list;    /* [n_pages] */
    int32_t *n_free;       /* [1] */
    int32_t B;             /* rows, up to 4096 */
    int32_t max_pages;
    int32_t n_pages;       /* up to 2^20 */
    int32_t page;          /* tokens per page: 16, 32, 64 or 128 */
} lookat_page_state;

/* One array that is kept by pages: page p is the page_bytes bytes at base + p * page_bytes.  A cache is four of them
 * (k, v, k_amax, v_amax), a model four per layer.  page_bytes is a multiple of 4, base 16-byte aligned. */
typedef struct lookat_page_pool {
    void *base;
    int64_t page_bytes;
} lookat_page_pool;
enum { LOOKAT_MAX_POOLS = 256 };

/*
 * Room for n_new[b] more tokens in every row; seq_lens rises by n_new.  Rows in order: a row that has a begun last page
 * (seq_lens % page != 0) held by others too (refs > 1, counting down as rows of this call leave it) gets a copy of it in
 * every pool -- the last of the holders keeps the page --, then a page for each further block.  Pages come off the top
 * of the free list.  All or nothing: if the pages do not suffice, a row would pass max_pages, or a length or a begun page's
 * entry is out of range, nothing changes but n_new, which is set to 0 for every row, and lookat_last_error reports it.
 *   n_new   in/out int32 [B]; negative counts are taken as 0, and a row with 0 keeps its pages as they are
 */
lookat_status lookat_pages_extend(lookat_ctx *ctx, const lookat_page_state *state, int32_t *n_new, const lookat_page_pool *pools,
                                  int32_t n_pools);

/*
 * Every row b continues from row parents[b] as it was before the call (a beam reorder); several rows may name the same
 * parent, and then share all of its pages.  A parent outside 0..B-1 leaves the row empty.  Pages that no row holds any
 * longer go onto the free list in ascending order.
 *   parents  int32 [B]
 */
lookat_status lookat_pages_fork(lookat_ctx *ctx, const lookat_page_state *state, const int32_t *parents);

/*
 * Moves the U pages with refs > 0 into pages 0..U-1: those already there stay, the others, in ascending order, fill the
 * gaps in ascending order.  Tables, refs and the pools follow; the free list becomes n_pages-1 down to U (U on top).
 *   remap  NULL, or out int32 [n_pages]: where each page went (itself if it stayed), -1 for pages with refs 0
 */
lookat_status lookat_pages_compact(lookat_ctx *ctx, const lookat_page_state *state, const lookat_page_pool *pools, int32_t n_pools,
                                   int32_t *remap);

#ifdef __cplusplus
}
#endif
#endif /* LOOKAT_Q8_H */
