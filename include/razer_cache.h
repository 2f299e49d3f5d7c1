/*
 * razer_cache.h -- the 8-bit paged key/value cache of the MI355X (gfx950) RaZeR library and the
 * attention that reads it: what a decoder layer needs between its {q,k,v} and its o projection.
 *
 *   razer_cache_plan       block tables, slots, positions and offsets of one serving step, from the
 *                          requests' lengths (once per step)
 *   razer_cache_append     the step's new keys and values into the cache (once per layer)
 *   razer_cache_attention  the step's queries over the cached keys and values (once per layer)
 *
 * Format.  Elements are FP8-E4M3 codes (S|EEEE|MMM, value 2^(E-7)(1+M/8), E=0: M/512; the equation
 * of the activation scales in razer.h).  Each page of `page` tokens has, per key/value head, one
 * exponent byte b for its keys and one for its values; an element's value is code * 2^(b-127), exact
 * in bf16.  b is the smallest byte in [RAZER_CACHE_MIN_EXPONENT, RAZER_CACHE_MAX_EXPONENT] with
 * absmax <= 448 * 2^(b-127) over what the page holds; it only grows while a page fills, and codes
 * already there are then divided by the power of two and rounded to nearest even (exact except at
 * the subnormal end).  The range is 2^-50 .. 2^50 times that of E4M3; beyond it elements saturate or
 * become 0.  A byte outside the range (of a page that no token was written to) is read as the nearer
 * end of it.  The scale is a power of two because a page fills token by token: any other scale would
 * round every element again each time it grows.
 *
 * Like razer.h: device pointers, the caller's stream, status codes, no allocation, no
 * synchronisation, nothing kept from one call to the next.  All values that steer memory accesses
 * on the device (slots, table entries, offsets) are checked there: an entry out of range is skipped
 * or counts as absent.
 */
#ifndef RAZER_CACHE_H
#define RAZER_CACHE_H

#include "razer.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RAZER_CACHE_MIN_EXPONENT 77
#define RAZER_CACHE_MAX_EXPONENT 177

typedef struct {
    uint8_t *k_codes;          /* [pages][kv_heads][page][head_dim]                     */
    uint8_t *v_codes;          /* [pages][kv_heads][head_dim][page]: tokens contiguous  */
    uint8_t *k_scales;         /* [pages][kv_heads] exponent bytes                      */
    uint8_t *v_scales;         /* [pages][kv_heads]                                     */
    int64_t pages;
    int32_t kv_heads;          /* 1 .. 8192                                             */
    int32_t head_dim;          /* 64, 128, 192 or 256                                   */
    int32_t page;              /* tokens per page: 16, 32, 64 or 128                    */
} razer_cache;

/* The bookkeeping of one step over `requests` requests, request r with lens[r] tokens in the cache and
 * fresh[r] new ones (each >= 0, together at most `tokens`; the rest of the step's `tokens` rows is padding):
 *   cu[requests+1]     offsets of the requests' new tokens (exclusive sums of fresh)
 *   total[requests]    lens + fresh
 *   table              [requests][ld_table], table_width entries used: entry i is the page of the request's
 *                      tokens i*page .. i*page+page-1.  The entries of the first ceil(lens/page) pages are
 *                      read, those of the pages that the new tokens begin are written: pages are taken from
 *                      free_pages[0 .. free_count) in the order of the requests, -1 where the list is too short.
 *   slots[tokens]      page * page_tokens + place of each new token; -1: no page, past table_width, or padding
 *   positions[tokens]  position of the token in its request (padding: 0)
 *   request_of[tokens] its request (padding: -1)
 *   used[1]            pages that the step wants from the list (> free_count: some tokens got none)
 * Any of positions and request_of may be NULL.  lens, fresh, free_pages and the outputs must not overlap.
 * `page` as in razer_cache.                                                                          */
razer_status razer_cache_plan(const int32_t *lens, const int32_t *fresh, int32_t requests,
                              int32_t *table, int32_t table_width, int64_t ld_table,
                              const int32_t *free_pages, int32_t free_count, int32_t page, int64_t tokens,
                              int32_t *cu, int32_t *total, int64_t *slots, int32_t *positions,
                              int32_t *request_of, int32_t *used, void *hip_stream);

/* Quantizes keys and values of `tokens` tokens into the slots that razer_cache_plan gave them.
 *   k, v     device, dtype fp32 or bf16: element d of head h of token t at t * ld + h * head_dim + d
 *   slots    [tokens]; negative or beyond the cache: the token is skipped
 * In one call the tokens of one page have to stand within `page` rows, in ascending slots, with no other
 * page's token between them (as razer_cache_plan leaves them); any of them may be skipped, and slots may be
 * left out: such a place keeps what it held, and attention over the page reads that.  Tokens in consecutive
 * rows and slots are encoded together, a page's stretches of them one after the other.  A page is begun anew
 * when its place 0 is written, and what it held is then of no concern; without place 0 it goes on with the
 * exponent byte that it has.  Non-finite elements: NaN is stored as 0, an infinity as +-448 * 2^(b-127), and
 * neither counts for the scale, so that no later reader of the page meets them.
 * Requirements: k, v and the cache's codes 16-byte aligned, ld * sizeof(elt) % 16 == 0,
 * ld >= kv_heads * head_dim, tokens < 2^24, tokens * kv_heads < 2^26.                                */
razer_status razer_cache_append(const razer_cache *cache, const void *k, int64_t ld_k, const void *v, int64_t ld_v,
                                int32_t dtype, int64_t tokens, const int64_t *slots, void *hip_stream);

/* Attention of new tokens over the cache.  Request r has n = cu[r+1] - cu[r] query tokens, the last n of
 * its total[r]: token i of them stands at position p = total[r] - n + i.  Query head h reads key/value
 * head h / (q_heads / kv_heads).  The scores of query (i, h) are
 *     s_j = scale * <q, k_j>;   cap > 0: s_j = cap * tanh(s_j / cap);   slopes: s_j -= slopes[h] * |p - j|
 * over the keys j < total[r] that it sees:
 *     (j <= p and (window == 0 or j > p - window)) or j < prefix[r]
 * (prefix: tokens that every query of the request sees, before or behind it, inside or outside the
 * window).  out = sum_j softmax(s)_j v_j, rounded to bf16 once; 0 for a query that sees no key.  A key
 * whose table entry is not a page of the cache, or lies past table_width, counts as not seen, and so
 * do keys from 2^30 on.
 * Products are accumulated in fp32, queries and exactly decoded keys multiplied as bf16, the softmax's
 * maxima and sums held in fp32.  A cap of any size costs a score at most 2^-18 of itself.  For the product
 * with the values (exactly decoded f16) a weight times its page's scale is rounded to f16, relative to the
 * largest such product of the row.
 * cu, total, table and prefix may begin at any of a step's requests: the other requests' rows of out are left
 * alone.  The kernel follows from the longest new part, so a step of prompts beside requests with few new
 * tokens and many keys is faster as two calls.                                                          */
typedef struct {
    const void *q;             /* bf16: head h of token t at t * ld_q + h * head_dim    */
    int64_t ld_q;
    void *out;                 /* bf16, the same with ld_out                            */
    int64_t ld_out;
    int64_t tokens;            /* rows of q and out; those outside cu[0] .. cu[requests] are not touched */
    int32_t q_heads;           /* a multiple of kv_heads                                */
    int32_t requests;
    const int32_t *cu;         /* [requests+1]                                          */
    const int32_t *total;      /* [requests]                                            */
    const int32_t *table;      /* [requests][ld_table]                                  */
    int64_t ld_table;
    int32_t table_width;
    int32_t max_new;           /* about how many new tokens a request has at most, and  */
    int64_t max_len;           /* how long one is at most: both only choose kernels and */
                               /* the split of the work, any value gives right results; */
                               /* <= 0: unknown                                         */
    float scale;
    float cap;                 /* 0: none                                               */
    int32_t window;            /* 0: none                                               */
    const float *slopes;       /* [q_heads] or NULL                                     */
    const int32_t *prefix;     /* [requests] or NULL                                    */
} razer_attention;

/* workspace: device, 16-byte aligned, >= razer_attention_workspace_bytes(cache, args) bytes (0: may be
 * NULL), which depends on the sizes, max_new, max_len and the window alone.  It is no smaller for a larger
 * max_len (<= 0: the largest) and no larger with a window than without one, so that one allocation serves
 * every window and every shorter length; calls that overlap in time need their own.
 * Requirements: q, out and the cache's codes 16-byte aligned, ld_q and ld_out multiples of 8 and
 * >= q_heads * head_dim; tokens * q_heads <= 2^27, requests * kv_heads <= 2^22.  */
size_t razer_attention_workspace_bytes(const razer_cache *cache, const razer_attention *args);
razer_status razer_cache_attention(const razer_cache *cache, const razer_attention *args,
                                   void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* RAZER_CACHE_H */
