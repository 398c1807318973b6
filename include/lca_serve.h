/*
 * liblca — operators of a serving step around the condensed attention of lca.h: ragged batches over a paged cache held
 * in 8 bits, and packed prompts, for AMD MI355X (gfx950), C ABI.
 *
 * The calls of lca.h take B sequences of one length in buffers of their own.  Layers that stay dense, requests shorter
 * than the window, and batches whose requests come and go need the forms below: B requests of any lengths whose T new
 * rows (tokens) lie behind one another, keys and values in blocks of `page` tokens from one pool, and scores that may be
 * capped, biased by distance and masked by document, window and prefix.
 *
 * Score rule of both attention calls, for the row at position i of a request (document) and its key at position j:
 *     s = scale * <q_i, k_j>;   softcap > 0: s = softcap * tanh(s / softcap);   slopes: s = s - slopes[h] * |i - j|
 *     visible(i, j) = 0 <= j < n  and  ( (j <= i and (window == 0 or i - j < window))  or  j < prefix_len )
 * with n the tokens of the request.  O = softmax-weighted sum of the visible values, lse = ln sum exp s; a row that sees
 * nothing gets O = 0 and lse = -infinity.  Keys and values that a row does not see have no part in it, whatever they hold
 * (infinities and NaN included).  S is the number of KV heads, query head h uses KV head h / (H / S).  As in lca.h's
 * GQA mode SEL are the keys and POOL the values.
 *
 * The cache.  A pool of n_blocks blocks of `page` tokens; a token's slot is block * page + place in the block.
 *     sel_q8  [n_blocks, S, page, d_sel]           codes of the keys
 *     pool_q8 [n_blocks, S, page / 16, d_pool, 16]  codes of the values, sixteen tokens of a column next to each other
 *     scales  [n_blocks, S, 2] float                (pooled, selected): a power of two per block, KV head and component
 * Codes are OCP FP8 E4M3 bytes and stand for decode(code) * scale.
 *
 * Conventions are those of lca.h: device pointers, 16-byte aligned (index and float arrays: 4-byte), row-major, the
 * caller owns every buffer and the stream, nothing is allocated, nothing synchronised, an lca_status, lca_last_error().
 * What the device arrays hold cannot be checked on the host; the kernels check it, and none of it makes them read or write
 * outside the buffers: a block number outside [0, n_blocks) has no tokens to see and takes none, a length beyond
 * max_blocks * page counts as that many, starts outside [0, T] are clamped.  Two calls that overlap in time need
 * workspaces of their own.
 */
#ifndef LCA_SERVE_H
#define LCA_SERVE_H

#include "lca.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int32_t B, T;               /* requests (documents); rows of the packed arrays (>= the step's tokens)           */
    int32_t H, S;               /* query heads, KV heads (H % S == 0)                                               */
    int32_t d_pool, d_sel;      /* widths of values and keys: multiples of 8 (f32: 4) up to 1024; cache: of 16, up to 256 */
    int32_t dtype;              /* lca_dtype of Q, SEL, POOL, O; the cache calls take the two 16-bit types           */
    int32_t page;               /* tokens of a block: a multiple of 16 up to 1024                                   */
    int32_t n_blocks;           /* blocks of the pool; n_blocks * page < 2^31                                       */
    int32_t max_blocks;         /* columns of the block table; max_blocks * page <= 2^30                            */
    int32_t max_q, max_kv;      /* most new rows of a request, longest request: hints for how the work is split, 0 = not known; results never depend on
                                   their being right beyond rounding, speed does                                    */
    int32_t window;             /* 0 = none                                                                         */
    float scale, softcap;       /* softcap 0 = none; 16-bit types: up to 1024.  Refused where scale * log2(e), 2 softcap * log2(e) or their quotient is beyond fp32 */
    int64_t q_row, sel_row, pool_row;   /* elements between tokens of Q, SEL, POOL (a piece of a fused projection), multiples of 16 bytes; 0 = H * d_sel,
                                   S * d_sel, S * d_pool.  Heads of a token are contiguous; O is always [T,H,d_pool]  */
} lca_serve_desc;

/* Bytes of workspace that any call below needs for this descriptor (host only). */
lca_status lca_serve_workspace_size(const lca_serve_desc *desc, size_t *bytes);

/*
 * Block tables, slots and positions of one step, from the requests' lengths (B, T, page, n_blocks, max_blocks are read).
 * Request b holds cached_len[b] tokens, in blocks block_table[b][0 .. ceil(cached_len[b] / page)), and brings new_len[b]
 * (0: none) that follow one another in the packed arrays, request after request.  New blocks come from the top of a stack,
 * in request order: with need_b = ceil((cached_len + new_len) / page) - ceil(cached_len / page) and cum_b its sum up to and
 * including b, the r-th of request b is free_list[free_count - 1 - (cum_b - need_b) - r].
 * A request is refused -- gets no blocks, slots of -1, seq_len 0 -- if its rows end behind T, its tokens do not fit
 * max_blocks, a length is negative (need_b = 0 in these cases), or need_b > 0 and cum_b > free_count.  What it holds stays as it
 * is: its cached_len is the caller's to keep (seq_len of the others is their next cached_len).
 * In:  cached_len, new_len [B], free_list [n_blocks], free_count [1].
 * Out: free_left [1] (may be free_count itself), block_table [B,max_blocks] (new entries only), q_start [B+1] (clamped to T),
 *      seq_len [B] (cached_len + new_len), slot, position, request [T] (rows behind the last request: -1, 0, -1).
 * All int32.
 */
lca_status lca_page_tables(const lca_serve_desc *desc, const int32_t *cached_len, const int32_t *new_len, const int32_t *free_list, const int32_t *free_count,
                           int32_t *free_left, int32_t *block_table, int32_t *q_start, int32_t *seq_len, int32_t *slot, int32_t *position, int32_t *request,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * Finished requests give their blocks back: for every b with finished[b] != 0, in order, the entries block_table[b][0 ..
 * ceil(cached_len[b] / page)) that are block numbers are pushed on the stack and become -1, and cached_len[b] becomes 0
 * (so that a second release returns nothing).  A push beyond n_blocks is dropped.
 * In: finished [B].  In and out: cached_len [B], block_table, free_list, free_count.  All int32.
 */
lca_status lca_page_release(const lca_serve_desc *desc, const int32_t *finished, int32_t *cached_len, int32_t *block_table, int32_t *free_list,
                            int32_t *free_count, void *stream);

/*
 * Writes the keys and values of T tokens into the cache at slot[t] (outside [0, n_blocks * page): the token is skipped).
 * The tokens of a block that one call writes follow one another in the packed arrays, in slots that do, as
 * lca_page_tables lays them out; a block that a call names in two places holds codes of either, its other blocks are not
 * affected.  Per block, KV head and component, with amax the largest finite or infinite magnitude of the new values:
 *     e = the exponent with amax / 2^e in (224, 448], within [-100, 119] (bf16) or [-15, 7] (f16); the lowest for amax = 0
 * If the first new slot is not the block's first, the block's older tokens stay: the scale becomes the larger of 2^e
 * and the old one, and if it rose they are recoded (decode(code) * old / new, to the nearest code).  A new value x becomes the code
 * nearest to x / scale (ties to even), magnitudes beyond 448 the code of 448, NaN a NaN.
 * In:  SEL [T,S,d_sel], POOL [T,S,d_pool], slot [T].  In and out: sel_q8, pool_q8, scales.
 */
lca_status lca_page_store_q8(const lca_serve_desc *desc, const void *SEL, const void *POOL, const int32_t *slot, uint8_t *sel_q8, uint8_t *pool_q8,
                             float *scales, void *stream);

/*
 * Attention of a step's rows over the cache: single tokens, a few at a time, chunks of prompts, in one batch.  Request b
 * has rows q_start[b] .. q_start[b+1]-1, the last of its seq_len[b] tokens (all in the cache); a row whose position would
 * be negative sees nothing.  Rows behind q_start[B] are left as they are.
 * In:  q [T,H,d_sel], q_start [B+1], seq_len [B], prefix_len [B] or NULL (0), slopes [H] float or NULL, block_table
 *      [B,max_blocks], sel_q8, pool_q8, scales.
 * Out: O [T,H,d_pool], lse [T,H] float, may be NULL.
 */
lca_status lca_page_attn_q8(const lca_serve_desc *desc, const void *q, const int32_t *q_start, const int32_t *seq_len, const int32_t *prefix_len,
                            const float *slopes, const int32_t *block_table, const uint8_t *sel_q8, const uint8_t *pool_q8, const float *scales, void *O,
                            float *lse, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention over packed prompts: document b is rows doc_start[b] .. doc_start[b+1]-1 of Q, SEL and POOL and sees itself
 * only, its first prefix_len[b] tokens in both directions.  Rows behind doc_start[B] are left as they are.
 * In:  Q [T,H,d_sel], SEL [T,S,d_sel], POOL [T,S,d_pool], doc_start [B+1], prefix_len [B] or NULL, slopes [H] float or NULL.
 * Out: O [T,H,d_pool], lse [T,H] float, may be NULL.
 */
lca_status lca_packed_attn(const lca_serve_desc *desc, const void *Q, const void *SEL, const void *POOL, const int32_t *doc_start,
                           const int32_t *prefix_len, const float *slopes, void *O, float *lse, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LCA_SERVE_H */
