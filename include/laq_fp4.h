/*
 * laq_fp4.h -- C ABI of the paged 4-bit cache that decoding continues on (part of liblaq.so).
 *
 * What an eviction keeps (Sec. 4.3) may go, instead of into laq_compact's packed rows, into a pool of blocks
 * that requests take and give back as they grow and shrink, with the rows' numbers in 4 bits: 68 bytes a row of
 * 128 instead of 256.  The steps, all of them on the device and free of host lengths, so that a decoding loop can be
 * captured:
 *   laq_block_map        lengths -> blocks of every request, a slot for every new row
 *   laq_fp4_store        rows of new tokens -> their slots
 *   laq_fp4_compact      the rows that laq_select names -> their slots
 *   laq_fp4_attention    tokens attend to the cache: one per request, a few, or a chunk of a prompt
 *   laq_fp4_load         rows back, as laq_score reads them (another eviction of the same cache)
 *
 * The conventions of laq.h hold: device pointers, work enqueued on `stream`, arguments checked before
 * anything is enqueued, no allocation, results a pure function of the inputs.  `budget` is a HOST array; lengths,
 * tables and slots are DEVICE arrays whose values the host cannot see: the kernels check every block number and slot
 * against the cache and touch nothing outside of it, whatever they hold.  Outputs do not overlap inputs.  Calls that use one cache,
 * one pool (rows, block_table, free_blocks, state) or one workspace run one after another: on one stream, or on streams that wait
 * for each other; several captured graphs may hold the same ones on that condition.  A batch of no tokens is LAQ_OK and does nothing.
 *
 * Numbers: a row of d numbers is d / 32 blocks of 32 in the microscaling format with 4-bit elements (e2m1): a scale byte s stands for
 * 2^(s - 127), a code for a sign (8) and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; number 2j of the row is in the low half of byte j,
 * 2j + 1 in the high one.  Stored, a block's scale is 2^(floor(log2 a) - 2) for its largest magnitude a, twice that from
 * a = 1.75 * 2^floor(log2 a) on (where rounding to the nearest would reach 8), held within 2^-100 and 2^125 (a block of zeros: 2^-100);
 * every number is rounded to the nearest code, ties to the even one.  A block with an infinity or a NaN gets s = 255 and codes 0,
 * and stands for NaN.  Scales that the library never stores: 0 .. 26 are numbers like the others; of 253 and 254, laq_fp4_load gives what does not
 * fit its type as infinities, and what laq_fp4_attention makes of requests that hold such rows is not defined.
 */
#ifndef LAQ_FP4_H
#define LAQ_FP4_H

#include "laq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A pool of n_blocks blocks of block_rows rows for each of Hkv KV heads, K and V apart. */
typedef struct laq_fp4_cache {
  uint8_t *k, *k_scale;  /* codes [n_blocks, Hkv, block_rows, d / 2] and scales [n_blocks, Hkv, block_rows, d / 32] */
  uint8_t *v, *v_scale;
  int32_t n_blocks;      /* >= 1; n_blocks * block_rows < 2^31 */
  int32_t Hkv;           /* <= 32768 */
  int32_t block_rows;    /* a multiple of 16 */
  int32_t d;             /* head size, a multiple of 32, <= 256 */
  /*
   * Distances in bytes between blocks, KV heads and rows, of the codes and of the scales; K and V alike.  All six zero: dense as
   * above.  Token-major blocks [block_rows, Hkv, ...]: {block, d / 2, Hkv * d / 2} and {block, d / 32, Hkv * d / 32}.  Those of
   * the codes are multiples of 16 (as are the codes' addresses); blocks are less than 2^32 apart, rows at most 2^27; rows must not
   * overlap (not checked).
   */
  int64_t stride_block, stride_head, stride_row;
  int64_t scale_stride_block, scale_stride_head, scale_stride_row;
} laq_fp4_cache;

/*
 * Block tables and slots from lengths: n requests change their numbers of rows, blocks are given back to a free list and taken from it.
 *   add          int32 [n]  rows that request i appends (> 0) or drops from its end (< 0; at most all of them)
 *   rows         int32 [n]  in: rows that it holds; out: rows that it holds then
 *   block_table  int32 [n, blocks_per_inst]  row j of request i is row j % block_rows of block block_table[i][j / block_rows].
 *                New blocks are entered; entries behind a request's last block are left as they were
 *   free_blocks  int32 [n_blocks]  the free blocks, a stack of state[0] entries
 *   state        int32 [4]  in and out: state[0] = number of free blocks; out: state[1] = number of requests refused; the others are
 *                the library's, 0 before the first call and after every one
 *   start        int32 [n + 1], may be NULL: the appended rows of request i are numbers start[i] .. start[i+1]-1 of the batch (exclusive
 *                sums of max(add, 0), at most 2^31 - 1), as laq_fp4_attention takes it
 *   slots        int32 [n_slots] (NULL with n_slots = 0: none): slots[start[i] + t] = block * block_rows + row in it, for the t-th
 *                appended row of request i.  -1: a row of a refused request, or an entry behind the last appended row (a
 *                batch padded to n_slots).  Rows from number n_slots on get no entry
 * First all blocks given back go on top of the list (those of the last request first, of each its last one first), then requests
 * take what they need from the top, in their order: dropping what was just appended restores the list.  A request is refused, its rows
 * left as they were, if it would need more than blocks_per_inst blocks, or if it needs blocks and those that it and the requests
 * before it need are more than there are.  Lengths outside of the table count as its nearest end, and state[0] as 0 .. n_blocks.
 * block_rows a multiple of 16, n_blocks * block_rows and blocks_per_inst * block_rows below 2^31; n * blocks_per_inst too
 * (LAQ_ERR_UNSUPPORTED).
 */
int laq_block_map(int32_t n, int32_t block_rows, int32_t n_blocks, int32_t blocks_per_inst, const int32_t *add, int32_t *rows,
                  int32_t *block_table, int32_t *free_blocks, int32_t *state, int32_t *start, int32_t *slots, int64_t n_slots,
                  void *stream);

/*
 * Rows of new tokens into the cache (the decoding after Sec. 4.3 appends a row per token).
 *   dtype         laq_dtype of k and v
 *   k, v          [n_tokens, Hkv, d], rows contiguous, stride_token and stride_head elements apart (both zero: dense); multiples
 *                 of 16 bytes, as are the addresses.  Both or one of them (the other NULL and left alone)
 *   slots         int32 [n_tokens] as laq_block_map writes them; a token whose slot is not one of the cache is left out.  Two
 *                 tokens of one call must not have the same slot (which of them each block of 32 numbers comes from is not defined)
 * n_tokens * Hkv * d / 8 up to 2^32 - 256 (LAQ_ERR_UNSUPPORTED), for laq_fp4_load too; a KV head's rows * 32 * Hkv for laq_fp4_compact.
 */
int laq_fp4_store(const laq_fp4_cache *cache, int32_t dtype, int64_t n_tokens, const void *k, const void *v, int64_t stride_token,
                  int64_t stride_head, const int32_t *slots, void *stream);

/*
 * Cache compaction into the 4-bit cache (laq_compact with another destination, Sec. 4.3).
 *   shape, k, v, idx, budget  as for laq_compact (strided and paged sources too); shape->Hkv and d are the cache's.  v may be NULL
 *   slots         int32 [sum of Bk(i)]: the slots of instance i's rows, for all its KV heads, start at the sum of Bk of earlier
 *                 instances; as laq_block_map writes them for add[i] = Bk(i)
 * Rows whose index is outside of [0, L) or whose slot is not one of the cache are left out.
 */
int laq_fp4_compact(const laq_shape *shape, const void *k, const void *v, const int32_t *idx, const int32_t *budget,
                    const laq_fp4_cache *cache, const int32_t *slots, void *stream);

/*
 * Rows of the cache as numbers: the inverse of laq_fp4_store.
 *   k, v          [n_tokens, Hkv, d] out, dense, of type dtype (exact in both: two bits of fraction and a power of two); one may be NULL
 *   slots         int32 [n_tokens]; a row whose slot is not one of the cache is 0
 */
int laq_fp4_load(const laq_fp4_cache *cache, int32_t dtype, int64_t n_tokens, const int32_t *slots, void *k, void *v, void *stream);

/*
 * Attention over the cache: tokens of n requests attend to the rows that their request holds, the tokens' own rows (the last ones)
 * among them, each to those up to its own.
 *   Hq, dtype, scale  query heads (a multiple of the cache's Hkv, <= 65535), laq_dtype of q and out, logit scale (<= 0: 1/sqrt(d))
 *   n_tokens      tokens of the batch; n_tokens * Hq < 2^31
 *   start         int32 [n + 1]: tokens start[i] .. start[i+1]-1 are those of request i, in order; ascending, start[0] = 0.
 *                 Tokens from start[n] on (padding) are left alone.  NULL: one token per request (n_tokens = n)
 *   q             [n_tokens, Hq, d], rows contiguous, stride_token and stride_head elements apart (both zero: dense); multiples of
 *                 16 bytes, as is the address
 *   block_table   int32 [n, blocks_per_inst]; rows of blocks whose number is not one of the pool are not there for anybody
 *   rows          int32 [n]: rows that request i holds; at most blocks_per_inst * block_rows count
 *   max_rows      the caller's bound on them, from which the launch is planned (rows beyond are attended to all the same, more
 *                 slowly); 1 .. blocks_per_inst * block_rows
 *   out           [n_tokens, Hq, d] of type dtype, dense: token t of the T tokens of a request of r rows sees rows 0 .. r - T + t;
 *                 out = sum_j softmax_j(scale * <q, K_j>) V_j over these.  0 where there are none
 *   lse           fp32 [n_tokens, Hq], may be NULL: log sum_j exp(scale * <q, K_j>) (-infinity where there are none): with it two
 *                 attentions over different rows can be joined
 *   ws / ws_bytes optional device scratch.  With at least laq_fp4_attention_workspace_bytes() bytes (same arguments), long rows of
 *                 small calls are spread over several workgroups; LAQ_ERR_WORKSPACE if given but smaller or not 16-byte aligned.
 *                 With and without it the last bits of `out` may differ
 * A call that needs more than 2^24 workgroups (about n * Hkv of them, or n_tokens * Hq / 16) is LAQ_ERR_UNSUPPORTED.
 * bf16: the products of q and K are exact, sums, maxima and weights are fp32, weights are rounded to bf16 for the product with V, out
 * is rounded once.  fp32: q and weights as three bf16 parts each (2^-24), V exact, sums fp32.  Weights are up to 2^8 before they are divided by their sum: sums over
 * numbers of V beyond 2^88 may overflow.
 */
size_t laq_fp4_attention_workspace_bytes(const laq_fp4_cache *cache, int32_t Hq, int32_t dtype, int32_t n, int64_t n_tokens,
                                         int32_t max_rows);
int laq_fp4_attention(const laq_fp4_cache *cache, int32_t Hq, int32_t dtype, float scale, int32_t n, int64_t n_tokens,
                      const int32_t *start, const void *q, int64_t stride_token, int64_t stride_head, const int32_t *block_table,
                      int32_t blocks_per_inst, const int32_t *rows, int32_t max_rows, void *out, float *lse, void *ws,
                      size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LAQ_FP4_H */
