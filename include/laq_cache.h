/*
 * laq_cache.h -- C ABI of rotary positions and of the paged cache in 32, 16 or 8 bits (part of liblaq.so).
 *
 * The caches of this library hold keys that are rotated to their positions, and an eviction (Sec. 4.3) leaves every kept key at the
 * position it had.  laq_rope rotates queries and keys of new tokens; the paged cache holds what an eviction keeps as it is (fp32, bf16) or
 * in 8 bits (129 bytes a row of 128), and grows with the tokens, where the packed rows of laq_compact cannot.  All of it is on the device
 * and free of host lengths, so that a decoding loop can be captured:
 *   laq_block_map (laq_fp4.h)  lengths -> blocks of every request, a slot for every new row
 *   laq_cache_append           rows of new tokens -> their slots, keys (and queries) rotated on the way
 *   laq_cache_compact          the rows that laq_select names -> their slots
 *   laq_cache_attention        tokens attend to the cache: one per request, a few, or a chunk of a prompt
 *   laq_cache_load             rows back, as laq_score reads them (another eviction of the same cache)
 *
 * The conventions of laq.h hold: device pointers, work enqueued on `stream`, arguments checked before anything is enqueued, no
 * allocation, results a pure function of the inputs.  Lengths, tables, slots and positions are DEVICE arrays whose values the host
 * cannot see: the kernels check every block number and slot against the cache and touch nothing outside of it, whatever they hold.  Outputs do
 * not overlap inputs, but laq_rope's and laq_cache_append's rotated heads may be written where they are read (same address and strides).
 * Calls that use one cache or one workspace run one after another: on one stream, or on streams that wait for each other; several
 * captured graphs may hold the same ones on that condition.  A batch of no tokens is LAQ_OK and does nothing.
 *
 * 8 bits: a row of d numbers of one KV head is a scale byte s, which stands for 2^(s - 127), and d numbers in e4m3 (sign, 4 bits of
 * exponent, 3 of fraction; largest 448, no infinities).  Stored, the scale is 2^(floor(log2 a) - 8) for the row's largest magnitude a, twice
 * that above 1.75 * 2^floor(log2 a) (what 448 does not reach), at least 2^-100 (a row of zeros: 2^-100); every number is rounded to the nearest,
 * ties to even.  A row with an infinity or a NaN gets s = 255 and zeros, and stands for NaN.  Of scales that the library never stores,
 * 0 .. 26 and 248 .. 254 stand for what they say as long as 32 bits hold it.
 */
#ifndef LAQ_CACHE_H
#define LAQ_CACHE_H

#include "laq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The third type that a cache's numbers can have, beside those of laq_dtype. */
enum { LAQ_E4M3 = 2 };

/* Rows of tokens: [n_tokens, heads, d], the d numbers contiguous.  Distances in elements; both zero: dense.  Strides are multiples of 16 bytes, as is
 * the address. */
typedef struct laq_heads {
  void *x;               /* NULL: none */
  int32_t heads;
  int64_t stride_token, stride_head;
} laq_heads;

/* Which numbers of a head make the pairs that are rotated. */
typedef enum { LAQ_ROPE_HALF = 0, LAQ_ROPE_INTERLEAVED = 1 } laq_rope_layout;

/*
 * Rotary positions: of the first `rot` numbers of a head, pair i -- (i, i + rot / 2) in the half layout, (2i, 2i + 1) in the interleaved one -- is turned by
 * position * inv_freq[i] and multiplied with mscale; the numbers behind them stay as they are.
 *   inv_freq   DEVICE fp32 [rot / 2], any frequencies (scaled ones for long contexts, see laq_rope_frequencies of the Python package) with which angles
 *              stay below 2^40
 *   rot        even, 2 <= rot <= d
 *   mscale     factor of both sine and cosine; finite (1: a rotation)
 * Positions are int32, negative ones too (a key moved back).  The angle is a product in 64 bits, reduced and its sine and cosine taken there,
 * and these, times mscale, are rounded to fp32; the rotation is made in fp32 (two products and their sum, each rounded) and rounded once to the type of the output.
 */
typedef struct laq_rope_plan {
  const float *inv_freq;
  int32_t rot;
  int32_t layout;        /* laq_rope_layout */
  float mscale;
} laq_rope_plan;

/*
 * Rotates heads of tokens.
 *   dtype        laq_dtype of q, k, q_out, k_out
 *   d            head size, a multiple of 8, <= 256
 *   q, k         rows of tokens; one of them may be NULL or have x = NULL
 *   q_out, k_out out, of as many heads
 *   positions    int32 [n_tokens]
 * Up to 2^25 tokens (LAQ_ERR_UNSUPPORTED beyond), for laq_cache_append too.
 */
int laq_rope(const laq_rope_plan *rope, int32_t dtype, int64_t n_tokens, int32_t d, const laq_heads *q, const laq_heads *k, const int32_t *positions,
             const laq_heads *q_out, const laq_heads *k_out, void *stream);

/* A pool of n_blocks blocks of block_rows rows for each of Hkv KV heads, K and V apart. */
typedef struct laq_cache {
  void *k, *v;                  /* [n_blocks, Hkv, block_rows, d] of type `type` */
  uint8_t *k_scale, *v_scale;   /* LAQ_E4M3: [n_blocks, Hkv, block_rows], dense; otherwise not used */
  int32_t n_blocks;             /* >= 1; n_blocks * block_rows < 2^31 */
  int32_t Hkv;                  /* <= 32768 */
  int32_t block_rows;           /* a multiple of 16 */
  int32_t d;                    /* head size, a multiple of 8, <= 256 */
  int32_t type;                 /* LAQ_F32, LAQ_BF16 or LAQ_E4M3 */
  /*
   * Distances in elements between blocks, KV heads and rows of k and of v.  All three zero: dense as above.  Token-major blocks [block_rows, Hkv, d]:
   * {block_rows * Hkv * d, d, Hkv * d}.  Multiples of 8; rows at most 2^24 apart; rows must not overlap (not checked).  All four addresses are
   * multiples of 16 bytes.
   */
  int64_t stride_block, stride_head, stride_row;
} laq_cache;

/*
 * Rows of new tokens into the cache (the decoding after Sec. 4.3 appends a row per token).
 *   dtype        laq_dtype of k, v, q, q_out; every one goes with every type of cache (rounded once, or quantised as above)
 *   k, v         [n_tokens, Hkv, d]; both or one of them (the other NULL, or x = NULL, and left alone)
 *   slots        int32 [n_tokens], slot = block * block_rows + row as laq_block_map writes them; a token whose slot is not one of the cache is
 *                left out.  Two tokens of one call must not have the same slot (which of them each part of the row comes from is not defined)
 *   rope, positions   NULL: k is stored as it is.  Otherwise k is rotated first (v never)
 *   q, q_out     with rope: queries of the same tokens, rotated as laq_rope does (those without a slot too); NULL: none
 * Numbers go from the rotation to the cache's type in one rounding.
 */
int laq_cache_append(const laq_cache *cache, int32_t dtype, int64_t n_tokens, const laq_heads *k, const laq_heads *v, const int32_t *slots,
                     const laq_rope_plan *rope, const int32_t *positions, const laq_heads *q, const laq_heads *q_out, void *stream);

/*
 * Cache compaction into the paged cache (laq_compact with another destination, Sec. 4.3).
 *   shape, k, v, idx, budget  as for laq_compact (strided and paged sources too); shape->Hkv and d are the cache's.  v may be NULL
 *   slots         int32 [sum of Bk(i)]: the slots of instance i's rows, for all its KV heads, start at the sum of Bk of earlier
 *                 instances; as laq_block_map writes them for add[i] = Bk(i)
 * Rows whose index is outside of [0, L) or whose slot is not one of the cache are left out.  Up to 2^26 rows of an instance and KV head
 * (LAQ_ERR_UNSUPPORTED beyond).
 */
int laq_cache_compact(const laq_shape *shape, const void *k, const void *v, const int32_t *idx, const int32_t *budget, const laq_cache *cache,
                      const int32_t *slots, void *stream);

/*
 * Rows of the cache as numbers.
 *   k, v          [n_tokens, Hkv, d] out, dense, of type dtype (rounded where that has fewer bits than the cache); one may be NULL
 *   slots         int32 [n_tokens]; a row whose slot is not one of the cache is 0
 * n_tokens * Hkv up to 2^26 (LAQ_ERR_UNSUPPORTED beyond).
 */
int laq_cache_load(const laq_cache *cache, int32_t dtype, int64_t n_tokens, const int32_t *slots, void *k, void *v, void *stream);

/*
 * Attention over the cache: tokens of n requests (1 at least) attend to the rows that their request holds, the tokens' own rows (the last ones) among
 * them, each to those up to its own.
 *   Hq, dtype, scale  query heads (a multiple of the cache's Hkv, <= 65535), laq_dtype of q and out, logit scale (<= 0: 1/sqrt(d)).  LAQ_BF16 goes with
 *                 caches of LAQ_BF16 and LAQ_E4M3 (LAQ_ERR_UNSUPPORTED with LAQ_F32), LAQ_F32 with all
 *   n_tokens      tokens of the batch; n_tokens * Hq < 2^31
 *   start         int32 [n + 1]: tokens start[i] .. start[i+1]-1 are those of request i, in order; ascending, start[0] = 0.
 *                 Tokens from start[n] on (padding) are left alone.  NULL: one token per request (n_tokens = n).  Of numbers in another order
 *                 nothing is touched but out, lse and ws, and what they hold afterwards is not defined
 *   q             [n_tokens, Hq, d]: q->heads = Hq
 *   block_table   int32 [n, blocks_per_inst]; rows of blocks whose number is not one of the pool are not there for anybody
 *   rows          int32 [n]: rows that request i holds; at most blocks_per_inst * block_rows count
 *   max_rows      the caller's bound on them, from which the launch is planned (rows beyond are attended to all the same, more
 *                 slowly); 1 .. blocks_per_inst * block_rows
 *   out           [n_tokens, Hq, d] of type dtype, dense: token t of the T tokens of a request of r rows sees rows 0 .. r - T + t;
 *                 out = sum_j softmax_j(scale * <q, K_j>) V_j over these.  0 where there are none
 *   lse           fp32 [n_tokens, Hq], may be NULL: log sum_j exp(scale * <q, K_j>) (-infinity where there are none): with it two
 *                 attentions over different rows can be joined
 *   ws / ws_bytes optional device scratch, as it comes.  With at least laq_cache_attention_workspace_bytes() bytes (same arguments; it does not grow with
 *                 max_rows) the keys of all requests are shared out evenly among as many workgroups as the device holds; without it a KV head's
 *                 keys are read by one workgroup for every 16 or 32 score rows.  0 bytes: the batch is taken for chunks of a prompt (bf16, d <= 128,
 *                 more than 32 score rows per request on average, padding counted, and enough workgroups), where a workgroup reads a KV head's keys
 *                 for 128 score rows.  That is so for every request of the batch: decoding requests of long caches beside a chunk, and decoding
 *                 batches with much padding, take less time in calls of their own and without it.  LAQ_ERR_WORKSPACE if given but
 *                 smaller or not 16-byte aligned.  With and without it the last bits of `out` may differ
 * A call that needs more than 2^24 workgroups is LAQ_ERR_UNSUPPORTED.  What the rows behind r, other blocks of the pool and rows that a token does
 * not see hold (infinities and NaN too) does not reach out or lse.
 * bf16: the products of q and K are exact, sums, maxima and weights are fp32; for the product with V a weight is the sum of two bf16 (2^-16), in
 * chunks of a prompt, and over 8 bits where requests have more than 16 score rows on average, one (2^-8); out is rounded once.
 * fp32: products and sums in fp32; over caches of bf16 and 8 bits, which are exact in bf16, as bf16 products of queries and weights that are the sums of
 * three bf16 (2^-24; parts below 2^-126 count as 0).
 * Weights are up to 2^8 before they are divided by their sum: sums over numbers of V beyond 2^88 may overflow.  A score of -infinity, from an infinity in q
 * or in K, has the weight 0, and visible scores that are all -infinity give 0 and an lse of -infinity; one of +infinity or NaN makes NaN of its token.  An infinity
 * in V that is seen with a weight so small that fp32 has 0 for it may give a NaN.
 */
size_t laq_cache_attention_workspace_bytes(const laq_cache *cache, int32_t Hq, int32_t dtype, int32_t n, int64_t n_tokens, int32_t max_rows);
int laq_cache_attention(const laq_cache *cache, int32_t dtype, float scale, int32_t n, int64_t n_tokens, const int32_t *start, const laq_heads *q,
                        const int32_t *block_table, int32_t blocks_per_inst, const int32_t *rows, int32_t max_rows, void *out, float *lse,
                        void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LAQ_CACHE_H */
