/*
 * kvl_attn -- what a model does with one layer of a loaded cache: write the new
 * tokens' keys and values into it, rotated by their positions, and attend to it.
 *
 *   kvl_attn_plan     host: from the batch that kvl_plan takes (hit prefix,
 *                     appended tail, block table of each request) to the lists
 *                     of work of both calls below; once per batch, for all layers
 *   kvl_append_layer  the appended tokens' keys and values into one layer's pool
 *   kvl_attn_layer    attention of the appended tokens' queries over that pool
 *
 * They fit between the load of a layer and the way out of it: the computation that
 * kvl_stream_layers calls for each layer can make these two calls on its stream.
 *
 * New tokens.  Request r has hit_r cached tokens and append_r new ones; new token i
 * of it is at position hit_r + i.  Queries, new keys, new values and outputs hold the
 * new tokens of all requests, request after request: token-major
 * [tokens][heads][head_dim], the heads of a token dense, tokens at a stride.
 *
 * Pool (one layer): planes K and V, bytes [pool_blocks][block_tokens][kv_heads][head_dim]
 * of cache_dtype: two of kvl.h's planes with rows of kv_heads * head_dim elements, so
 * kvl_plan and its calls move them.  With cache_dtype KVL_E4M3 two more planes follow,
 * the scales of K and of V: float [pool_blocks][kv_heads].  A code c in block b of head h
 * stands for c * scale[b][h].  (A kvl_plan of block_tokens 1 and rows of 4 * kv_heads
 * bytes, with the number of a request's blocks as its hit tokens, moves those.)
 *
 * Conventions (errors, streams, ownership, devices) are those of kvl.h.  Both calls only
 * enqueue work; they can be captured into a HIP graph.
 */
#ifndef KVL_ATTN_H
#define KVL_ATTN_H

#include "kvl.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define KVL_BF16 1u
#define KVL_F16  2u
#define KVL_E4M3 3u   /* 8 bits: 4 of exponent, 3 of mantissa, no infinities, largest 448 */

/* which elements of a head the rotation takes together */
#define KVL_ROPE_HALVES     0u   /* (j, j + rope_dim/2) */
#define KVL_ROPE_NEIGHBOURS 1u   /* (2j, 2j + 1) */

typedef struct kvl_attn_plan_s kvl_attn_plan_t;   /* opaque, library-owned */

typedef struct {
    uint32_t block_tokens;
    uint32_t q_heads;       /* a multiple of kv_heads: query head H reads head H / (q_heads / kv_heads) */
    uint32_t kv_heads;
    uint32_t head_dim;      /* 64 or 128 */
    uint32_t dtype;         /* KVL_BF16 or KVL_F16: queries, new keys and values, outputs */
    uint32_t cache_dtype;   /* dtype, or KVL_E4M3 */
    uint32_t window;        /* 0: none; else a query at position p sees the keys p - window < t */
    uint32_t sinks;         /* first tokens that stay visible outside the window */
    uint32_t rope_dim;      /* leading elements of each head that kvl_append_layer rotates: a multiple of 16, 0: none */
    uint32_t rope_pairs;    /* KVL_ROPE_* */
    uint64_t pool_blocks;
} kvl_attn_layout_t;

/* Build a plan.  flags: KVL_SCATTER (the plan may be used with kvl_append_layer) and / or
 * KVL_GATHER (with kvl_attn_layer); which keys attention sees, as kvl_plan's rows: by default
 * the hit prefix alone (what can be done before the new keys are there), KVL_TOKENS_APPEND the
 * appended tail, KVL_TOKENS_ALL both; KVL_HOST_ONLY, KVL_NO_POINTER_CHECKS and KVL_CALLER_SYNCS
 * as in kvl_plan.  KVL_ERANGE: a block id outside the pool, a table too short, a request of 2^31
 * tokens or more, 2^32 pool rows or new tokens or more, more work than a launch holds (2^24 pieces of attention
 * work times cache heads, or as many workgroups that join them; with KVL_SCATTER and an 8-bit cache more than 2^23 blocks that
 * receive new tokens times cache heads, or new tokens beyond a block's row 2^28); KVL_EALIAS: with KVL_SCATTER, a block
 * that receives new tokens is named twice by the tables' receiving parts (requests may share the
 * blocks that they only read). */
int kvl_attn_plan(const kvl_attn_layout_t *layout, const kvl_request_t *requests, uint32_t n_req,
                  uint32_t flags, kvl_attn_plan_t **out);
/* As kvl_plan_destroy: does not wait for the device. */
void kvl_attn_plan_destroy(kvl_attn_plan_t *plan);
int kvl_attn_plan_tokens(const kvl_attn_plan_t *plan, uint64_t *new_tokens);
/* Device memory that kvl_attn_layer wants to join what different workgroups found for one query (may be 0). */
int kvl_attn_plan_workspace(const kvl_attn_plan_t *plan, uint64_t *bytes);

/* One piece of attention work, for every head of the cache: n_rows rows of queries (row i of a
 * request is new token i / group, head i % group of the query heads that share a cache head) over the
 * keys at places [begin, end) of the row of the visible ones, in which place v is token
 * v < sinks ? v : v + gap. */
typedef struct {
    uint32_t request;
    uint32_t first_row;
    uint32_t n_rows;
    uint32_t begin;
    uint32_t end;
    uint32_t sinks;
    uint32_t gap;
    uint32_t pieces;     /* that the keys of these rows are cut into */
} kvl_attn_item_t;
/* Copy up to capacity items into out (host array); *n_items gets the total.  Host side only. */
int kvl_attn_plan_items(const kvl_attn_plan_t *plan, kvl_attn_item_t *out, uint64_t capacity, uint64_t *n_items);

/* New keys and values of one layer into its pool, keys rotated; queries rotated beside them.
 * rope: device, float [rope_positions][rope_dim / 2][2], cosine and sine of each position and pair
 * (position * frequency wants 64 bits where the table is made); rope_positions must be above every
 * position of the batch (KVL_ESPACE).  A pair (a, b) becomes (a cos - b sin, b cos + a sin); elements from
 * rope_dim on stay.  The rotation is computed in 32 bits and rounded once, for an 8-bit cache in 64.
 *
 * 8-bit cache: the scale of a block and head is the power of two 2^e with the least e in [-32, 63]
 * for which no finite new value of the block is above 448 * 2^e; in a block that already holds hit
 * tokens it is at least the scale that is there (taken as kvl_attn_layer takes it, from 2^-32 to 2^63, NaN as
 * 2^-32), and where it grows the codes that are there are rounded again to the new one.  (e4m3 floats: a power of two costs no precision, and the second rounding
 * loses only what falls below the least normal.)  Codes are rounded to the nearest, ties to even; what
 * is not finite becomes NaN, and what is above 448 * 2^63 becomes 448 * 2^63.
 *
 * Strides are in elements, 0: dense; multiples of 8, tokens apart; pointers 16-byte aligned (KVL_EINVAL).
 * q == NULL: no queries.  q_out may be q itself (with its stride); else inputs and outputs must not overlap.  Rows of the
 * pool that hold no new token keep their bytes (but for codes rounded again).  Needs a KVL_SCATTER plan. */
typedef struct {
    const void *k;
    const void *v;
    const void *q;
    void *q_out;
    uint64_t k_stride;
    uint64_t v_stride;
    uint64_t q_stride;
    uint64_t q_out_stride;
    const float *rope;
    uint64_t rope_positions;
} kvl_append_t;
int kvl_append_layer(const kvl_attn_plan_t *plan, const kvl_append_t *args, void *const *pool_planes, void *stream);

/* Attention of the new tokens over one layer's pool:
 *   out = sum_t softmax_t(scale * <q, K_t>) V_t  over the visible keys t: those of the plan's range with
 *   t <= p and (window == 0 or p - t < window or t < sinks), p the query's position.
 * A query that sees no key gets zeros (and lse -inf).  lse (optional, float [tokens][q_heads]): the natural
 * logarithm of the sum of the exponentials, by which results over different ranges can be joined.
 * Scores, sums and outputs are held in 32 bits, softmax weights are rounded to dtype (or finer) before they multiply values.
 * Over an 8-bit cache keys and values are c * scale exactly, but where scales are no powers of two and a request has more than
 * 64 rows of queries (new tokens times q_heads / kv_heads): there they may be rounded to dtype once.
 * Keys that a query does not see do not reach its result, whatever they hold.  scale must be finite and positive.
 * out may be q itself (with its stride); else out, lse and workspace must not overlap each other or what is read.
 * workspace: device memory of at least kvl_attn_plan_workspace bytes, 256-byte aligned, in nobody else's
 * use until the call's work is done.  With KVL_E4M3, scales are taken as at least 2^-32 and at most 2^63. */
typedef struct {
    const void *q;
    void *out;
    float *lse;
    uint64_t q_stride;
    uint64_t out_stride;
    void *workspace;
    uint64_t workspace_bytes;
    float scale;
} kvl_attn_t;
int kvl_attn_layer(const kvl_attn_plan_t *plan, const kvl_attn_t *args, const void *const *pool_planes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* KVL_ATTN_H */
