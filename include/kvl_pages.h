/*
 * kvl_pages -- whose the blocks of a paged cache are, and copies of blocks.
 *
 *   kvl_pages          host: sequences of tokens and their block tables; blocks are shared where sequences
 *                      were forked, taken and given back as they grow, shrink and end
 *   kvl_page_pools     once: the planes of all layers of a pool
 *   kvl_copy_blocks    device: blocks of all layers to other blocks of the same pool, one launch
 *
 * A sequence has a number of tokens and a table of ceil(tokens / block_tokens) blocks, of which kvl_plan and
 * kvl_attn_plan take the table as it is.  A block is free, or in use by one sequence or more; the free block of the lowest number is
 * taken first.  A block that several sequences use is not written to: kvl_pages_extend gives a sequence whose last block is shared and not
 * full a block of its own, and says which copy has to be made before the new tokens are written (kvl_copy_blocks, on the stream of the
 * kvl_append_layer that follows).
 *
 * Conventions are those of kvl.h.  The host functions touch no device and change nothing unless they return 0; a kvl_pages_t
 * may be used by one thread at a time.  Sequences are named by numbers that are not used again; one that is not there is KVL_EINVAL, and so
 * is one that a list of kvl_pages_extend, kvl_pages_truncate or kvl_pages_free names twice.
 */
#ifndef KVL_PAGES_H
#define KVL_PAGES_H

#include "kvl.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct kvl_pages_s kvl_pages_t;             /* opaque, library-owned */
typedef struct kvl_page_pools_s kvl_page_pools_t;   /* likewise */

/* One copy of a block. */
typedef struct {
    int32_t from;
    int32_t to;
} kvl_block_copy_t;

/* All blocks free.  KVL_ERANGE: more than 2^31 - 1 blocks. */
int kvl_pages(uint32_t block_tokens, uint64_t pool_blocks, kvl_pages_t **out);
void kvl_pages_destroy(kvl_pages_t *pages);

/* New sequences of hit + append tokens each, out of tables that are there already (made by another allocator, or of a cache that was
 * loaded); with no tokens, an empty one.  Tables may share blocks with each other and with sequences that are there.  sequences: host
 * array of n_req, gets their numbers.  KVL_ERANGE: a table too short, a block outside the pool, 2^31 tokens or more; KVL_EALIAS: a table names a block twice. */
int kvl_pages_adopt(kvl_pages_t *pages, const kvl_request_t *requests, uint32_t n_req, uint64_t *sequences);
/* New sequences that are what others are now (one may be named several times): all blocks are shared. */
int kvl_pages_fork(kvl_pages_t *pages, const uint64_t *sequences, uint32_t n, uint64_t *forks);
/* Sequences grow by tokens[i] each, one after the other.  copies: host array of n; *n_copies gets how many there are.  A sequence's copy is of its last
 * block as it was (which others keep) to the one that it has now.  KVL_ESPACE: too few free blocks; KVL_ERANGE: a sequence of 2^31 tokens or more. */
int kvl_pages_extend(kvl_pages_t *pages, const uint64_t *sequences, const uint32_t *tokens, uint32_t n, kvl_block_copy_t *copies,
                     uint32_t *n_copies);
/* Sequences keep their first tokens[i] tokens (KVL_ERANGE: they have fewer), and the blocks of these. */
int kvl_pages_truncate(kvl_pages_t *pages, const uint64_t *sequences, const uint32_t *tokens, uint32_t n);
/* Sequences end. */
int kvl_pages_free(kvl_pages_t *pages, const uint64_t *sequences, uint32_t n);
/* Blocks in use move to the front of the pool: the last one in use to the first free one, until `most` have moved or no free block lies
 * before one in use.  All tables follow.  It looks at all blocks beyond as many as are in use, and at all tables, whatever `most` is.  copies: host array of `most`; *n_copies: how many have moved.  No copy's source is another's destination; the copies have to be made
 * before anything else is written to the pool's blocks. */
int kvl_pages_compact(kvl_pages_t *pages, uint32_t most, kvl_block_copy_t *copies, uint32_t *n_copies);

/* Tables of sequences, one after the other: first[i] (host array of n + 1) gets where sequence i's begins, first[n] the length of all;
 * table: host array of `capacity` entries (KVL_ESPACE: too few; first[] is filled all the same), NULL with 0. */
int kvl_pages_tables(const kvl_pages_t *pages, const uint64_t *sequences, uint32_t n, int32_t *table, uint64_t capacity, uint64_t *first);
int kvl_pages_tokens(const kvl_pages_t *pages, const uint64_t *sequences, uint32_t n, uint32_t *tokens);
typedef struct {
    uint64_t free_blocks;
    uint64_t used_blocks;
    uint64_t shared_blocks;     /* used by more than one sequence */
    uint64_t moves;             /* that kvl_pages_compact would make */
    uint64_t sequences;
} kvl_pages_stats_t;
int kvl_pages_stats(const kvl_pages_t *pages, kvl_pages_stats_t *out);

/* The planes of a pool that copies go through: a block of plane p has block_bytes[p] bytes in each layer (two of kvl_attn.h's 8-bit cache are
 * block_tokens * kv_heads * head_dim codes, two are 4 * kv_heads bytes of scales), block b at b * block_bytes[p].
 * planes: host array [n_layers][n_planes] of device pointers, borrowed for the call; the memory has to stay.
 * flags: KVL_NO_POINTER_CHECKS, KVL_CALLER_SYNCS, as in kvl_plan.  KVL_ERANGE: more than 2^31 - 1 blocks, or a block of a plane of more than 2^32 bytes. */
typedef struct {
    uint32_t n_layers;                      /* up to 4096 */
    uint32_t n_planes;                      /* up to KVL_MAX_PLANES */
    uint64_t block_bytes[KVL_MAX_PLANES];
    uint64_t pool_blocks;
} kvl_page_layout_t;
int kvl_page_pools(const kvl_page_layout_t *layout, void *const *planes, uint32_t flags, kvl_page_pools_t **out);
/* As kvl_plan_destroy: does not wait for the device. */
void kvl_page_pools_destroy(kvl_page_pools_t *pools);
/* Copy blocks of every layer and plane (copies: host array, borrowed for the call).  KVL_ERANGE: a block outside the pool, or more than a launch holds: 2^32 lanes
 * or more for one copy, where a plane of a layer takes a lane for each 16 bytes of a block (4 where its size, or where it begins in some layer, is a multiple
 * of 4 and not of 16; 1 where it is of neither) and 256 more.  So up to nearly 2^36 bytes a copy (2^34, 2^32) are taken.  KVL_EALIAS: a block is the destination of two copies, or
 * of one and the source of one.  Takes no device memory, and can be captured into a HIP graph, which then repeats these copies. */
int kvl_copy_blocks(const kvl_page_pools_t *pools, const kvl_block_copy_t *copies, uint64_t n, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* KVL_PAGES_H */
