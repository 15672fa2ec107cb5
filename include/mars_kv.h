/*
 * mars_kv.h -- the paged 4-bit KV cache around a verification step of libmars.
 *
 * The paper's decode cycle runs the target model once over all draft positions and afterwards keeps
 * the accepted path and drops the rest (Sec. 2.2; Algorithm 1 returns the accepted tokens, "rollback"
 * of the rest).  The calls here are the cache side of that cycle:
 *
 *   mars_kv_resize       room for the next tree's nodes (and trimming, and releasing sequences)
 *   mars_kv_append       K and V rows of the draft nodes (or of a prompt) into the pages
 *   mars_tree_attention  attention of the draft nodes over the cached tokens and their own ancestors
 *   (LM head + mars_verify_tree / _lmhead_verify -> accept_len, path_nodes)
 *   mars_kv_commit       the accepted path's rows move up behind the committed ones
 *   mars_kv_fork         one sequence continued several ways, full pages shared
 *   mars_kv_gather       rows of the cache as 16- or 32-bit values
 *
 * The conventions of mars.h hold: device pointers owned by the caller, nothing allocated, nothing
 * synchronised, work enqueued on `cuda_stream`; host-detectable errors are returned and nothing is
 * launched then; problems that only the data shows are reported per sequence.  A call reads and
 * writes nothing before its predecessor on the stream has completed.
 *
 * Format.  16 consecutive tokens of one KV head form a block of 18*d bytes: K codes [16][d/2],
 * V codes [16][d/2], K scales [16][d/16], V scales [16][d/16].  A code is a 4-bit E2M1 number (sign,
 * two exponent bits, one mantissa bit: 0 .5 1 1.5 2 3 4 6); the low nibble of a byte is the even
 * element.  A scale is one E4M3 byte for 16 neighbouring elements of a row.  A page of page_size
 * tokens is page_size/16 blocks; the pool is [layers][num_pages][kv_heads][page].  Stored value =
 * code * scale * scales[layer][0 = K, 1 = V][head]; 4.5 bits each.  Slots behind the written tokens
 * may hold anything.
 *
 * Sequences.  Sequence b's token at position p lies in page block_table[b][p / page_size], slot
 * p % page_size.  seq_len[b] tokens are committed; the nodes of a draft tree (or the tokens of a
 * prompt) take the positions seq_len[b] + i until mars_kv_commit.  In calls with a batch, batch row b
 * is sequence b.  seq_len may be set by the program, but not back into a page that another sequence
 * holds too (count above 1): rows appended there would be the other's as well.
 *
 * Pages.  page_refs[p] counts the sequences that hold page p; bit p%32 of free_bits[p/32] is set iff
 * page p is free.  A new cache has all counts and tables at zero / -1 and all bits of existing pages
 * set.  These arrays are changed by mars_kv_resize and mars_kv_fork only.  New pages are the lowest
 * free ones in request order, so the result does not depend on the order in which threads run.
 * A page id outside the pool, which these calls never write, is never followed: rows behind it are
 * skipped (mars_kv_append, _commit, _gather), read as NaN (mars_tree_attention), refused
 * (mars_kv_fork) or dropped from the table without effect (mars_kv_resize).
 */
#ifndef MARS_KV_H_
#define MARS_KV_H_

#include "mars.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MARS_FP16 2 /* third value of the dtype arguments below; other entry points refuse it */

#define MARS_KV_MAX_SEQS 8192 /* cap on seqs of a cache and on the pairs of one fork */

/* per-sequence (per-pair for mars_kv_fork) status values, besides MARS_SEQ_OK and MARS_SEQ_BAD_TREE */
#define MARS_SEQ_NO_ROOM 5      /* the positions asked for lie behind the sequence's pages, or the
                                   pages do not fit its row of the table                           */
#define MARS_SEQ_OUT_OF_PAGES 7 /* not enough free pages; the sequence is as it was                */
#define MARS_SEQ_BAD_PATH 8     /* accept_len or path_nodes do not name a rising path inside the
                                   sequence's pages; nothing moved                                 */
#define MARS_SEQ_BAD_FORK 9     /* source or destination out of range or equal, destination not
                                   empty or named by an earlier pair, source's table inconsistent  */

/* A cache; lives in HOST memory, its pointers are device pointers. */
typedef struct {
    void *pages;          /* [layers][num_pages][kv_heads][page_size*head_dim*9/8 bytes], 16-byte aligned */
    const float *scales;  /* [layers][2][kv_heads], positive and finite: K scales, V scales        */
    int32_t *block_table; /* [seqs][table_width] page ids                                          */
    int32_t *seq_len;     /* [seqs] committed tokens                                               */
    int32_t *seq_pages;   /* [seqs] pages held: the first seq_pages[b] entries of the table row    */
    int32_t *page_refs;   /* [num_pages]                                                           */
    uint32_t *free_bits;  /* [(num_pages + 31) / 32]                                               */
    int layers, num_pages, kv_heads;
    int head_dim;         /* 64 or 128                                                             */
    int page_size;        /* 16, 32, 64 or 128 tokens                                              */
    int seqs;             /* <= MARS_KV_MAX_SEQS                                                   */
    int table_width;      /* table_width * page_size <= 2^30, seqs * table_width < 2^31            */
} mars_kv_cache_t;

/* Bytes of the page pool of a cache with these sizes; 0 for unsupported sizes.  Host, pure. */
size_t mars_kv_pool_bytes(int layers, int num_pages, int kv_heads, int head_dim, int page_size);

/*
 * Rows of K and V into the cache: row (b, i) goes to position seq_len[b] + i of sequence b.
 * Sixteen neighbouring values x share a scale: with a = max|x|, s = e4m3((a / 6) / g) and code =
 * e2m1(x / (s * g)), g the head's scale, each operation one fp32 IEEE operation, both conversions to
 * nearest even and saturating; NaN counts as 0; s * g = 0 gives zero codes.
 *   k, v       `dt` (MARS_BF16, MARS_FP32, MARS_FP16); row b*N + i, head h at k + (b*N + i)*k_row +
 *              h*k_head (elements), unit inner stride; rows and heads must start on 16-byte boundaries.
 *   N          at most 2^24.
 *   count      int32 [B], rows of sequence b that are taken (the first ones), or NULL: all N.
 *              Counts below 0 read as 0, above N as N.
 *   seq_status int32 [B] or NULL: MARS_SEQ_OK, or MARS_SEQ_NO_ROOM: nothing of that sequence written.
 */
mars_status_t mars_kv_append(const mars_kv_cache_t *cache, int layer, const void *k, int64_t k_row,
                             int64_t k_head, const void *v, int64_t v_row, int64_t v_head, int dt,
                             int B, int N, const int32_t *count, int32_t *seq_status,
                             void *cuda_stream);

/*
 * Attention of the nodes of draft trees (Sec. 2.3 of the paper: many prefixes verified in one pass)
 * over the cache: node i of sequence b, for every query head j, attends positions
 * 0 .. seq_len[b]-1 and, behind them, the positions seq_len[b] + m of its ancestors m and of itself:
 * O = softmax(scale * q K^T) V, K and V of head j / (q_heads / kv_heads).  The nodes' own rows must
 * be in the cache (mars_kv_append).  A single new token is a chain with N = 1, a prompt a chain.
 *   q, out     `dt` (MARS_BF16 or MARS_FP16); row b*N + i, head j at q + (b*N + i)*q_row + j*q_head
 *              (elements), unit inner stride, rows and heads on 16-byte boundaries; out may not
 *              overlap q or the cache.
 *   parent     int32 [B, N] ([N] with MARS_SHARED_PARENT) as for mars_verify_tree, N <=
 *              MARS_MAX_NODES; or NULL: chains (parent[i] = i - 1), any N.
 *   count      int32 [B] or NULL, as for mars_kv_append.
 *   flags      MARS_SHARED_PARENT; MARS_COUNTERS_ZERO: the caller vouches that `workspace` was zeroed
 *              once and used by completed calls of this function only since; otherwise the call
 *              clears its counters (one stream operation more).
 *   seq_status int32 [B] or NULL: MARS_SEQ_OK, MARS_SEQ_NO_ROOM (no row written), MARS_SEQ_BAD_TREE
 *              (only the root's row is computed).  MARS_SEQ_TIMEOUT: a bounded wait inside the kernel
 *              gave up (a second without progress); rows of that sequence that were not computed are
 *              NaN.  The other sequences' rows and the workspace are sound.  With more than
 *              32 query rows per KV head it costs one stream operation (the statuses begin as OK).
 *   Rows i >= count[b] and rows of absent nodes (parent -1, i > 0, and what hangs below them) stay as
 *   they were; the slots of such nodes in the cache need not have been written.
 *   Scores, maxima, sums and the output are accumulated in fp32; products run on the tensor cores
 *   with K, V and q exact in fp16 (q scaled by a power of two per row) and the probabilities rounded
 *   to fp16.  Results do not vary from run to run.
 *   workspace  mars_tree_attention_workspace_bytes() bytes (never less for a larger N, whatever B),
 *              256-byte aligned; two calls that may overlap on the GPU need separate workspaces.
 */
size_t mars_tree_attention_workspace_bytes(int B, int N, int q_heads, int kv_heads, int head_dim);
mars_status_t mars_tree_attention(const mars_kv_cache_t *cache, int layer, const void *q, int64_t q_row,
                                  int64_t q_head, int dt, int q_heads, int B, int N,
                                  const int32_t *parent, const int32_t *count, float scale,
                                  uint32_t flags, void *out, int64_t out_row, int64_t out_head,
                                  int32_t *seq_status, void *workspace, size_t workspace_bytes,
                                  void *cuda_stream);

/*
 * After a verification: of the draft nodes at positions seq_len[b] + i the rows of the accepted path
 * move, in every layer, to seq_len[b], seq_len[b] + 1, ..., and the sequence grows by them.
 *   path_nodes int32 [B, path_width], root first, as mars_verify_tree writes it (path_width = Dcap+1),
 *              rising; or NULL: the path is 0, 1, 2, ... (chains) and nothing has to move.
 *   accept_len int32 [B]: a drafts accepted, so a + 1 rows stay (root and drafts); -1: none.
 *   new_len    int32 [B], receives seq_len[b] + a + 1; may be cache->seq_len itself.
 *   seq_status int32 [B] or NULL: MARS_SEQ_OK or MARS_SEQ_BAD_PATH (nothing moved, length unchanged).
 */
mars_status_t mars_kv_commit(const mars_kv_cache_t *cache, const int32_t *path_nodes, int path_width,
                             const int32_t *accept_len, int B, int32_t *new_len, int32_t *seq_status,
                             void *cuda_stream);

/*
 * Sequence dst[p] becomes a copy of sequence src[p], for every pair p: full pages are shared (their
 * counts rise), the rows of a last page that is not full are copied to a new page in every layer, so
 * that both may be continued.  dst must hold no pages.  Sources are read as they stood before the call.
 *   status     int32 [pairs], required: MARS_SEQ_OK, MARS_SEQ_OUT_OF_PAGES or MARS_SEQ_BAD_FORK; a pair
 *              that is not OK changes nothing.
 */
mars_status_t mars_kv_fork(const mars_kv_cache_t *cache, const int32_t *src, const int32_t *dst, int pairs,
                           int32_t *status, void *cuda_stream);

/*
 * Pages of every sequence b of the cache for seq_len[b] + extra[b] tokens: missing pages are added,
 * surplus ones given back (their table entries become -1).  extra[b] = 0 trims to the committed
 * tokens, -1 releases the sequence (length 0, no pages), anything below leaves it as it is.
 * All pages given back in the call are free before the first is taken; requests are served in order
 * of b until one does not fit, and from that one on every growing request gets MARS_SEQ_OUT_OF_PAGES.
 *   extra      int32 [seqs].
 *   seq_status int32 [seqs] or NULL: MARS_SEQ_OK, MARS_SEQ_OUT_OF_PAGES or MARS_SEQ_NO_ROOM (more
 *              pages than the table row holds); the sequence is as it was then.
 */
mars_status_t mars_kv_resize(const mars_kv_cache_t *cache, const int32_t *extra, int32_t *seq_status,
                             void *cuda_stream);

/*
 * Rows of the cache as values: for layers layer0 .. layer0+layers-1 and sequences b < B, positions
 * start[b] .. start[b] + count[b] - 1 to rows 0 .. of k_out and v_out, [layers][B][rows][kv_heads]
 * [head_dim] contiguous on 16-byte boundaries, of `dt` (MARS_BF16, MARS_FP32, MARS_FP16), rounded once
 * (bf16 results below 2^-126 after a rounding to fp32); `rows` is at most 2^24.  Rows from count[b]
 * on, and positions that lie outside the sequence's pages, stay as they were.
 *   start      int32 [B] or NULL: 0.      count  int32 [B] or NULL: all `rows`.
 */
mars_status_t mars_kv_gather(const mars_kv_cache_t *cache, int layer0, int layers, int B,
                             const int32_t *start, const int32_t *count, int rows, void *k_out,
                             void *v_out, int dt, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* MARS_KV_H_ */
