/*
 * prefixshield_kv.h -- C ABI of the operators on the KV pages whose block ids
 * the prefix-cache step (prefixshield.h) hands out.
 *
 * A pool holds the keys and values of num_pages pages of page_size tokens, for
 * num_layers layers.  Page ids below first_page belong to the prefix cache (the
 * block ids of ps_step()); the ids from first_page on are private pages of
 * running requests, counted by a reference array (ps_kv_fork() and the calls
 * after it).  Nothing holds the prefix cache's pages for a running request:
 * ps_step() keeps the blocks of its own batch only, and a later step may evict
 * one that a row's table still names (it lists them in evicted_ids and
 * invalidated_ids) and give it to another prompt, whose ps_kv_append() then
 * writes over it.  So either no step runs while rows name cached pages, or,
 * after the step and before its appends, each listed page that a row names is
 * copied to a private page (ps_kv_copy()) that takes its place in the table.
 * The operators:
 *   ps_step_blocks   the block ids of every request of the last ps_step();
 *   ps_kv_append     norm of queries and keys for each head, position
 *                    rotation, write of keys and values into their pages;
 *   ps_kv_plan, ps_kv_attention
 *                    attention over the pages of a batch of requests, a prefix
 *                    shared by a group of requests read once for all of them;
 *   ps_kv_copy, ps_kv_fork, ps_kv_release, ps_kv_compact
 *                    page copies, forks of sequences, freeing, compaction.
 *
 * Conventions are prefixshield.h's: d_* pointers (and every pointer inside the
 * argument structures) are device pointers, streams are void* holding a
 * cudaStream_t, every buffer is the caller's, nothing is allocated on the
 * device, every call is enqueued and returns an int32 status (PS_OK or
 * PS_ERR_*) without synchronizing.  What the host can see wrong is refused
 * before any work is enqueued.  What only the device can see wrong (an id or
 * an offset out of range) is never followed: it is reported in the call's
 * d_status, a device int32 that the caller zeroes beforehand and that the
 * calls only ever set to an error, so that one word can watch a whole step
 * (NULL: not reported).  A handle is not thread-safe; calls on one handle must
 * be issued in order on one stream (or with equivalent ordering).
 */
#ifndef PREFIXSHIELD_KV_H
#define PREFIXSHIELD_KV_H

#include "prefixshield.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of a pool (and of the queries and outputs that go with it). */
typedef enum { PS_KV_BF16 = 0, PS_KV_F16 = 1 } ps_kv_dtype_t;

#define PS_KV_MAX_HEAD_DIM 128
#define PS_KV_MAX_HEADS 1024      /* query heads */

/* The pool and the bounds of later calls.  Element (layer, page, t, head, e)
 * of K is k[layer * layer_stride + page * page_stride + t * token_stride +
 * head * head_stride + e], and V likewise: token-major and head-major pages,
 * keys and values in one tensor or in two.  K and V start on 16-byte
 * boundaries, strides are non-negative multiples of 8 elements, and distinct
 * elements have distinct addresses. */
typedef struct {
  void* k;
  void* v;
  int64_t num_pages;      /* page ids are [0, num_pages), at most 2^30 */
  int64_t first_page;     /* first private page; from num_pages on: there are none */
  int64_t layer_stride, page_stride, token_stride, head_stride; /* in elements */
  int32_t num_layers;
  int32_t page_size;      /* tokens: 2, 4, 8, 16, 32 or 64, as ps_create()'s block_size */
  int32_t num_kv_heads;
  int32_t num_q_heads;    /* a multiple of num_kv_heads: query head h reads kv head h / (num_q_heads / num_kv_heads) */
  int32_t head_dim;       /* a multiple of 8, 8..PS_KV_MAX_HEAD_DIM */
  int32_t dtype;          /* ps_kv_dtype_t */
  int32_t max_requests;   /* rows of a batch, and items of one page call: 1..2^18 - 1 */
  int32_t max_tokens;     /* query tokens of a batch, 1..2^22, and max_tokens * num_q_heads < 2^30 */
  int32_t max_row_pages;  /* pages of one request: max_row_pages * page_size < 2^30 */
  int32_t pad0;
} ps_kv_config_t;

typedef struct ps_kv ps_kv_t;

/* Bytes of device workspace a handle needs (256-byte aligned base required),
 * or 0 if the configuration is invalid.  It holds the page calls' scratch, a
 * batch's plan and the partial results of splits and shared prefixes: 1 MB for
 * each element of a head, and more with max_tokens and max_requests (402 MB in
 * all for 256 requests of 4096 tokens with 32 query heads of 128 on 8). */
size_t ps_kv_workspace_bytes(const ps_kv_config_t* cfg);

/* Create a handle on the current device; clearing a few counters of the
 * workspace is enqueued on 'stream'.  The workspace must stay allocated and
 * untouched until ps_kv_destroy(). */
int32_t ps_kv_create(ps_kv_t** out, const ps_kv_config_t* cfg, void* d_workspace, size_t workspace_bytes,
                     void* stream);

/* Free the host-side handle.  The workspace is the caller's to free. */
void ps_kv_destroy(ps_kv_t* kv);

/* The block ids of every request of the last ps_step() of h: request i's
 * leading blocks resident after the step (its cached prefix, its in-step hits
 * and its own admitted blocks, up to the first block the pool could not hold)
 * go to d_tables[i * table_stride ...] in position order, at most table_stride
 * of them, and their number to d_counts[i].  d_group_ids: that step's;
 * num_requests: its number of requests, or fewer (the leading ones).
 * Must follow the step, in stream order, before any other call on h (they
 * share scratch): refused before the first step, for more requests than the
 * last one had, and after ps_cached_prefix() or ps_reset().  After a step that
 * failed, every count is 0.  *d_status: an error if the step failed or a row was
 * cut at table_stride. */
int32_t ps_step_blocks(ps_handle_t* h, void* stream, int32_t num_requests, const int32_t* d_group_ids,
                       int32_t* d_tables, int64_t table_stride, int32_t* d_counts, int32_t* d_status);

/* One layer's new tokens.  For each head x of a token's queries and keys:
 *   x <- x * w / sqrt(mean(x^2) + eps)              if the weight w is given,
 *   (a, b) <- (a cos - b sin, b cos + a sin)        for each rotated pair,
 * in 32 bits, rounded once; queries go to q_out, keys and values to the pool.
 * Head h, element e of token t's queries is q[t * q_stride[0] + h *
 * q_stride[1] + e], and so on; inputs and q_out start on 16-byte boundaries
 * with strides that are multiples of 8 elements.  q_out may be q itself; else
 * it lies on none of q, k and v (refused). */
typedef struct {
  const void* q;
  const void* k;
  const void* v;
  void* q_out;
  int64_t q_stride[2], k_stride[2], v_stride[2], q_out_stride[2]; /* token, head; in elements */
  const int64_t* slots;      /* [T] page * page_size + offset, distinct; negative: the token's K and V are not written */
  const int32_t* positions;  /* [T] row of the rotation table (NULL without one) */
  const float* rope;         /* [rope_rows][rope_dim]: rope_dim / 2 cosines, then the sines; NULL: no rotation */
  const void* q_weight;      /* [head_dim], the pool's type; NULL: no norm of the queries */
  const void* k_weight;      /* [head_dim]; NULL: no norm of the keys */
  float eps;                 /* > 0 */
  int32_t num_tokens;        /* T, 0..2^30 */
  int32_t rope_rows;
  int32_t rope_dim;          /* rotated leading elements of a head: a multiple of 8, at most head_dim */
  int32_t rope_interleaved;  /* pairs (2i, 2i + 1) instead of (i, i + rope_dim / 2) */
  int32_t fill;              /* nonzero: q_out of a token that is left out becomes NaN (for memory that nothing wrote before) */
} ps_kv_append_t;

/* Append to layer 'layer'.  A token whose slot is past the pool or whose
 * position is outside the table is left out (its q_out, but for 'fill', K and V
 * stay as they were) and *d_status becomes PS_ERR_INVALID_ARG. */
int32_t ps_kv_append(ps_kv_t* kv, void* stream, int32_t layer, const ps_kv_append_t* a, int32_t* d_status);

/* A batch of requests.  Request i's queries are the rows [q_offsets[i],
 * q_offsets[i+1]) of a token array (offsets start at 0, do not decrease, and
 * end at num_tokens; a request may have none); they are the last of its
 * kv_lens[i] tokens, whose keys and values lie in the pages tables[i *
 * table_stride ...].  Causal: token j of the n new ones sees the keys before
 * position kv_len - n + j + 1; else every query sees all kv_len keys.  A query
 * that sees no key gives 0 (and -infinity in lse).  What a query does not see
 * does not reach it, infinities and NaN included.
 * group_offsets (NULL: no sharing) divides the requests into num_groups runs
 * [group_offsets[g], group_offsets[g+1]) of neighbours that may share a
 * prefix: how many leading pages all of them have in common is found from the
 * tables, so a grouping never changes a result, only what is read twice. */
typedef struct {
  const int32_t* q_offsets;     /* [num_requests + 1] */
  const int32_t* kv_lens;       /* [num_requests] */
  const int32_t* tables;        /* page ids */
  const int32_t* group_offsets; /* [num_groups + 1] or NULL */
  int64_t table_stride;         /* elements between rows; a row holds min(table_stride, max_row_pages) ids */
  int32_t num_requests;
  int32_t num_groups;           /* 1..num_requests; not looked at in a batch of no requests */
  int32_t num_tokens;
  int32_t causal;
} ps_kv_batch_t;

/* Divide a batch's attention over the GPU: finds the shared prefixes and cuts
 * the work into equal parts.  One plan serves every layer of a step; the
 * batch's arrays must stay unchanged until the last ps_kv_attention() of the
 * plan has run.  Bad offsets, lengths or page ids make *d_status
 * PS_ERR_INVALID_ARG and the plan empty: attention on it writes nothing (but for 'fill').  Until
 * the first plan has run (a captured one runs when its graph does) it is empty, too. */
int32_t ps_kv_plan(ps_kv_t* kv, void* stream, const ps_kv_batch_t* batch, int32_t* d_status);

/* softmax(scale q k^T) v of one layer for the planned batch, softmax and sums
 * in 32 bits.  q and out: element (t, h, e) at t * stride[0] + h * stride[1] +
 * e, on 16-byte boundaries with strides that are multiples of 8 elements; out
 * does not overlap q (refused).  lse (NULL: none): float [num_tokens][num_q_heads], log of the sum of the
 * exponentials of a query's scaled scores.  Results do not depend on timing:
 * the same call gives the same bits.  *d_status: PS_ERR_TIMEOUT if a wait inside
 * the kernel ran out (never expected). */
typedef struct {
  const void* q;
  void* out;
  float* lse;
  int64_t q_stride[2], out_stride[2]; /* token, head; in elements */
  float scale;
  int32_t fill; /* nonzero: after an empty plan out becomes NaN (for memory that nothing wrote before) */
} ps_kv_attention_t;
int32_t ps_kv_attention(ps_kv_t* kv, void* stream, int32_t layer, const ps_kv_attention_t* a, int32_t* d_status);

/* Copy whole pages, all layers: page d_dst[i] becomes a copy of page d_src[i].
 * The destinations are distinct and none is a source.  An id out of range
 * drops its pair and sets *d_status. */
int32_t ps_kv_copy(ps_kv_t* kv, void* stream, int32_t n, const int32_t* d_src, const int32_t* d_dst, int32_t* d_status);

/* The sequences of the page calls: row r holds held[r] pages, ids
 * tables[r * table_stride ...], with lens[r] tokens written.  refs[id -
 * first_page] counts the rows that hold a private page; 0 means free.
 * Where a pool has no private pages the references may be NULL.
 * num_rows may exceed max_requests. */
typedef struct {
  int32_t* tables;
  int32_t* lens;
  int32_t* held;
  int64_t table_stride;
  int32_t num_rows;
  int32_t pad0;
} ps_kv_rows_t;

/* For each item i, row children[i] becomes a continuation of row parents[i]
 * (its lens[parent] tokens) with pages for room[i] tokens in all:
 *  - parent == child: the row grows in place;
 *  - parent == -1: a new row of no tokens;
 *  - else a fork: the parent's full pages are shared, its partly filled page's
 *    tokens are copied (all layers) to a page of the child's own.
 * New pages are the free private pages of the lowest ids, in item order.  The
 * child's former row is forgotten (release it first).  No child is another
 * item's child or parent.  All or nothing: an item out of range sets *d_status
 * to PS_ERR_INVALID_ARG, too few free pages to PS_ERR_CAPACITY, and then
 * nothing changes but refs_out, which becomes refs_in.  refs_out may be
 * refs_in, but not overlap it otherwise (refused).  n is at most max_requests. */
int32_t ps_kv_fork(ps_kv_t* kv, void* stream, int32_t n, const int32_t* d_parents, const int32_t* d_children,
                   const int32_t* d_room, const ps_kv_rows_t* rows, const int32_t* d_refs_in, int32_t* d_refs_out,
                   int32_t* d_status);

/* Free the rows d_rows[i] (distinct): each private page they hold loses one
 * reference, their lens and held become 0.  A row out of range, a page id out
 * of range or a reference below zero is left out and sets *d_status. */
int32_t ps_kv_release(ps_kv_t* kv, void* stream, int32_t n, const int32_t* d_rows, const ps_kv_rows_t* rows,
                      int32_t* d_refs, int32_t* d_status);

/* Move the private pages in use to the lowest private ids: with L of them, the
 * lowest free page below first_page + L takes over the highest page in use at
 * or above it, and so on.  Their keys and values are copied (all layers), the
 * tables (all num_rows rows' held pages) are written to d_tables_out with the
 * new ids (entries past held are copied as they are), and the references to
 * d_refs_out; both may be the inputs themselves, but not overlap them otherwise
 * (refused).  d_counts [2]: L, and the pages moved.  Rows may be wider than
 * max_row_pages.  Held ids out of range are copied as they are and set
 * *d_status; a row with fewer than 0 or more than table_stride pages sets it,
 * too, and has none or all of its ids rewritten. */
int32_t ps_kv_compact(ps_kv_t* kv, void* stream, const ps_kv_rows_t* rows, const int32_t* d_refs_in,
                      int32_t* d_tables_out, int32_t* d_refs_out, int32_t* d_counts, int32_t* d_status);

#ifdef __cplusplus
}
#endif

#endif /* PREFIXSHIELD_KV_H */
