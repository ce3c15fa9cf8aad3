/*
 * unison_kv.h -- C ABI of the operators on the KV cache itself.
 *
 * include/unison.h decides which agent session's KV cache stays resident and
 * in which tier.  The entry points here are the serving step that reads and
 * shrinks that cache, on one paged cache of many sessions:
 *
 *   unison_kv_attend   attention of a tree of drafted tokens over the cache
 *   unison_kv_verify   verification of the drafts against the target's
 *                      probabilities, from given random numbers
 *   unison_kv_observe  the attention weight that each cached token gets from
 *                      the accepted tokens, added to its account
 *   unison_kv_commit   the accepted tokens' keys and values into the pages
 *   unison_kv_evict    the least attended tokens out of the cache, in place or
 *                      into another tier's cache
 *
 * Conventions (those of unison.h): every function returns an int status,
 * nothing aborts or throws; all pointers inside the structs are device
 * pointers owned by the caller, valid until the work queued on the stream has
 * finished; structs themselves are read during the call only; work is queued
 * on cuda_stream without any synchronisation, and may be captured into a
 * graph.  No device memory is allocated: calls that need scratch take a
 * workspace, which may hold anything before the call and is free for other use
 * by later work of the same stream.  Calls that overlap on the GPU need
 * workspaces of their own.  An empty batch (n_seqs = 0) does nothing.
 *
 * Values in device memory that are out of their documented range (a page id
 * outside the pool, a length beyond the page table, offsets that do not
 * ascend) are never followed: lengths and offsets are clamped, a slot without
 * a page counts as absent, and, where the cache has a status array, the
 * session's word receives UNISON_ERR_RANGE.  The calls never clear it.  Waits
 * inside the kernels are bounded; one that gives up (no input makes it) leaves
 * UNISON_ERR_TIMEOUT there, and that session's results are undefined.
 */
#ifndef UNISON_KV_H
#define UNISON_KV_H

#include <stdint.h>

#include "unison.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { UNISON_KV_BF16 = 0, UNISON_KV_FP16 = 1, UNISON_KV_FP32 = 2 };

#define UNISON_KV_MAX_TOKENS 64 /* new tokens of one session in one call */

/* The paged KV cache of n_seqs sessions (one layer).  Slot x of session b is
 * slot x % page_size of page page_table[b * max_pages + x / page_size]; slots
 * 0 .. length[b]-1 are in use.  Different sessions' pages are disjoint.  The
 * keys carry their rotation already, so the order of slots means nothing to
 * attention; pos keeps each slot's position in its session.
 * Strides are in elements, of the page, head and slot axes; the head_dim axis
 * is contiguous.  k and v start on 16-byte boundaries, their strides are
 * multiples of 8.  head_dim: a multiple of 8, 8 .. 256; n_heads: KV heads;
 * dtype: UNISON_KV_BF16 or _FP16; page_size >= 1; max_pages * page_size < 2^31 - 2^16.
 * A call that does not use an array takes NULL for it. */
typedef struct {
  void *k;
  void *v;
  float *mass;               /* [page, head, slot] accumulated attention weight  */
  int32_t *pos;              /* [page, head, slot] position in the session       */
  const int32_t *page_table; /* [n_seqs, max_pages]                              */
  int32_t *length;           /* [n_seqs] slots in use                            */
  int32_t *next_pos;         /* [n_seqs] position of the session's next token    */
  int32_t *status;           /* [n_seqs], or NULL                                */
  int64_t k_page, k_head, k_slot;
  int64_t v_page, v_head, v_slot;
  int64_t m_page, m_head, m_slot; /* of mass and of pos */
  int32_t n_seqs, max_pages, n_pages, page_size;
  int32_t n_heads, head_dim, dtype, reserved;
} unison_kv_cache;

/* The new tokens of a step: session b owns tokens offsets[b] .. offsets[b+1]-1
 * of the step's arrays, at most max_tokens (1 .. 64) of them.  Node 0 of a
 * session is its last sampled token, the root; the others are drafts.
 *   mask    bit j of mask[i]: node i sees node j of its session (normally
 *           itself and its ancestors).  NULL: a chain, bits 0 .. i.
 *   parent  node index of each node's parent, below the node's own (node 0:
 *           ignored; a node whose parent is not such an index is never
 *           reached).  Read by unison_kv_verify only. */
typedef struct {
  const int32_t *offsets; /* [n_seqs + 1] */
  const uint64_t *mask;   /* [n_tokens], or NULL */
  const int32_t *parent;  /* [n_tokens] */
  int32_t n_seqs, n_tokens, max_tokens, reserved;
} unison_kv_tree;

/* The step's arrays: row i is token i, strides in elements (multiples of 8),
 * 16-byte aligned, the type of the cache.  n_q_heads is a multiple of n_heads,
 * at most 64 times it; query head g belongs to KV head g / (n_q_heads /
 * n_heads).  A call reads those of the arrays that it names below. */
typedef struct {
  const void *q;     /* [n_tokens, n_q_heads, head_dim] */
  const void *k_new; /* [n_tokens, n_heads, head_dim]   */
  const void *v_new; /* [n_tokens, n_heads, head_dim]   */
  void *out;         /* [n_tokens, n_q_heads, head_dim] */
  float *lse;        /* [n_tokens, n_q_heads], dense    */
  float *mass_new;   /* [n_tokens, n_heads], dense      */
  int64_t q_token, q_head;
  int64_t k_token, k_head;
  int64_t v_token, v_head;
  int64_t out_token, out_head;
  int32_t n_q_heads;
  float scale; /* factor of every product q . k */
} unison_kv_step;

/* Accepted path of each session: node indices path[b][0 .. n_path[b]-1],
 * ascending, path_stride int32 from one session to the next.  path = NULL:
 * every node of the session. */
typedef struct {
  const int32_t *path;
  const int32_t *n_path; /* [n_seqs] */
  int64_t path_stride;
} unison_kv_path;

/* Attention of every new token over its session's cached tokens and the new
 * tokens that its mask names:
 *   S = scale q . k,  lse = ln sum exp S,  out = sum exp(S - lse) v.
 * A row that sees nothing gets out = 0 and lse = -inf.  What a mask hides does
 * not reach the result, NaN and infinities included.  Products are of the
 * type's values, sums in 32 bits; the weights exp(S - max) are rounded to the
 * type before they meet v (in FP16 multiplied by 2^7 or more before that, so
 * that 2^-31 still counts, unless scores are beyond 2^19).  Reads q, k_new,
 * v_new; writes out, lse (lse may be NULL).  Tokens outside every session's
 * range are not written.
 * The result does not depend on timing: the same call gives the same bits.
 * UNISON_ERR_ARG: null or misaligned arrays, sizes that do not fit together,
 * a workspace that is too small (or not 16-byte aligned); UNISON_ERR_RANGE:
 * limits above; UNISON_ERR_CUDA: the launch. */
uint64_t unison_kv_attend_workspace(const unison_kv_cache *cache, const unison_kv_tree *tree, int n_q_heads);
int unison_kv_attend(const unison_kv_cache *cache, const unison_kv_tree *tree, const unison_kv_step *step,
                     void *workspace, uint64_t workspace_bytes, void *cuda_stream);

/* Adds to cache->mass, for every cached token and KV head, the attention
 * weight sum exp(S - lse) that the accepted tokens give it, over the query
 * heads of that KV head; lse is what unison_kv_attend returned.  mass_new
 * receives the same of the new tokens themselves (0 for a node that no
 * accepted one sees).  Rows with lse = -inf give nothing, nor do nodes of the
 * path that the session has not (UNISON_ERR_RANGE).  Reads q, k_new, lse; writes
 * mass and mass_new (NULL: not wanted; k_new is not read then). */
int unison_kv_observe(const unison_kv_cache *cache, const unison_kv_tree *tree, const unison_kv_step *step,
                      const unison_kv_path *path, void *cuda_stream);

/* Appends the accepted tokens: node path[b][i] goes to slot length[b] + i with
 * position next_pos[b] + i and the weight mass_new (0 where that is NULL);
 * then length[b] and next_pos[b] grow by the number of tokens.  mass, pos and
 * next_pos of the cache may be NULL.  A session whose pages do not hold them
 * all stays as it is, and its status word receives UNISON_ERR_CAPACITY; so does
 * one whose path names a node that it has not, with UNISON_ERR_RANGE.
 * Reads k_new, v_new, mass_new. */
int unison_kv_commit(const unison_kv_cache *cache, const unison_kv_tree *tree, const unison_kv_step *step,
                     const unison_kv_path *path, void *cuda_stream);

/* Keeps min(length[b], keep[b]) slots of every session, for each KV head on
 * its own: protected slots first (pos < sink or pos >= next_pos[b] - recent),
 * among them the lower slot; then the larger mass, and of equal masses the
 * lower slot (NaN is below every number, -0 equals 0).  keep: device
 * int32[n_seqs], below 0 counts as 0.  Without pos (or next_pos) a slot's
 * index is its position and length[b] the next one.
 *   into = NULL  in place.  With n = slots kept, the i-th kept slot at or above
 *                n moves into the i-th evicted slot below n: nothing else
 *                moves.  length[b] becomes n.
 *   into         the i-th kept slot goes to slot i of the session in the other
 *                cache, which shares no page with this one and has the same
 *                n_seqs, n_heads, head_dim and dtype; its length[b] becomes n,
 *                its next_pos[b] this one's.  This cache stays as it is.  keep
 *                is clamped to the other page table's room, with
 *                UNISON_ERR_CAPACITY in the other cache's status word.
 * Keys, values, mass and pos move together (mass and pos where both caches
 * have them).  mass of this cache is required. */
uint64_t unison_kv_evict_workspace(const unison_kv_cache *cache);
int unison_kv_evict(const unison_kv_cache *cache, const unison_kv_cache *into, const int32_t *keep, int32_t sink,
                    int32_t recent, void *workspace, uint64_t workspace_bytes, void *cuda_stream);

/* Verification of drafted tokens (recursive rejection sampling).  p row i is
 * the target's distribution after node i, q row i the draft model's, from
 * which the children of node i were drawn; token[i] is node i's token.  For
 * every session, with w(x) = x clamped to [0, 1] and NaN taken as 0:
 *   cur = 0, d = w(p_cur), z = 1; then for the nodes i = 1, 2, .. whose parent
 *   is cur, in that order:
 *     accepted if (u[i] * w(q_cur[t])) * z < d[t], t = token[i]:
 *         cur = i, d = w(p_cur), z = 1
 *     else d = max(d - z * w(q_cur), 0), z = sum floor(d 2^40) / 2^40
 *   next = the least v with sum_{x <= v} floor(d[x] 2^40) > floor(u_sample[b] W),
 *   W the sum over all x; if W = 0, with d = w(p_cur); if that has none, -1.
 * q = NULL stands for drafts that were certain (q = 1 at the child's token):
 * accepted if u[i] * z < d[t], else d[t] = 0.  The 32-bit products are rounded
 * one by one and the sums are of whole numbers, so a decision does not depend
 * on the order of summation.  u and u_sample are in [0, 1); u_sample counts in
 * steps of 2^-24.  A node whose token is outside [0, vocab) is passed over.
 * Outputs: path[b][0 .. n_path[b]-1] the accepted nodes, the root first, -1
 * behind them (path_stride >= max_tokens); n_path[b]; next_token[b].  A
 * session without nodes gets n_path 0 and next_token -1.
 * dtype of p and q: BF16, FP16 or FP32; row strides in elements; vocab 1 ..
 * 2^22. */
typedef struct {
  const void *p;
  const void *q;
  int64_t p_row, q_row;
  const int32_t *token;  /* [n_tokens] */
  const float *u;        /* [n_tokens] */
  const float *u_sample; /* [n_seqs]   */
  int32_t *path;
  int32_t *n_path;
  int32_t *next_token;
  int64_t path_stride;
  int32_t vocab, dtype;
} unison_kv_verify_args;
int unison_kv_verify(const unison_kv_tree *tree, const unison_kv_verify_args *args, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* UNISON_KV_H */
