/*
 * spdraft.h - C ABI of drafted tokens over the paged cache of spattn.h, on MI355X (gfx950).
 *
 * A small model drafts trees of tokens behind sequences; the large one takes all of a tree's nodes in one pass and says which of them stay.  A step of
 * serving: spdraft_symbolic brings the trees' structure into the form that the kernels walk, once for all layers; in every layer spcache_append
 * puts the nodes' keys and values into the pages and spdraft_attend computes their attention; spdraft_verify chooses the nodes that stay and the
 * token that follows; spdraft_keep moves what stays together in the pages of all layers.  (spcache_fork with parent[r] = r and the lengths that
 * spdraft_keep leaves gives back the pages that a row no longer needs.)
 *
 * Conventions: those of spattn.h (tensors, handle, stream, scratch memory, status codes).  No call but spdraft_symbolic, where it is given `checked`, waits for the stream.
 */
#ifndef SPDRAFT_H_
#define SPDRAFT_H_

#include "spattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Nodes of a tree, at most. */
#define SPDRAFT_MOST 256

/* Element types of rows of probabilities: those of spattn_dtype, and 32 bits. */
#define SPDRAFT_F32 2

/* The trees of a batch: nodes ptr[s] .. ptr[s+1] - 1 are sequence s's.  Within its tree node i has the number i; parent[i] < i is the node that it
 * continues, -1 the context alone.  A tree may be empty, and may have several nodes that continue the context; only spdraft_verify asks that the first node be the root of what it walks. */
typedef struct {
  int64_t rows;          /* sequences */
  int64_t tokens;        /* nodes of all trees, below 2^24 */
  const int64_t* ptr;    /* device, rows + 1, from 0 to tokens */
  const int32_t* parent; /* device, tokens */
  int32_t most;          /* no tree has more nodes: 1 to SPDRAFT_MOST */
} spdraft_trees;

/* Device memory that a plan of these trees takes (only tokens and most count); 0 for trees that spdraft_symbolic refuses. */
size_t spdraft_plan_bytes(const spdraft_trees* t);

/* The trees' structure into plan_mem (device, caller-owned, 256-byte aligned, spdraft_plan_bytes).  `parent` is not needed after that; ptr is, by every call that the plan is given to.
 * checked: host, or null.  Given, the call waits, and a ptr that does not go from 0 to tokens in ascending order, a tree of more than `most` nodes or a parent
 * that is not an earlier node is SPGEMM_INVALID_INPUT (checked: 0, else 1).  Without it ptr is cut to what exists, such a parent counts as -1, and nodes behind a tree's `most` first
 * are left out by every call: nothing is written for them. */
int spdraft_symbolic(spgemm_handle h, const spdraft_trees* t, void* plan_mem, size_t plan_bytes, int32_t* checked);

/* o = attention of the trees' nodes (q and o: node ptr[s] + i) over their sequences' cache.  The nodes are the last tokens of their sequence, in their order: lens[s]
 * counts them, ctx = lens[s] - nodes of s.  Node i sees the ctx tokens before the tree, its ancestors and itself.  It stands at ctx + depth(i), a node without
 * a parent at ctx; distances (slopes, window) are between such places: with window > 0 it sees only what stands less than `window` before it.  Scores as in spattn_args.  A node
 * that sees nothing (a sequence with fewer tokens than its tree) has the output 0; of a table without the pages the last tokens that it has count, as in spcache_attend.
 * What a node does not see it does not feel: a key or value that is not finite reaches those alone that see it. */
int spdraft_attend(spgemm_handle h, const spcache* c, int64_t layer, const spgemm_csr* table, const int32_t* lens, const spdraft_trees* t, const void* plan_mem,
                   int32_t heads, int32_t dtype, float scale, float cap, const float* slopes, int64_t window, spattn_tensor q, spattn_tensor o);

/* Rows of probabilities: row i at data + i * stride elements. */
typedef struct {
  const void* data;
  int64_t stride;
} spdraft_rows;

/* Which nodes stay, so that the tokens are distributed as the target's.  Node 0 of a tree is the token that the step before ended with: it stays.  ids[i] is node i's token; row i of
 * target holds the target's probabilities behind node i, row i of draft those that i's children were drawn from, one after the other, without replacement.
 * At a node let r and q be its rows; children are asked in order.  Child i with token x is taken if u[i] q(x) < r(x), and the walk goes on there.  Otherwise r becomes max(r - q, 0) and q
 * loses x, both divided by their sums (an r of which nothing is left stays as it was).  Without draft (data null: children that were not drawn but chosen) q is
 * 1 at x and 0 elsewhere.  Where no child is taken, next[s] is the first token v at which r(0) + .. + r(v) passes u[root] times the sum of r.
 * Rows are taken as they are, not brought to the sum 1 first.  Entries that are negative or NaN count as 0, an infinite one leaves the result unspecified; a child whose token is not in the vocabulary
 * is passed over.  Differences and sums are in 64 bits.
 *   vocab: 1 to 2^24.  ids: device, tokens.  u: device, tokens, from 0 to below 1.  dtype: of both rows.
 *   path: device, tokens: path[ptr[s]] .. are the nodes of s that stay, in order, -1 behind them.  kept: device, rows: how many.  next: device, rows; -1 for an
 *   empty tree and where r has no entry above 0.  Outputs must not overlap inputs. */
int spdraft_verify(spgemm_handle h, const spdraft_trees* t, const void* plan_mem, int64_t vocab, int32_t dtype, spdraft_rows target, spdraft_rows draft, const int32_t* ids,
                   const float* u, int32_t* path, int32_t* kept, int32_t* next);

/* In all layers, token path[ptr[s] + i] of the tree of s becomes its token i, i < kept[s]; new_lens[s] = ctx + kept[s].  A path ascends; one that does not, or leaves the tree, ends before
 * that entry.  A token that comes from another page is rounded under the scale of its new page, which grows as with spcache_append where the token does not
 * fit; the tokens before and beside it are then rounded again.  Bytes behind the tokens that stay are left as they were.  A sequence with
 * fewer tokens than its tree, or whose table lacks pages that the tree's nodes lie in, is left as it is, new_lens[s] = lens[s].
 * Pages that hold a tree's nodes belong to its sequence alone.  new_lens: device, rows; it must not overlap lens, path or kept. */
int spdraft_keep(spgemm_handle h, const spcache* c, const spgemm_csr* table, const int32_t* lens, const spdraft_trees* t, const int32_t* path, const int32_t* kept,
                 int32_t* new_lens);

#ifdef __cplusplus
}
#endif
#endif /* SPDRAFT_H_ */
