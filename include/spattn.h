/*
 * spattn.h - C ABI of attention over sparse structures on MI355X (gfx950), beside the products of spgemm.h.
 *
 * Attention is the product P * V of a sparse matrix whose entries are made on the way: P's structure is a mask (here: documents given
 * by row pointers, and optionally a compressed pattern of tiles, such as a product's structure), its entries the row-wise softmax of the
 * sampled product Q * K^T.  As in spgemm.h a symbolic call brings the structure into the form that the kernels walk, and numeric calls
 * (forward, backward) use it as often as they like.  The second half serves one token after another: a cache of pages in 8 bits, a
 * page table in compressed rows, attention over both, and the table's steps from one choice of sequences to the next.
 *
 * Conventions: those of spgemm.h (handle, stream, status codes, spgemm_last_error).  Further:
 *   - Tensors are device pointers to 16-bit elements, rows of head_dim contiguous elements, at base + token * token_stride + head *
 *     head_stride (strides in elements).  Base and strides must be multiples of 16 bytes, a token stride below 2^23 elements.
 *   - head_dim is a multiple of 8 from 8 to 128.
 *   - A call only enqueues work on the handle's stream, unless it is given a host pointer for its result: then it waits for the stream.
 *   - Scratch memory comes from the handle's allocator, grows with the largest call and stays with the handle.  A call that needs more than
 *     any before waits for the stream, so a graph is best captured after a call of its size.  What a captured call uses stays where it is until
 *     spgemm_destroy, whatever calls follow: a graph may be replayed for as long as the handle that it was captured with lives.  All calls and graphs of a
 *     handle share the scratch memory, so no two of them run at the same time: they go to the handle's stream, or are ordered by the caller.
 *   - spgemm_destroy waits for the handle's stream where such calls were made: the stream has to exist still, and no capture be under way.
 *   - Sums, maxima and logarithms are held in 32 bits; probabilities and their gradients are rounded to the 16-bit type where they
 *     become an operand of a matrix instruction.  The same inputs give the same bits.  (Values are added up before they are divided: where the largest, times
 *     the tokens of a row, reach 2^128, or 2^96 with a cap, the result is infinite.)
 */
#ifndef SPATTN_H_
#define SPATTN_H_

#include "spgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SPATTN_F16 = 0, SPATTN_BF16 = 1 } spattn_dtype;

/* A tensor of tokens and heads.  Elements of q, k, v and all results have one type. */
typedef struct {
  void* data;
  int64_t token_stride, head_stride; /* elements */
} spattn_tensor;

/* Rows and columns of a tile of a pattern. */
#define SPATTN_TILE 128

/* Which keys a query sees.  Queries q_ptr[d] .. q_ptr[d+1] - 1 and keys k_ptr[d] .. k_ptr[d+1] - 1 belong to document d; a document may have no
 * queries, no keys, or more of either.  Its last query stands at its last key: query i stands at key
 * diag = i + k_ptr[d+1] - q_ptr[d+1].  It sees the keys of its document from lo to before hi:
 *   hi: the document's end or, with causal, max(k_ptr[d] + prefix[d], diag + 1);  lo: the document's begin or, with window > 0, diag - window + 1.
 * With a pattern, (i, j) is visible only if entry (i / SPATTN_TILE, j / SPATTN_TILE) is stored; its columns may be in any order and
 * repeat, values are not read.  Rows that see nothing have the output 0, the logarithm -inf and no gradient.
 * Queries and keys outside all documents see nothing and are seen by nobody; their elements are not used.  Inside one, what a
 * query does not see has no weight.  But products go over tiles of 128 queries and 128 keys: an element that is not finite may make NaN (as 0 * inf
 * does) the results of any row or key of a tile that it lies in, whether that sees it or not. */
typedef struct {
  int64_t q_len, k_len;   /* below 2^30 */
  int64_t docs;           /* 0: one document of everything */
  const int64_t* q_ptr;   /* device, docs + 1, ascending; null when docs is 0 */
  const int64_t* k_ptr;   /* device, docs + 1 */
  const int64_t* prefix;  /* device, docs (1 when docs is 0), or null: no prefix */
  int32_t causal;         /* 0 or 1 */
  int64_t window;         /* 0: none */
  const spgemm_csr* tiles; /* pattern, ceil(q_len / 128) x ceil(k_len / 128), or null */
} spattn_mask;

/* Device memory that a plan of this mask takes (only sizes and the presence of a pattern count); 0 for a mask that spattn_symbolic refuses. */
size_t spattn_plan_bytes(const spattn_mask* mask);

/* The mask's structure into plan_mem (device, caller-owned, 256-byte aligned, spattn_plan_bytes).  After that the mask's arrays are not needed.
 * checked: host, or null.  Given, the call waits, and documents that are not ascending or leave the tensors and pattern columns out of range
 * are SPGEMM_INVALID_INPUT (checked: 0, else 1); without it they are cut to what exists. */
int spattn_symbolic(spgemm_handle h, const spattn_mask* mask, void* plan_mem, size_t plan_bytes, int32_t* checked);

/* What both passes have in common.  heads is a multiple of kv_heads; query head h uses key head h / (heads / kv_heads).
 * The score of a visible pair is cap * tanh(scale * q.k / cap) - slopes[h] * |diag - j|, without the tanh where cap is 0, without the
 * distance where slopes is null.  The tanh is off by at most 3e-7, a capped score so by 3e-7 * cap: a cap far above the scores costs digits.
 * slopes are constants: no gradient is formed for them. */
typedef struct {
  const spattn_mask* mask;  /* sizes and the presence of a pattern as at spattn_symbolic */
  const void* plan_mem;
  int32_t dtype;            /* spattn_dtype */
  int32_t heads, kv_heads, head_dim;
  float scale;              /* above 0 */
  float cap;                /* 0: none */
  const float* slopes;      /* device, heads, or null */
  spattn_tensor q, k, v;
} spattn_args;

/* o = softmax(scores) * v, lse = the logarithm of each row's sum (device float, heads x q_len). */
int spattn_forward(spgemm_handle h, const spattn_args* a, spattn_tensor o, float* lse);

/* Gradients of sum(o * d_o) with respect to q, k and v, from forward's o and lse.  Key heads that several query heads share get the sum.
 * Probabilities and the scores' gradients are rounded to the type once, as operands, and so is o, which the row sums of o * d_o are made from: against 64 bits
 * dq and dk are off by 1.65 to 1.9 times what rounding the result alone costs.  In float16 both operands are scaled by powers of two, a row's or key's
 * own where its gradients are large, so that neither small nor large ones, nor long rows, lose digits before the result is rounded. */
int spattn_backward(spgemm_handle h, const spattn_args* a, spattn_tensor o, const float* lse, spattn_tensor d_o, spattn_tensor dq,
                    spattn_tensor dk, spattn_tensor dv);

/* ---- cache ------------------------------------------------------------------------------------
 * A page holds SPCACHE_PAGE tokens of one sequence.  Every page, layer and key head has a scale for keys and one for values, a power of
 * two: the least with which the largest finite magnitude that was put into the page stays within 448.  An entry x is kept as x / scale in e4m3, rounded
 * to nearest (ties to even); infinities become the largest value.  room is 64 for a head_dim of at most 64, else 128.
 * Bytes behind a sequence's last token and channels from head_dim to room may hold anything. */
#define SPCACHE_PAGE 64

typedef struct {
  int64_t layers, pages;  /* pages below 2^24 */
  int32_t kv_heads, head_dim;
  void* k;                /* device, [layers][pages][kv_heads][SPCACHE_PAGE][room], 16-byte aligned */
  void* v;                /* device, [layers][pages][kv_heads][room][SPCACHE_PAGE] */
  float* k_scale;         /* device, [layers][pages][kv_heads] */
  float* v_scale;
} spcache;

/* A page table is a spgemm_csr: row s lists the pages of sequence s in order (rows: sequences, cols: the cache's pages; values and dtype are
 * not used).  lens[s] (device) is how many tokens sequence s has.  Sequences may share pages that they have whole. */

/* New tokens into a layer: rows new_ptr[s] .. new_ptr[s+1] - 1 (device, rows + 1, from 0 to tokens) of k and v become the last tokens of sequence
 * s, whose lens[s] counts them already.  A page that gets its first token starts with a new scale; where a later token needs a larger one, the
 * tokens before are rounded again.  A sequence whose table does not have the pages is left as far as they lack. */
int spcache_append(spgemm_handle h, const spcache* c, int64_t layer, const spgemm_csr* table, const int32_t* lens, const int64_t* new_ptr,
                   int64_t tokens, int32_t dtype, spattn_tensor k, spattn_tensor v);

/* o = attention of the last q_len tokens of every sequence (q and o: token s * q_len + i) over its cache.  Token i sees the keys up to itself, with
 * window > 0 only the last `window` of those.  Scores as in spattn_args.  A token before the sequence's first has the output 0.
 * q_len * heads is at most 65535. */
int spcache_attend(spgemm_handle h, const spcache* c, int64_t layer, const spgemm_csr* table, const int32_t* lens, int64_t q_len, int32_t heads,
                   int32_t dtype, float scale, float cap, const float* slopes, int64_t window, spattn_tensor q, spattn_tensor o);

/* The table's next step: row r of the new table continues row parent[r] of the old one (-1: nothing) and has new_lens[r] tokens, of which
 * min(lens[parent[r]], new_lens[r]) are the parent's.  So rows are copied, cut, grown and, where no row continues them, ended.  Pages that a
 * row has whole are shared.  A page in which rows end stays with the first of them, unless another row has it whole; the others get a copy,
 * in all layers.  New pages are those with the least numbers that no row of the new table kept, rows in order.
 *   parent, new_lens: device, n_out.  out_rowptr: device, n_out + 1; out_pages: device, room entries; refs: device, pages: how often
 *   the new table has each page.  Outputs must not overlap inputs.
 *   nnz_out: host, or null.  Given, the call waits and SPGEMM_INVALID_INPUT (a parent or page out of range, a parent without its pages, room too
 *   small) and SPGEMM_ALLOC_FAILED (no page left, or a row longer than the whole cache) are reported; without it such a call leaves the cache as it is and the
 *   outputs unspecified. */
int spcache_fork(spgemm_handle h, const spcache* c, const spgemm_csr* table, const int32_t* lens, int64_t n_out, const int32_t* parent,
                 const int32_t* new_lens, int64_t* out_rowptr, int32_t* out_pages, int64_t room, int32_t* refs, int64_t* nnz_out);

/* The pages in use (those of the table) to the front of the cache: the i-th of them at or behind their number goes to the i-th place before it that
 * is free, in all layers; out_pages (device, table->nnz, not the table's own) are the table's entries after that.
 *   live: host, or null: how many pages are in use.  Given, the call waits; a page out of range is SPGEMM_INVALID_INPUT (the cache is left as it is). */
int spcache_compact(spgemm_handle h, const spcache* c, const spgemm_csr* table, int32_t* out_pages, int64_t* live);

/* Page dst[i] becomes a copy of page src[i] in all layers (device, n each; destinations distinct, and none of them a source).  Pairs out of range are
 * passed over. */
int spcache_copy(spgemm_handle h, const spcache* c, int64_t n, const int32_t* src, const int32_t* dst);

#ifdef __cplusplus
}
#endif
#endif /* SPATTN_H_ */
