/*
 * codecgauge_tree.h -- trees of drafted tokens over the paged cache: a serving loop that drafts several
 * continuations of each request checks them all in one step.
 *
 * A request's drafted tokens are the nodes of a tree, in an order in which a parent stands before its children.
 * For the cache they are new tokens like any others: cg_page_plan gives them pages and slots, in their
 * order, behind the ctx tokens that the request holds; node k lies in row ctx + k. What differs is what they
 * see and where they stand: node k sees the request's history and, of the nodes, its ancestors and itself, and its
 * position is ctx + depth. One step of one layer:
 *   cg_page_plan       pages and slots (its positions are not the tree's)
 *   cg_tree_plan       positions and masks, once for all layers with the same window
 *   cg_rotary_append   with the tree's positions and the plan's slots
 *   cg_tree_attention
 * and once the program has accepted a node of each tree, cg_tree_commit moves the accepted path's keys and values
 * up behind the history, in the pools of all layers, and gives the pages back that no token is left in.
 *
 * The conventions of codecgauge_paged.h hold. Lengths, parents and tables are read on the device only, no
 * call waits for the GPU, all can be captured in a CUDA graph. Per request i: n_i = cu_new[i+1] - cu_new[i]
 * nodes, seq_lens[i] tokens with them, ctx_i = seq_lens[i] - n_i. Lengths that do not fit (a negative one, n_i
 * above max_new or seq_lens[i], cu_new outside 0 .. n_tok, for the attention and the commit more tokens than
 * max_pages hold) raise CG_FLAG_PAGED_RANGE and the request counts as without nodes.
 */
#ifndef CODECGAUGE_TREE_H
#define CODECGAUGE_TREE_H

#include "codecgauge_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Nodes of one tree at most (cg_tree_plan, cg_tree_commit). The plan is made for trees of up to some hundred: its time
 * grows with the square of the nodes, and one of 8192 takes a millisecond. */
#define CG_TREE_NODES 8192

/* ---- Positions and masks of the nodes ----
 * parents[cu_new[i] + k] is the parent of node k of request i, in [-1, k); -1: the last token held. With
 * depth(k) = 0 for parent -1, else depth(parent) + 1, and t = cu_new[i] + k:
 *   positions[t] = ctx_i + depth(k)
 *   masks[t]     : mask_words 32-bit words, bit b of the row (bit b & 31 of word b / 32) set if b is k or an
 *                  ancestor of k and, with a window, depth(k) - depth(b) < window or ctx_i + depth(b) < sinks
 * Rows from cu_new[n_req] on get position 0 and no bits. A parent outside [-1, k) raises CG_FLAG_PAGED_RANGE
 * and counts as -1.
 *   n_req : 1 .. 65536;  n_tok : rows of parents, positions and masks;  max_new : 0 .. CG_TREE_NODES, bound of the n_i
 *   window >= 0, sinks >= 0 (only with a window);  32 mask_words >= max_new
 * positions and masks must not alias the inputs. One launch. Integer arithmetic only. */
int cg_tree_plan(int32_t n_req, int32_t n_tok, int32_t max_new, int32_t window, int32_t sinks, const int32_t* parents,
                 const int32_t* seq_lens, const int32_t* cu_new, int32_t* positions, uint32_t* masks,
                 int32_t mask_words, void* stream);

/* ---- Attention of the nodes ----
 * cg_paged_attention (its formulas, types, strides, workspace, checks and flags), but for what a query sees:
 * the row of node k sees tokens t < ctx_i with (window == 0, or t > positions[..] - window, or t < sinks), and
 * node j, token ctx_i + j, if bit j of its mask is set. Bits from n_i on count for nothing; any masks are
 * allowed, not only a tree's (a row without bits sees the history alone; a row that sees nothing gives o = 0 and
 * lse = -inf). positions is read only with a window (else NULL may be given) that is shorter than a request can
 * be, max_pages * page; a position outside [ctx_i, ctx_i + k] then raises CG_FLAG_PAGED_RANGE and counts as the
 * nearest of them.
 * masks [n_tok][mask_words], 32 mask_words >= how->max_new. workspace: of
 * cg_paged_attention_workspace_bytes for the same pages and how. */
int cg_tree_attention(const cg_pages* pages, const cg_paged_attn* how, int32_t mask_words, const void* q, const void* pool,
                      const int32_t* block_table, const int32_t* seq_lens, const int32_t* cu_new,
                      const int32_t* positions, const uint32_t* masks, void* out, float* lse, void* workspace,
                      size_t workspace_bytes, void* stream);

/* ---- The accepted path ----
 * leaves[i] is the accepted node of request i, or -1: none; r_0 < ... < r_{m-1} = leaves[i] is its path from
 * the root (m = 0 for -1). In every layer's pool row ctx_i + r_k moves to row ctx_i + k, keys and values, and
 *   lens_left[i] = ctx_i + m
 * The pages of table entries P(lens_left[i]) .. P(seq_lens[i]) - 1 (P(n) = ceil(n / page)) go on the stack, in
 * order of request and entry, free_pages[free_count + k]; free_left = free_count + their number. As for
 * cg_page_release, an entry of -1 is passed over, another one outside the pool too and raises
 * CG_FLAG_PAGED_RANGE, and so do pages that the stack of n_pages entries has no room for; block_table is not
 * changed. Rows in pages outside the pool are not moved and raise the flag. Other rows are left as they are. A
 * leaf outside [-1, n_i) raises the flag and counts as -1; so does a parent outside [-1, k) of a node k of the path.
 *   layers : pools at `pool`, one after the other: [layers][2][n_pages][H][page][d]
 *   pool may be NULL (layers 0): only lengths and pages, H, d and dtype ignored; lens_left may be NULL (then free_pages, free_count
 *   and free_left too): only rows. A request may be committed once: its rows have moved then.
 * A request whose lengths do not fit keeps them: lens_left[i] = seq_lens[i] (0 for a negative one).
 * lens_left, free_left and free_pages must not alias the inputs or one another. max_new: 0 .. CG_TREE_NODES. One launch. */
int cg_tree_commit(const cg_pages* pages, int32_t n_tok, int32_t max_new, int32_t layers, const int32_t* parents,
                   const int32_t* leaves, const int32_t* seq_lens, const int32_t* cu_new, const int32_t* block_table,
                   void* pool, int32_t* lens_left, int32_t* free_pages, const int32_t* free_count,
                   int32_t* free_left, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CODECGAUGE_TREE_H */
