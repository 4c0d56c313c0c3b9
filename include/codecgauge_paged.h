/*
 * codecgauge_paged.h -- paged KV cache of libcodecgauge: the cache that a serving loop keeps
 * beside the codec, and the operators of one step on it.
 *
 * Many requests of different lengths share one pool of fixed-size pages. One layer's pool is
 *   pool : bf16 or fp16 [2][n_pages][H][page][d]      (0 = keys, 1 = values)
 * which is the codec's KV layout [L][2][B][H][T][d] with L = 1, B = n_pages and T = page: a bf16
 * pool (or a copy of a range of its pages) is coded by cg_encode and restored by cg_decode as it
 * stands. (The attention reads pages, not codes: coded pages are decoded first.) Token t of request i lives in page block_table[i][t / page], row t % page; its *slot*
 * is page_id * page + t % page. The tables are the same for every layer.
 *
 * One step: cg_page_plan once (pages for the new tokens, positions, slots), then for each layer
 * cg_rotary_append (turn queries and keys, write keys and values into their slots) and
 * cg_paged_attention (the new queries over their own request's pages). cg_page_release gives
 * the pages of finished requests back.
 *
 * The conventions of codecgauge.h hold: device pointers owned by the caller, asynchronous on
 * `stream`, an int status, a message in cg_last_error(), device status bits in cg_get_status().
 * Lengths and tables are read on the device only, so no call waits for the GPU and all calls can
 * be captured in a CUDA graph. What the device finds wrong in them (a length, page or slot out of
 * range) raises a status bit and is skipped: no access leaves the arrays that were passed.
 */
#ifndef CODECGAUGE_PAGED_H
#define CODECGAUGE_PAGED_H

#include "codecgauge.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of a pool, and of the queries, keys, values and outputs that go with it. */
#define CG_BF16 0
#define CG_FP16 1

/* Device status bits of the paged operators (cg_get_status). */
#define CG_FLAG_PAGES_EXHAUSTED 0x8  /* a plan needed more pages than were free                 */
#define CG_FLAG_PAGED_RANGE     0x10 /* a length, page id, slot or table width was out of range */

/* Pool and block table.
 *   dtype     : CG_BF16 or CG_FP16 (ignored by the plan and the release)
 *   n_pages   : pages in the pool, >= 1; n_pages * page < 2^31
 *   page      : tokens per page: 16, 32, 64, 128 or 256
 *   H, d      : KV heads (1 .. 1024) and head dimension: 64, 128 or 256
 *   n_req     : rows of the block table, 1 .. 65536
 *   max_pages : columns of the block table, >= 1; a request holds at most max_pages * page tokens */
typedef struct {
    int32_t dtype;
    int32_t n_pages, page;
    int32_t H, d;
    int32_t n_req, max_pages;
} cg_pages;

/* ---- Page plan: lengths -> pages, positions and slots ----
 * Request i holds ctx_lens[i] tokens and gets new_lens[i] more; P(n) = ceil(n / page):
 *   fresh_i         = P(ctx_i + new_i) - P(ctx_i), F = exclusive prefix sum of fresh
 *   block_table[i][P(ctx_i) + j] = free_pages[free_count - 1 - (F_i + j)],  0 <= j < fresh_i
 *   seq_lens[i]     = ctx_i + new_i
 *   cu_new[i]       = sum of new_lens below i   (n_req + 1 entries)
 * and for the tokens in order, request by request, token k of request i at t = cu_new[i] + k:
 *   positions[t] = ctx_i + k,  slots[t] = block_table[i][positions[t] / page] * page + positions[t] % page
 * free_left[0] = free_count[0] - sum of fresh. free_pages is a stack: [n_pages] entries, of which
 * the first free_count[0] are free (a count outside 0 .. n_pages raises CG_FLAG_PAGED_RANGE).
 * n_tok is the size of positions and slots; entries past the last token get position 0 and slot -1
 * (a padded batch). seq_lens and free_left must not alias ctx_lens, new_lens and free_count: the
 * call changes nothing that it reads (block_table entries of tokens already held among them), so a
 * plan that ran out of pages can be dropped and made again: then CG_FLAG_PAGES_EXHAUSTED is
 * raised, free_left is negative (the pages that lack), and tokens without a page have slot -1.
 * A request that outgrows max_pages, a negative length, more than n_tok new tokens or a bad entry
 * of free_pages or block_table raises CG_FLAG_PAGED_RANGE; the tokens concerned get slot -1. More
 * than n_tok tokens in all raise it too; of the pages that these would need, the first n_tok + n_req
 * are dealt out.
 * One launch. Integer arithmetic only. n_tok may be 0. */
int cg_page_plan(const cg_pages* pages, int32_t n_tok, const int32_t* ctx_lens, const int32_t* new_lens,
                 const int32_t* free_pages, const int32_t* free_count, int32_t* block_table,
                 int32_t* seq_lens, int32_t* cu_new, int32_t* positions, int64_t* slots,
                 int32_t* free_left, void* stream);

/* The same with a stack of n_stack entries, which may be fewer than n_pages (what a program never
 * gives back needs no place; with n_stack 0 free_pages may be NULL). A free_count above n_stack
 * raises CG_FLAG_PAGED_RANGE and counts as n_stack. */
int cg_page_plan_stack(const cg_pages* pages, int32_t n_tok, const int32_t* ctx_lens, const int32_t* new_lens,
                       const int32_t* free_pages, int32_t n_stack, const int32_t* free_count, int32_t* block_table,
                       int32_t* seq_lens, int32_t* cu_new, int32_t* positions, int64_t* slots, int32_t* free_left,
                       void* stream);

/* Give back the pages of every request with done[i] != 0: with n = lens[i] tokens held, the pages
 * in its first P(n) table entries go on the stack in order of request and entry,
 * free_pages[free_count + k]; free_left = free_count + their number; lens_left[i] = 0 for these and
 * lens[i] for the others. An entry of -1 is no page and is passed over: what a plan that ran out of
 * pages leaves, and what a program writes in place of a page that it has put back on the stack itself
 * (a windowed request's old ones; an entry left standing would come on the stack a second time). Any
 * other entry outside the pool is passed over too and raises CG_FLAG_PAGED_RANGE, as pages do that
 * the stack of n_pages entries has no room for. block_table is not changed. free_left and lens_left
 * must not alias free_count and lens. */
int cg_page_release(const cg_pages* pages, const int32_t* lens, const int32_t* done, const int32_t* block_table,
                    int32_t* free_pages, const int32_t* free_count, int32_t* lens_left, int32_t* free_left,
                    void* stream);

/* ---- Rotary positions ----
 * The first `rot` channels of a head turn in rot / 2 pairs; pair c of a token at position p by the
 * angle p f_c:  (a, b) -> mscale (a cos - b sin, b cos + a sin).
 *   interleaved = 0 : pair c is channels (c, c + rot / 2);  1 : channels (2c, 2c + 1)
 *   transpose = 1   : the transposed map, (a, b) -> mscale (a cos + b sin, b cos - a sin): the
 *                     gradient of the map, and its inverse where mscale is 1
 * Channels from rot on are copied. Arithmetic in fp32, one rounding to the output type.
 * rot: a multiple of 16, 0 .. d (0 turns nothing). table: device, int64 [rot / 2], the frequency in
 * 2^-64 of a turn per position, round(2^64 f_c / (2 pi)) modulo 2^64, from cg_rotary_table. p times
 * it modulo 2^64 is the angle's fraction of a turn, exact in integers: long positions lose no
 * accuracy. */
typedef struct {
    int32_t rot;
    int32_t interleaved;
    int32_t transpose;
    float   mscale;
} cg_rotary_params;

/* Frequency rules for cg_rotary_table. f_c = base^(-2c / rot), then
 *   CG_ROPE_NONE   : as they are
 *   CG_ROPE_LINEAR : f_c / factor (interpolated positions)
 *   CG_ROPE_BANDS  : with u = original * f_c / (2 pi) turns over the original context and
 *                    t = clamp((u - low) / (high - low), 0, 1): (1 - t) f_c / factor + t f_c
 *   CG_ROPE_YARN   : pair index ramp: at(n) = rot ln(original / (2 pi n)) / (2 ln base),
 *                    lo = max(floor(at(high)), 0), hi = min(ceil(at(low)), rot - 1),
 *                    t = 1 - clamp((c - lo) / max(hi - lo, 0.001), 0, 1): (1 - t) f_c / factor + t f_c,
 *                    and mscale = 0.1 ln(factor) + 1 (1 for factor <= 1)
 * (BANDS commonly has low 1, high 4; YARN low 1, high 32.) */
#define CG_ROPE_NONE   0
#define CG_ROPE_LINEAR 1
#define CG_ROPE_BANDS  2
#define CG_ROPE_YARN   3
typedef struct {
    int32_t kind;
    double  base;      /* > 1 */
    double  factor;    /* > 0 */
    double  original;  /* > 0: context length the frequencies were trained for (BANDS, YARN) */
    double  low, high; /* turns, 0 < low < high (BANDS, YARN) */
} cg_rope_scaling;

/* Host-only: the table of rot / 2 pairs into host_table (rot / 2 integers), and mscale. */
int cg_rotary_table(int32_t rot, const cg_rope_scaling* scaling, int64_t* host_table, float* mscale);

/* out = rotary(x), x and out [n_tok][heads][d] with the given strides in elements (multiples of 8;
 * the last dimension is contiguous; 0 repeats an element of x, and is refused for out unless there is
 * but one). out may be x itself with the same strides. positions int32
 * [n_tok]; dtype and d as in cg_pages (d 64, 128 or 256). Pointers 16-byte aligned. */
int cg_rotary(const cg_rotary_params* rotary, int32_t dtype, int32_t n_tok, int32_t heads, int32_t d,
              const void* x, int64_t x_tok, int64_t x_head, const int32_t* positions, const int64_t* table,
              void* out, int64_t out_tok, int64_t out_head, void* stream);

/* Strides in elements of the queries, keys and values of cg_rotary_append (multiples of 8; o of q_out,
 * not 0 over more than one element). */
typedef struct {
    int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;
} cg_append_strides;

/* q_out = rotary(q) (q [n_tok][q_heads][d]), rotary(k) into the key half and v into the value half
 * of the pool at slots[t] (k, v [n_tok][H][d]). Slot -1 writes nothing to the pool; a slot outside
 * the pool raises CG_FLAG_PAGED_RANGE and writes nothing. No two tokens may have one slot. q_heads
 * may be 0 (q, q_out then unused). q_out may be q itself with the same strides. One launch. */
int cg_rotary_append(const cg_pages* pages, const cg_rotary_params* rotary, int32_t n_tok, int32_t q_heads,
                     const cg_append_strides* strides, const void* q, const void* k, const void* v,
                     const int32_t* positions, const int64_t* slots, const int64_t* table, void* q_out, void* pool,
                     void* stream);

/* ---- Attention of new tokens over a paged cache ----
 * Request i has seq_lens[i] tokens in the pool, the last n_i = cu_new[i+1] - cu_new[i] of which are
 * new and bring queries: query row cu_new[i] + k stands at position p = seq_lens[i] - n_i + k and
 * sees the tokens t <= p with (window == 0, or t > p - window, or t < sinks). Query head j reads KV
 * head j / n_rep:
 *   o = sum_t softmax_t(scale q . k_t) v_t,   lse = ln sum_t exp(scale q . k_t)
 * A query that sees nothing (a negative position) gives o = 0 and lse = -inf. Scores, softmax and
 * sums are fp32; the weights enter the value product rounded to the pool's type (summed before that),
 * the row's largest among them unless the request has few query rows; o is rounded once.
 * Values may be as large as fp32 has room for their sum over the visible tokens.
 * Rows of the pool past a request's length are never used, whatever they hold (NaN and infinities
 * too); block table entries of pages that no query sees are not used either (a windowed request's old
 * pages may be back on the stack, with -1 in their entries). A visible token whose entry is no page
 * raises CG_FLAG_PAGED_RANGE and counts with a key and a value of zeros.
 *   n_tok   : rows of q, out and lse; cu_new[n_req] <= n_tok (rows from cu_new[n_req] on are left
 *             untouched)
 *   n_rep   : query heads per KV head, 1 .. 64
 *   max_new : an upper bound of the n_i (sizes the launches; a request with more raises
 *             CG_FLAG_PAGED_RANGE and its output is not written)
 *   window  : >= 0, sinks : >= 0 (only with a window);  scale : finite
 *   strides in elements, multiples of 8 (o of out, not 0 over more than one element).
 *   q [n_tok][H * n_rep][d], out alike, lse fp32
 *   [n_tok][H * n_rep] contiguous or NULL.
 * workspace: device scratch of cg_paged_attention_workspace_bytes, owned by the caller; needs no
 * initial value and may be shared by calls that are issued one after the other on one stream. (A call
 * is up to three launches: two host threads that call at the same time, on one stream too, may mix
 * theirs and need a workspace each.) Its size does not depend on n_req, n_tok or the pages, and does
 * not shrink as n_rep or max_new grow. */
typedef struct {
    int32_t n_tok, n_rep, max_new;
    int32_t window, sinks;
    float   scale;
    int64_t q_tok, q_head, o_tok, o_head;
} cg_paged_attn;

int cg_paged_attention_workspace_bytes(const cg_pages* pages, const cg_paged_attn* how, size_t* workspace_bytes);
int cg_paged_attention(const cg_pages* pages, const cg_paged_attn* how, const void* q, const void* pool,
                       const int32_t* block_table, const int32_t* seq_lens, const int32_t* cu_new, void* out,
                       float* lse, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CODECGAUGE_PAGED_H */
