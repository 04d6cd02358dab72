/*
 * span_paged.h — C ABI of the operators on a key / value cache in pages (MI355X, gfx950).
 *
 * A pool holds num_pages pages of K rows and as many of V rows; a sequence's cache is the pages that its row of the
 * block table names, so caches grow page by page and need not be allocated to their maximum length.  Several query
 * heads may share a KV head (query head i reads KV head i / (heads / kv_heads)).
 *
 * Conventions are those of span_attn.h: device memory is the caller's, work is enqueued on desc->stream and the calls
 * return without synchronising or allocating; 0 = OK, negative = refused on the host before anything was launched;
 * nothing throws or aborts across this ABI.  The device that owns desc->stream has to be the current one.  Every call
 * can be recorded into a HIP graph; lengths and block tables are read on the device by every replay.
 *
 * Layouts, all contiguous and aligned to 16 bytes:
 *   k_pages, v_pages   desc->dtype  [num_pages, kv_heads, page_size, head_dim]
 *   block_table        int32        [batch, table_pages]: position p of sequence b is row p % page_size of page
 *                                   block_table[b, p / page_size].  A page outside [0, num_pages) is never read or
 *                                   written: its positions are attended by nobody, rows for it are dropped.
 *   ctx_lens           int32 [batch]: positions in use.  Those from table_pages * page_size on have no row: a token there keeps
 *                                   its position (what a window hides from it goes by that), and nobody attends it.  A negative
 *                                   length counts as 0
 *   q_offsets          int32 [batch + 1]: rows q_offsets[b] .. q_offsets[b + 1] - 1 of q / k_new / v_new / out are the
 *                                   new tokens of sequence b, the last of them at position ctx_lens[b] - 1 (ctx_lens
 *                                   counts them already); not decreasing, within [0, num_tokens].  Rows that belong to
 *                                   no sequence are left alone.
 *   weights            fp32  [batch, kv_heads, table_pages * page_size]: attention weight gathered by a position
 *   positions          int32 [batch, kv_heads, table_pages * page_size]: true position of the row a slot holds
 */
#ifndef SPAN_PAGED_H_
#define SPAN_PAGED_H_

#include "span_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct span_paged_desc {
  int32_t batch;           /* 1 .. 65535                                                                    */
  int32_t heads, kv_heads; /* heads is a multiple of kv_heads, 16 times kv_heads at most                    */
  int32_t head_dim;        /* 64 or 128                                                                     */
  int32_t dtype;           /* span_dtype_t of the pages, q and the new rows                                 */
  int32_t page_size;       /* rows of a page: a power of two, 16 .. 1024                                    */
  int32_t num_pages;       /* pages of the pool; num_pages * page_size < 2^31                               */
  int32_t table_pages;     /* entries of a sequence in block_table; table_pages * page_size <= 2^22         */
  int32_t num_tokens;      /* paged_append, paged_prompt_attn: rows of k_new / q                            */
  int32_t window, sinks;   /* paged_decode_attn, paged_prompt_attn: a token sees the last `window` positions up
                              to its own (0: all of them) and the first `sinks`; paged_evict: the first `sinks`
                              positions always stay; paged_select: their pages are listed in any case       */
  int32_t num_intervals;   /* paged_span_decode_attn: entries held by span_starts / span_ends               */
  int32_t num_splits;      /* one-token calls: 0 = the library cuts the caches into slices as it finds best, > 0 =
                              so many slices per sequence                                                   */
  int32_t budget, recent;  /* paged_evict: rows of a cache that stay, the last of them in any case; paged_select,
                              paged_selected_decode_attn: pages of a list; paged_select: the last positions, whose
                              pages are listed in any case                                                  */
  const int64_t* tokens_per_seq; /* paged_span_decode_attn: HOST int64 [batch] or NULL: attended positions of every
                              sequence as span_validate returns them; they only set the slices (a wrong number costs
                              time, not correctness).  Read during the call only.                           */
  void* workspace;         /* device, 256-byte aligned, at least paged_workspace_bytes(); for one-token calls,
                              paged_select and paged_evict its ticket counters (the first 4 * batch * (kv_heads + 1) bytes, rounded up to
                              256) must be zero before the first call (paged_workspace_init); every call leaves them
                              zero again.  A workspace that served another batch, another number of KV heads or
                              paged_prompt_attn is initialised again.  Two calls that may overlap in time must not share one.    */
  size_t workspace_bytes;
  void* stream;            /* hipStream_t; NULL = the default stream                                        */
} span_paged_desc_t;

/* SPAN_OK, or what any call with this descriptor is refused with for its sizes and type. */
int paged_check(const span_paged_desc_t* desc);

/* What a workspace is for. */
typedef enum {
  PAGED_DECODE = 0,              /* paged_decode_attn                                                        */
  PAGED_DECODE_WEIGHTS = 1,      /* paged_decode_attn with weights                                           */
  PAGED_SPAN_DECODE = 2,         /* paged_span_decode_attn                                                   */
  PAGED_SPAN_DECODE_WEIGHTS = 3, /* paged_span_decode_attn with weights                                      */
  PAGED_PROMPT = 4,              /* paged_prompt_attn                                                        */
  PAGED_EVICT = 5,               /* paged_evict                                                              */
  PAGED_SELECT = 16,             /* paged_select                                                             */
  PAGED_SELECTED_DECODE = 17,    /* paged_selected_decode_attn                                               */
  PAGED_DECODE_FP4 = 18,         /* paged_decode_attn_fp4                                                    */
  PAGED_SPAN_DECODE_FP4 = 19     /* paged_span_decode_attn_fp4                                               */
} span_paged_use_t;

/* Bytes of workspace the call described by desc wants (0: none; also for a descriptor that would be refused). */
size_t paged_workspace_bytes(const span_paged_desc_t* desc, int use);

/* Enqueues the zeroing of the ticket counters at the head of desc->workspace (a small kernel; can be recorded into a
 * graph).  Needed once after the workspace is allocated, and after anything else wrote to it. */
int paged_workspace_init(const span_paged_desc_t* desc);

/*
 * New rows into the pages: for every sequence b, new token j (of t = q_offsets[b+1] - q_offsets[b]), p = ctx_lens[b] - t + j,
 *   k_pages[block_table[b, p / page_size], h, p % page_size, :] = k_new[q_offsets[b] + j, h, :]   (same for V)
 *   positions[b, h, p] = seen[b] - t + j                                                         (if positions is given)
 *   k_new, v_new : device, desc->dtype, [num_tokens, kv_heads, head_dim]
 *   q_offsets    : NULL = one token per sequence (num_tokens == batch)
 *   seen         : device int32 [batch] or NULL: tokens of the sequence so far, the new ones among them; NULL = ctx_lens
 *                  (differs from it once rows were evicted)
 * Rows whose position lies outside [0, table_pages * page_size) are dropped, so that a full table keeps what it holds, and so are
 * those of a page outside the pool.  Pages written to must belong to one sequence only.
 */
int paged_append(const span_paged_desc_t* desc, const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                 const int32_t* block_table, const int32_t* ctx_lens, const int32_t* q_offsets, int32_t* positions,
                 const int32_t* seen);

/* Turns pairs of channels of a row by the angles of its token's position. */
typedef struct paged_rotation {
  const float* table;  /* device, 16-byte aligned, fp32 [positions, channels]: the cosines of a position's channels / 2 angles, then their sines */
  int32_t positions;
  int32_t channels;    /* of a row that are turned, its first ones: a multiple of 16, up to head_dim           */
  int32_t paired;      /* 0: channel i goes with channel i + channels / 2; otherwise 2 i with 2 i + 1; i-th angle */
} paged_rotation_t;

/*
 * paged_append with K turned on the way, and q (device, desc->dtype, [num_tokens, heads, head_dim], or NULL) into q_out (the same shape; q itself
 * or no part of it).  The token at true position t (seen[b] - t_new + j; seen = NULL: its slot) has angles table[t]:
 *   y_i = x_i cos - x_i' sin        y_i' = x_i sin + x_i' cos        in fp32, rounded once; channels past rotation->channels stay
 * Where the table has no position t the turned channels become NaN.  A row of q is turned also where its row of K is dropped; rows of
 * tokens of no sequence are left alone.
 * Calls of 2^26 waves or more are refused with SPAN_ERR_SHAPE.  A token takes one for each started 12 KiB of its rows of K, V and q (paged_append_fp4: 4 KiB; 2 KiB in both
 * where num_tokens is below 512; paged_read_fp4: 4 KiB of K and V), num_tokens is rounded up to four (4-bit calls from 512 tokens on: eight).  With 8 KV heads and 32 query
 * heads of 128, 16 bits, that is some 67 million tokens, in 4 bits 22 million.
 */
int paged_append_rotary(const span_paged_desc_t* desc, const paged_rotation_t* rotation, const void* k_new, const void* v_new, void* k_pages,
                        void* v_pages, const int32_t* block_table, const int32_t* ctx_lens, const int32_t* q_offsets, int32_t* positions,
                        const int32_t* seen, const void* q, void* q_out);

/*
 * ---- a cache held in 4 bits -------------------------------------------------------------------------------
 * The pools are uint8 [num_pages, kv_heads, page_size, head_dim / 2 + head_dim / 32]; desc->dtype is the type of the new rows, q and rows read back.
 * A block of 32 channels of a row has an exponent e, the least from -126 on with max |x| <= 7 * 2^e, and its values are held as 2^e times the nearest
 * of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives (of two equally near the one with an even number; 7 counts as nearest to 6).  A block with a value that is not finite,
 * or larger than 7 * 2^125, is NaN.
 * A (page, KV head) holds page_size * head_dim / 2 bytes of codes, then page_size * head_dim / 32 of exponents (e + 127; 255: NaN).  Code: sign bit 8 and number of the value in the list;
 * of two codes in a byte the lower channel's is the lower half.  r = row % 16 of group row / 16, c = channel:
 *   K codes   byte  group * 8 head_dim + (c / 32) * 256 + r * 16 + c % 32 / 2
 *   V codes   byte  group * 8 head_dim + (r / 4) * 2 head_dim + c / w * 2 w + (r % 4) * w / 2 + c % w / 2,     w = head_dim / 16
 *   exponents byte  group * head_dim / 2 + (c / 32) * 16 + r
 */

/* paged_append into such pools, K (and q) turned on the way as by paged_append_rotary if rotation is not NULL.  K is turned in 64 bits and rounded once.  Without
 * rotation rows of q go into q_out as they are. */
int paged_append_fp4(const span_paged_desc_t* desc, const paged_rotation_t* rotation, const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                     const int32_t* block_table, const int32_t* ctx_lens, const int32_t* q_offsets, const int32_t* seen, const void* q, void* q_out);

/* The rows that paged_append_fp4 with these lengths and offsets wrote, as values: k_rows, v_rows device, desc->dtype, [num_tokens, kv_heads, head_dim].  Rows that
 * have no place in the cache are left as they are.  (With q_offsets over whole sequences: a cache as paged_append takes it, for paged_prompt_attn.  A value that
 * fp16 does not hold becomes infinite there.) */
int paged_read_fp4(const span_paged_desc_t* desc, const void* k_pages, const void* v_pages, const int32_t* block_table, const int32_t* ctx_lens,
                   const int32_t* q_offsets, void* k_rows, void* v_rows);

/*
 * Attention of one new token per sequence (its row already appended) over S_b, the positions
 *   max(0, n - window) <= p < n  (all p < n for window 0)  and  p < min(sinks, n),      n = ctx_lens[b],
 * that the table has a row for:
 *   s_j = scale * q[b, i, :] . K[b, i / group, j, :]       out[b, i, :] = sum_j softmax_j(s)_j V[b, i / group, j, :]
 *   q   : device, desc->dtype, [batch, heads, head_dim]      out : device fp32 [batch, heads, head_dim]
 *   weights : device or NULL; if given, weights[b, h, j] += sum over the query heads of KV head h of softmax_j, j in S_b
 *             (what paged_evict goes by); other entries are left as they are
 * A sequence without positions gets rows of zeros.  An attended row whose score is NaN or +Inf makes its output rows NaN;
 * an attended V row that is not finite makes them NaN or infinite.  Rows outside S_b have no influence, whatever they hold.
 */
int paged_decode_attn(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages,
                      const int32_t* block_table, const int32_t* ctx_lens, float scale, float* weights, float* out);

/*
 * The same over each sequence's span (span_decode_attn over pages): intervals span_offsets[b] .. span_offsets[b+1] - 1,
 * interval i covers positions [span_starts[i], span_ends[i]), pairwise disjoint.  On a list that would not pass
 * span_validate the result is unspecified, yet no memory outside the pool is touched.
 */
int paged_span_decode_attn(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages,
                           const int32_t* block_table, const int32_t* span_offsets, const int32_t* span_starts,
                           const int32_t* span_ends, float scale, float* weights, float* out);

/* Both over a cache held in 4 bits, without weights. */
int paged_decode_attn_fp4(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                          const int32_t* ctx_lens, float scale, float* out);
int paged_span_decode_attn_fp4(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                               const int32_t* span_offsets, const int32_t* span_starts, const int32_t* span_ends, float scale, float* out);

/*
 * Which pages of a sequence a token's queries may find most in, for every KV head by itself.  bounds holds the least and the largest value of every channel
 * over a page's rows of K; a page's score is an upper bound of what the group's queries can score with one of its rows, added up over them:
 *   score_j = sum over d of  max_part_d * hi[j, d] + min_part_d * lo[j, d]     max_part_d = sum over the group of max(q_d, 0), min_part_d of min(q_d, 0)
 * in 64 bits, rounded to 32.  Listed are the pages of the first desc->sinks and of the last max(desc->recent, 1) positions and those that score highest of the
 * others, desc->budget at most, all where there are no more; of equal scores the lower page, NaN ahead of any number, a page outside the pool with a score
 * of minus infinity.  What the protected positions can lie on has to fit: ceil(sinks / page_size) + floor((max(recent, 1) + page_size - 2) / page_size) + 1 <= budget.
 *   q        : device, desc->dtype, [batch, heads, head_dim], turned as K is
 *   bounds   : device, desc->dtype, [num_pages, kv_heads, 2, head_dim] (least, largest): read, and written where rows are new
 *   since    : device int32 [batch] or NULL (ctx_lens - 1): positions from here on are new.  The bounds of their pages are made on the way, from the new rows and,
 *              where a page begins ahead of since[b], what its bounds are already.  0 after a prompt, or after rows moved
 *   selected : device int32 [batch, kv_heads, budget]: page numbers within the sequence (columns of block_table), ascending, then -1
 * Pages written to must belong to one sequence only.  A NaN in a new row makes its page's bounds NaN.
 */
int paged_select(const span_paged_desc_t* desc, const void* q, const void* k_pages, void* bounds, const int32_t* block_table, const int32_t* ctx_lens,
                 const int32_t* since, int32_t* selected);

/*
 * paged_decode_attn over the listed pages: S of (b, KV head) is the positions p < ctx_lens[b] on pages selected[b, h, i], i < desc->budget.  Entries outside
 * [0, table_pages) attend nothing; of a sequence of c pages the first min(c, budget) entries are looked at, which should differ from one another (a
 * page listed twice counts twice).
 */
int paged_selected_decode_attn(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                               const int32_t* ctx_lens, const int32_t* selected, float scale, float* out);

/*
 * Attention of all new tokens of every sequence (their rows already appended): a prompt, or a chunk of one behind a cached
 * beginning.  The token at position p sees the positions j <= p with j > p - window (all for window 0) or j < sinks.
 *   q   : device, desc->dtype, [num_tokens, heads, head_dim]
 *   out : device, desc->dtype, [num_tokens, heads, head_dim]: it goes on as an activation, in the type those have
 * Scores, maxima and sums are fp32; a weight of a 16-bit call is rounded to the storage type before it meets V, as the
 * output is after it.  A token that sees nothing (more new tokens than positions) gets a row of zeros.
 * A call is refused (SPAN_ERR_SHAPE) where num_tokens / T + min(batch, num_tokens) passes 65535, T = floor(128 / (heads / kv_heads)): with
 * one query head per KV head 8 million tokens, with 16 524000.
 */
int paged_prompt_attn(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages,
                      const int32_t* block_table, const int32_t* ctx_lens, const int32_t* q_offsets, float scale, void* out);

/*
 * Cuts every cache of more than desc->budget rows down to it, for every KV head by itself.  The rows that stay are those of
 * the first `sinks` positions, of the last `recent` (up to the largest position held), and of the others those with the
 * largest weights; of equal weights the lower slot stays, and a NaN weight counts as less than any other.  sinks + recent
 * <= budget.  Weights are gathered by the one-token calls only: right behind a prompt they are still what they were before it, and of equal
 * ones the first positions stay.
 * The i-th kept row in a slot from `budget` on moves to the i-th slot below it that falls free, both in ascending order, so
 * no other row is touched; the pages past the budget are the caller's again when the call's work is done.  Attention does not
 * depend on the order of the rows, but a window or a span over the slots means nothing afterwards.
 *   positions       : device or NULL: slot i holds position i
 *   weights_out, positions_out (the latter NULL if positions is): what the slots below ctx_lens[b] hold afterwards, weight 0
 *                     and position -1 in those that fell free; may be the arrays themselves
 *   new_lens        : device int32 [batch]: min(ctx_lens[b], table_pages * page_size, budget); may be ctx_lens itself
 * Pages of a sequence must differ from one another and belong to it alone.
 */
int paged_evict(const span_paged_desc_t* desc, void* k_pages, void* v_pages, const int32_t* block_table,
                const int32_t* ctx_lens, const float* weights, const int32_t* positions, float* weights_out,
                int32_t* positions_out, int32_t* new_lens);

#ifdef __cplusplus
}
#endif
#endif /* SPAN_PAGED_H_ */
