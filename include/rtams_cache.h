/*
 * rtams_cache.h - a paged cache of attention keys and values held in 4 bits, and the attention that reads it: what a
 * program that answers from what an index finds keeps beside the index.  Part of librtams.so; the conventions are those
 * of rtams.h (d_* are device pointers, calls enqueue on the stream given and return, the library owns no device memory,
 * every function returns RTAMS_OK or a negative rtams_status, rtams_last_error() describes a failure).
 *
 * The cache.  A sequence is a row of a page table: its tokens lie in pages of page_tokens tokens, for all layers
 * and heads, taken from a pool that is split into pages when the cache is created.  Everything that says where a token
 * lies - table, lengths, reference counts, free pages - lives in the pool and is changed by kernels, so a step of a
 * serving loop (extend, write and attend for every layer, trim) can be recorded into a HIP graph and launched again.
 * What a call does with pages is a function of the table alone: new pages are the lowest-numbered free ones, in the
 * order of the call's items, whatever came before.
 *
 * The format.  A row of head_dim channels is cut into groups of 32.  NaN becomes 0, channels are clamped to +-60000; with lo and hi the
 * least and largest of the group, step = half((hi - lo) / 15) and zero = half(lo); a channel's code is
 * rint((x - zero) * (1 / step)) clamped to 0..15 (0 where step is 0), in 32 bits, and stands for zero + step * code: 5 bits a channel with
 * step and zero.  Everything the cache holds is finite, so what a mask hides can never reach a result.
 *
 * Items.  A call works on n items.  Item i is the sequence d_seqs[i] (NULL: sequence i) and the rows d_starts[i] ..
 * d_starts[i + 1] - 1 of the call's row arrays (n + 1 ints; NULL: one row each), which stand for the LAST rows of the
 * sequence: row j of c is position length - c + j.  No sequence may be named twice in one call that changes something.
 * Both arrays are read on the device when the call runs.
 *
 * What only the device can see.  A call whose items are not what it asks for (a sequence outside 0..max_seqs - 1 or named
 * twice, more rows than max_new or than the sequence has, ...) raises EINVAL and a call that finds too few free pages
 * EPOOL, to be asked for with rtams_cache_poll_error; calls that change the table are then dropped as a whole, other
 * calls leave the item's rows as they are.  (Attention that is not causal asks for no positions: an item may have any
 * number of rows.)  After an extend that was dropped, writes are dropped too until an extend succeeds or
 * rtams_cache_clear_error is called.
 *
 * Devices.  A cache is its pool's device's, and so are the streams of its calls (NULL: that device's default stream), whichever device is the thread's
 * current one.
 *
 * Streams.  The calls of one cache run one after another; a call on another stream than the one before is ordered behind
 * it with an event.  A stream must live until the cache has been used on another one or destroyed.  Recorded calls
 * (stream capture) are ordered by their graph alone: the caller orders its launches with other calls.
 */
#ifndef RTAMS_CACHE_H
#define RTAMS_CACHE_H

#include "rtams.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct rtams_cache rtams_cache; /* opaque, host side */

enum rtams_type { RTAMS_TYPE_BF16 = 0, RTAMS_TYPE_F16 = 1, RTAMS_TYPE_F32 = 2 /* rtams_cache_read only */ };

typedef struct rtams_cache_config {
  int32_t layers;
  int32_t kv_heads;
  int32_t head_dim;    /* 64, 96, 128 or 256 */
  int32_t page_tokens; /* a multiple of 32, at most 1024 */
  int32_t max_seqs;    /* rows of the page table, at most 65536 */
  int32_t max_pages;   /* pages of one sequence; max_pages * page_tokens below 2^30 */
  void *d_pool;        /* device memory, 256-byte aligned: tables, then pages */
  size_t pool_bytes;
  void *d_scratch;     /* device memory, 256-byte aligned: parts of rows that several workgroups share */
  size_t scratch_bytes;
} rtams_cache_config;

/* Where things lie in the pool; all device memory, ordered like any other by the stream. */
typedef struct rtams_cache_view {
  int32_t *d_table;    /* [max_seqs][max_pages], -1 behind a sequence's last page */
  int32_t *d_lengths;  /* [max_seqs] tokens */
  int32_t *d_refs;     /* [pages] table entries that name the page; 0: free */
  void *d_pages;       /* [layers][pages][page_bytes]; opaque, but a page is moved as it is */
  int64_t pages;
  int64_t page_bytes;  /* of one layer: 1.25 * page_tokens * kv_heads * head_dim */
} rtams_cache_view;

/* Bytes of pool that `pages` pages take under this configuration (d_* ignored), and of scratch.  0 on bad arguments. */
size_t rtams_cache_pool_bytes_for(const rtams_cache_config *cfg, int64_t pages);
size_t rtams_cache_scratch_bytes_for(const rtams_cache_config *cfg);

/* Lays out and clears the pool (every sequence empty, every page free).  Synchronous. */
int rtams_cache_create(const rtams_cache_config *cfg, rtams_cache **out);
/* Waits for the cache's work and releases host resources; the device memory stays the caller's. */
int rtams_cache_destroy(rtams_cache *c);
int rtams_cache_layout(const rtams_cache *c, rtams_cache_view *out);

/* Room for the items' rows at the ends of their sequences.  A last page that is part full and shared with another
 * sequence is first replaced by a copy (all layers).  EPOOL, and nothing changed, where too few pages are free. */
int rtams_cache_extend(rtams_cache *c, int64_t n, const int32_t *d_seqs, const int32_t *d_starts, void *hip_stream);

/* One layer's keys and values of the items' rows: d_k and d_v [rows][kv_heads][head_dim] of `type` (BF16 or F16), rows and
 * heads `row_stride` and `head_stride` elements apart (below 2^24 and 2^40; of a single row or head it says nothing), channels
 * next to each other.  max_new: the most rows of one item.  The items of a sequence that is named twice are left out, with EINVAL.
 * Rows whose page another sequence shares are left out, with EINVAL: extend sees to it that new rows' pages are not. */
int rtams_cache_write(rtams_cache *c, int32_t layer, int64_t n, const int32_t *d_seqs, const int32_t *d_starts,
                      int64_t rows, int32_t max_new, const void *d_k, const void *d_v, int64_t row_stride,
                      int64_t head_stride, int32_t type, void *hip_stream);

/* The reverse: the values that the cache holds for the items' rows, [rows][kv_heads][head_dim] without gaps. */
int rtams_cache_read(rtams_cache *c, int32_t layer, int64_t n, const int32_t *d_seqs, const int32_t *d_starts,
                     int64_t rows, int32_t max_new, void *d_k, void *d_v, int32_t type, void *hip_stream);

typedef struct rtams_cache_query {
  int32_t layer;
  int32_t q_heads;     /* a multiple of kv_heads; head h reads kv head h / (q_heads / kv_heads) */
  int32_t type;        /* of q and out: BF16 or F16 */
  int32_t causal;      /* 1: a row sees the positions up to its own; 0: all of its sequence */
  int32_t window;      /* causal only: ... and of those the last `window`; 0: all */
  int32_t max_new;     /* the most rows of one item */
  float scale;         /* of the scores, before the softmax */
  const void *d_q;     /* [rows][q_heads][head_dim], strides in elements, channels next to each other */
  int64_t q_row_stride, q_head_stride;
  void *d_out;
  int64_t out_row_stride, out_head_stride;
  float *d_lse;        /* [rows][q_heads] logarithm of the sum of exp(score), or NULL */
} rtams_cache_query;

/* Attention of the items' rows over one layer.  Scores, their maximum, sum and the weighted values are held in 32 bits; the
 * products take halves: keys and values rounded once, queries times a power of two, and probabilities, of which a row's largest
 * stands at 2^7 to 2^15, so that one 2^-32 of it may be lost.  A row that sees nothing gives 0 and a logarithm of -inf; a row of
 * q that holds a NaN, an infinity or, times the scale, a number beyond the halves spoils its own output only.
 * Of more than 64 rows of a head, work is laid out by the longest item: n * kv_heads * (its rows of a head / 128 + 1) has to be
 * below 2^28, and what is laid out for shorter items in vain takes some 10 ns for each 256 rows. */
int rtams_cache_attend(rtams_cache *c, const rtams_cache_query *q, int64_t n, const int32_t *d_seqs,
                       const int32_t *d_starts, int64_t rows, void *hip_stream);

/* What rows see besides what a query says.  All zero: nothing else. */
typedef struct rtams_cache_sight {
  int32_t sinks;          /* with a window: the sequence's first `sinks` positions stay visible (up to a row's own) */
  int32_t tree_words;     /* words of a row of d_tree: a bit for each of max_new rows, at most 32 words */
  const uint32_t *d_tree; /* [rows][tree_words]: bit i of row j's words: it sees row i of its item.  NULL: the rows up to itself */
} rtams_cache_sight;

/* rtams_cache_attend with a sight (NULL: none).  With a tree, which is causal, the items' rows stand side by side in the cache, but each sees of
 * them those that its bits name, whatever their order, and what lies before the item's first row.  Its own position, from which a window
 * counts, is the one behind as many rows as its bits name: base + bits - 1, base being that of the item's first row; rows that it names it sees whatever the window.
 * (A tree that is a chain is what no tree is, while the window has room for the chain.)  Bits beyond the item's rows say nothing. */
int rtams_cache_attend_sight(rtams_cache *c, const rtams_cache_query *q, const rtams_cache_sight *sight, int64_t n,
                             const int32_t *d_seqs, const int32_t *d_starts, int64_t rows, void *hip_stream);

/* Trees of drafted tokens.  An item's rows are the nodes of a tree, at most 1024 of them: d_parents[row] is the number, within the item, of the row
 * that a row follows, which is lower than its own, or -1.  An item of which that does not hold raises EINVAL.
 *
 * What each row sees: d_tree as rtams_cache_sight takes it, its ancestors and itself, and d_positions (NULL: not asked for) the position in the
 * sequence that it would have if its path were all there is: rows of the same depth stand at the same one. */
int rtams_cache_tree(rtams_cache *c, int64_t n, const int32_t *d_seqs, const int32_t *d_starts, int64_t rows, int32_t max_new,
                     const int32_t *d_parents, uint32_t *d_tree, int32_t tree_words, int32_t *d_positions, void *hip_stream);

/* The path that a model's choices follow.  d_tokens[row] is the token of a row, d_chosen[row] the one that was chosen behind it.  The path begins at the
 * item's row 0 and goes on to the first row whose parent is the path's last and whose token, not negative, was chosen there.  d_path [rows]: the rows'
 * numbers within the item, then -1; d_kept [n]: how many; d_next [n]: the token chosen behind the last.  Items without rows have 0 and -1,
 * items that raise EINVAL -1 and -1.  (The cache's own state is not read.) */
int rtams_cache_walk(rtams_cache *c, int64_t n, const int32_t *d_starts, int64_t rows, int32_t max_new, const int32_t *d_parents,
                     const int32_t *d_tokens, const int32_t *d_chosen, int32_t *d_path, int32_t *d_kept, int32_t *d_next, void *hip_stream);

/* Of each item's rows the d_kept[i] that the first entries of its d_path name, in ascending order, move to the front, in all layers, and the sequence is cut
 * behind them; pages that nothing lies in any more are free.  A call that changes the table: dropped as a whole where an item is not what it asks for or would write into a
 * page that another sequence shares (EINVAL), and after an extend that was dropped. */
int rtams_cache_keep(rtams_cache *c, int64_t n, const int32_t *d_seqs, const int32_t *d_starts, int64_t rows, int32_t max_new,
                     const int32_t *d_path, const int32_t *d_kept, void *hip_stream);

/* Sequence d_dst[i], which is empty, becomes what d_src[i] is: naming the same pages, or (copy != 0) pages of its own with
 * the same contents.  A source may be named several times, a destination once and not as a source. */
int rtams_cache_fork(rtams_cache *c, int64_t n, const int32_t *d_src, const int32_t *d_dst, int32_t copy,
                     void *hip_stream);
/* Cuts sequences down to d_lengths[i] tokens (NULL: none); pages that no sequence names any more are free. */
int rtams_cache_trim(rtams_cache *c, int64_t n, const int32_t *d_seqs, const int32_t *d_lengths, void *hip_stream);
/* Moves the pages in use to the front of the pool: with u of them, the i-th lowest free page below u takes the i-th lowest used
 * page from u on.  What lies behind page u - 1 is then free. */
int rtams_cache_compact(rtams_cache *c, void *hip_stream);

/* Free pages, after waiting for the cache's work. */
int rtams_cache_free_pages(rtams_cache *c, int64_t *out);
/* The first error that a kernel raised since the last clear; RTAMS_OK if none.  Does not wait. */
int rtams_cache_poll_error(rtams_cache *c);
/* Waits for the cache's work and forgets it. */
int rtams_cache_clear_error(rtams_cache *c);

#ifdef __cplusplus
}
#endif
#endif /* RTAMS_CACHE_H */
