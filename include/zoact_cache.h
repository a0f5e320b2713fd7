/*
 * zoact_cache.h -- answering with the fine-tuned model (gfx950): a paged key/value
 * cache held in 8 bits, the attention that reads it, and the operations on its pages.
 *
 * The fine-tuned model of zoact.h is evaluated token by token: C is final, nothing is
 * perturbed, and each step multiplies a few rows (zoact_linear_rows in zoact.h), adds
 * their keys and values to a cache and attends over it.
 *
 * Conventions are those of zoact.h: device pointers unless a comment says "host",
 * caller-owned buffers, host-side validation before any enqueue, stream-ordered, no
 * allocation; every call can be captured into a graph.  Calls that change one cache, or
 * that share a workspace, must be ordered by the caller (one stream, or events).
 *
 * Cache.  A page holds the keys and values of ZOACT_CACHE_PAGE = 64 consecutive tokens of
 * one sequence, for every layer and key/value head.  They are int8 codes with one fp32
 * scale for each block of ZOACT_CACHE_BLOCK = 16 tokens and head (keys and values apart):
 * the value is scale * code, codes in [-127, 127].
 *   k        int8 [n_layers][n_pages][n_kv_heads][64][head_dim]
 *   v        int8 [n_layers][n_pages][n_kv_heads][head_dim][64], token 16 n + 4 g + i of
 *            the page (n, g, i < 4) at position 16 g + 4 n + i
 *   k_scale, v_scale  fp32 [n_layers][n_pages][n_kv_heads][4]
 * A sequence lives in a slot: len[slot] tokens on the pages table[slot][0 ..
 * ceil(len / 64) - 1] (entries past them mean nothing).  Several slots may hold one page;
 * refs[page] counts its holders, 0 = free.  The caller zeroes len and refs once; after
 * that the calls below keep all three, and a page that two slots hold is copied before
 * one of them writes to it.
 *
 * Batch.  The calls of one step share a batch of n entries: entry i is the new rows
 * [row_begin[i], row_begin[i + 1]) of slot slots[i] (row_begin NULL: max_new rows each,
 * row i * max_new on; slots NULL: slot i).  zoact_cache_extend reserves their places and
 * writes pos[i], the token index of entry i's first row; zoact_cache_append and
 * zoact_attention_cache of every layer read it.  An entry that a call cannot serve -- a
 * slot outside the cache or (extend) named before in the batch, rows outside [0, rows) or
 * more than max_new, places past the table, a page number outside the cache -- is left out
 * and ORs a bit into *status (nullable): extend gives it pos -1, append writes nothing for
 * it, attention writes zeros to its rows where their range is one.  pos[i] < 0 is left
 * out without a bit.  Rows that belong to no entry stay as they were; a batch of no rows at
 * all is served (its q, k, v and out may be NULL).  Outputs must not overlap inputs.
 */
#ifndef ZOACT_CACHE_H
#define ZOACT_CACHE_H

#include "zoact.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { ZOACT_CACHE_PAGE = 64, ZOACT_CACHE_BLOCK = 16, ZOACT_CACHE_MAX_BATCH = 1024 };

/* Bits of a device status word (bit 0 is the update's, see zoact_step). */
enum {
  ZOACT_STATUS_BAD_ENTRY = 2, /* an entry or a page number that does not fit the cache */
  ZOACT_STATUS_NO_PAGES = 4   /* extend: not enough free pages, nobody was served       */
};

typedef struct {
  int8_t* k;
  int8_t* v;
  float* k_scale;
  float* v_scale;
  int32_t* table;      /* [n_slots][max_pages]                                    */
  int32_t* len;        /* [n_slots]                                               */
  int32_t* refs;       /* [n_pages]                                               */
  int64_t n_pages;     /* below 2^31                                              */
  int32_t n_layers;
  int32_t n_kv_heads;
  int32_t head_dim;    /* 32, 64 or 128                                           */
  int32_t n_slots;
  int32_t max_pages;   /* pages a slot can hold; max_pages * 64 below 2^31        */
} zoact_cache;

typedef struct {
  int32_t n;                /* entries, 1 .. ZOACT_CACHE_MAX_BATCH                */
  int32_t max_new;          /* most rows of an entry, >= 1                        */
  int64_t rows;             /* rows of q, k, v and out                            */
  const int32_t* slots;     /* [n] or NULL                                        */
  const int32_t* row_begin; /* [n + 1] or NULL                                    */
  int32_t* pos;             /* [n]                                                */
  uint32_t* status;         /* [1] or NULL                                        */
} zoact_cache_batch;

/* Workspace of extend, fork and compact for this cache. */
size_t zoact_cache_workspace_bytes(const zoact_cache* c);

/* Reserves places for every entry's rows: pos[i] = len[slot], len[slot] += rows of entry
 * i, and pages for them.  Entries are served in order; each takes free pages, lowest
 * number first: one in place of its last page if that is partly full and another slot
 * still holds it (all layers are copied; refs of the old page falls by one), then those
 * its new tokens start.  An entry without rows is served (pos = len).  Too few free pages
 * for all: nothing changes, every pos is -1 and ZOACT_STATUS_NO_PAGES is set. */
zoact_status zoact_cache_extend(const zoact_cache* c, const zoact_cache_batch* b, void* ws, size_t ws_bytes,
                                zoact_stream stream);

/* Each dst[i] becomes a second holder of src[i]'s tokens and pages; what it held before
 * goes back.  All sources are read before any destination changes, so entries may
 * permute slots (a beam search's survivors).  A source may be named often; of equal
 * destinations the first counts, the others set ZOACT_STATUS_BAD_ENTRY.  src, dst [n],
 * n in 1 .. n_slots. */
zoact_status zoact_cache_fork(const zoact_cache* c, const int32_t* src, const int32_t* dst, int32_t n, void* ws,
                              size_t ws_bytes, uint32_t* status, zoact_stream stream);

/* Gives the pages of the slots back and empties them (a slot named twice is emptied once).
 * slots [n], n in 1 .. n_slots. */
zoact_status zoact_cache_free(const zoact_cache* c, const int32_t* slots, int32_t n, uint32_t* status,
                              zoact_stream stream);

/* Moves the pages together: with U pages in use, the k-th used page numbered U or more
 * moves (all layers) to the k-th free page below U, and tables and counts follow.  After
 * it pages 0 .. U - 1 are in use; *n_used = U (device, nullable). */
zoact_status zoact_cache_compact(const zoact_cache* c, void* ws, size_t ws_bytes, int32_t* n_used,
                                 zoact_stream stream);

/* Writes the new rows' keys and values into `layer` at the places extend reserved.
 * k [rows][ldk], v [rows][ldv] (n_kv_heads heads of head_dim from column 0) in dtype.  With
 * cos_t, sin_t (fp32 [n_pos][head_dim / 2], both or neither) keys are rotated as
 * zoact_rope does at their token index (clamped to n_pos - 1), in fp32 with one rounding
 * per operation and no rounding of the result.  Per block of 16 tokens and head:
 *   s = max |new values| * (1/127 as fp32), and if earlier tokens are in the block
 *   s = max(s, old scale), their codes becoming rint(code * (old scale / s));
 *   code = rint(value / s), or 0 where s == 0
 * in fp32, ties to even.  A block that gets a value that is not finite has a NaN scale and
 * new codes 0: whoever attends to it gets NaN.  Codes of tokens that the sequence does not
 * have yet stay as they were.  Rows and tables 16-byte aligned: ldk, ldv multiples of 8
 * (BF16) or 4 (F32).  No slot twice in one batch. */
zoact_status zoact_cache_append(const zoact_cache* c, int32_t layer, const void* k, int64_t ldk, const void* v,
                                int64_t ldv, int32_t dtype, const zoact_cache_batch* b, const float* cos_t,
                                const float* sin_t, int64_t n_pos, zoact_stream stream);

/* out[row][h] = sum_t softmax_t(scale * k_t . q[row][h]) v_t over tokens t <= the row's own
 * token index, q [rows][ldq] with n_heads heads (head h reads key/value head h / (n_heads /
 * n_kv_heads)), out [rows][n_heads * head_dim], both in dtype.  With cos_t, sin_t q is
 * rotated first, as append does.  Scores, softmax and sums fp32; in BF16 the rotated q and
 * the probabilities are rounded to 11 bits as they enter the products (an unrotated bf16 q
 * is not changed by this), in F32 to 22 bits or more, a probability times its value scale to
 * no finer than 2^-39 of the largest value scale the row attends to; one rounding of out.
 * max_len (host): a length that no entry's pos + rows is expected to pass; it only shapes
 * the split of the work, longer entries are served too (the split is that of the entry of most
 * rows for all: a single token far behind beside a chunk of rows is slow, 3.5 ms behind 131070
 * tokens where 52 us in a batch of its own).  ws: at least
 * zoact_attention_cache_workspace_bytes() bytes let long sequences be split over
 * workgroups (partial results are joined in a fixed order, the same values on every run);
 * NULL or smaller: not split. */
size_t zoact_attention_cache_workspace_bytes(const zoact_cache* c, const zoact_cache_batch* b, int32_t n_heads,
                                             int64_t max_len);
zoact_status zoact_attention_cache(const zoact_cache* c, int32_t layer, const void* q, int64_t ldq, int32_t dtype,
                                   int32_t n_heads, const zoact_cache_batch* b, float scale, int64_t max_len,
                                   const float* cos_t, const float* sin_t, int64_t n_pos, void* out, void* ws,
                                   size_t ws_bytes, zoact_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* ZOACT_CACHE_H */
