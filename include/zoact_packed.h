/*
 * zoact_packed.h -- batches whose sequences differ in length (gfx950): the forward's
 * operations over rows packed one sequence behind the other, and the selection of a
 * beam search.
 *
 * Fine-tuning text comes in sequences of many lengths.  Packed, a batch has no rows but
 * the sequences' own: the linears, norms and projections of zoact.h take its rows as they
 * are; the calls here are those that have to know where a sequence begins: rotary
 * positions, attention and the next-token loss.  They stand beside zoact_rope,
 * zoact_attention, zoact_xent_pm and zoact_linear_xent_pair, which take sequences of one
 * length.
 *
 * Conventions are those of zoact.h: device pointers unless a comment says "host",
 * caller-owned buffers, host-side validation before any enqueue, stream-ordered, no
 * allocation; every call can be captured into a graph.
 *
 * Packed sequences.  Sequence i is the rows [begin[i], begin[i + 1]) (none if equal);
 * begin ascends from 0 or more to `rows` or less.  Rows that belong to no sequence do not
 * matter and are not written.  Where begin does not ascend or leaves [0, rows], rows of any
 * sequence may stay unwritten; no other memory is touched.
 */
#ifndef ZOACT_PACKED_H
#define ZOACT_PACKED_H

#include "zoact.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  const int32_t* begin; /* [n + 1]                                                     */
  int32_t n;            /* sequences, 1 .. 2^24                                        */
  int64_t rows;         /* rows of the tensors, 0 .. 2^31 - 1024                       */
} zoact_packed;

/* Causal attention within each sequence: for rows t of sequence i and heads h,
 *   out[t][h] = sum_s softmax_s(scale q[t][h] . k[s][g]) v[s][g],  begin[i] <= s <= t,
 * g = h / (n_heads / n_kv_heads).  q [rows][ldq], k [rows][ldk], v [rows][ldv] hold their
 * heads from column 0 (they may be column slices of one buffer), out [rows][n_heads *
 * head_dim], all in dtype (F32 or BF16); out must not overlap them.  head_dim 1 .. 256.
 * Scores, softmax and sums fp32; with BF16 a probability, relative to the largest so far
 * of its row or to one within a factor 2^8 of it, is rounded to bf16 as it enters the
 * product with v (the normaliser sums it unrounded); one rounding of out.  What a row may
 * not attend to does not reach it, whatever it holds.  A head_dim up to 128 of whole
 * 16-byte pieces runs on the matrix cores if rows are 16-byte aligned (as the next of 32,
 * 64 and 128); others run one wave a row and head. */
zoact_status zoact_attention_packed(const zoact_packed* s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                    const void* v, int64_t ldv, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                    float scale, int32_t dtype, void* out, zoact_stream stream);

/* Rotary positions of rows whose token indexes are given: for each of n_heads heads of
 * head_dim columns (from column 0) of x [rows][ldx], the first rot_dim values are turned
 * in pairs (a, b) -> (a c - b s, b c + a s), c, s = cos_t, sin_t[p][j], j < rot_dim / 2,
 * p = pos[row] clamped to [0, n_pos - 1] (pos NULL: the row's index); the others are
 * copied.  Pair j is (x[j], x[j + rot_dim / 2]) with ZOACT_ROPE_HALF and
 * (x[2 j], x[2 j + 1]) with ZOACT_ROPE_INTERLEAVED.  x and out [rows][ldo] in dtype, out
 * may be x itself (ldo == ldx) and must not overlap it otherwise; tables fp32
 * [n_pos][rot_dim / 2].  fp32 arithmetic, one rounding of out.  1 <= rot_dim / 2,
 * rot_dim even and at most head_dim, n_heads * head_dim < 2^31; tables and pos 4-byte
 * aligned, x and out to their type. */
enum { ZOACT_ROPE_HALF = 0, ZOACT_ROPE_INTERLEAVED = 1 };
zoact_status zoact_rope_at(const void* x, int64_t ldx, void* out, int64_t ldo, int32_t dtype, int64_t rows,
                           int32_t n_heads, int32_t head_dim, int32_t rot_dim, int32_t layout, const int32_t* pos,
                           const float* cos_t, const float* sin_t, int64_t n_pos, zoact_stream stream);

/* Next-token cross entropy of both halves over packed rows: loss_pm[h] = mean, over the
 * rows t whose next row is of the same sequence, of -log softmax(logits[h][t])[tokens[t +
 * 1]] (ids clamped to the vocabulary).  A batch without such a row has no mean: NaN.
 * zoact_xent_packed: from logits fp32 [2][rows][V], 4-byte aligned; ws of
 * zoact_loss_workspace_bytes().
 * zoact_linear_xent_packed: fused with the head's product as zoact_linear_xent_pair is
 * (rows T = s->rows >= 1 in place of B * S; its requirements, workspace and errors).
 * Sums of fp32 values in fp64, in a fixed order. */
zoact_status zoact_xent_packed(const float* logits, const int32_t* tokens, const zoact_packed* s, int64_t V,
                               float* loss_pm, void* ws, size_t ws_bytes, zoact_stream stream);
zoact_status zoact_linear_xent_packed(const zoact_linear* L, const zoact_arena* A, const void* x, const zoact_packed* s,
                                      const void* p, const zoact_pert_pair* pp, const int32_t* tokens, float* loss_pm,
                                      void* ws, size_t ws_bytes, zoact_stream stream);

/* One step of a beam search over n prompts.  Prompt i holds beams_in candidates with their
 * summed log probabilities score[i][b] and the tokens hist[i][b][0 .. length - 1]; row
 * i * beams_in + b of logits is the model's over the token that follows.  Candidate (b, v)
 * has the value
 *   score[i][b] + logits[b][v] - log sum_u exp(logits[b][u])
 * or, where b has ended (eos >= 0, length > 0 and its last token is eos), score[i][b] for
 * v = eos and -inf for every other v.  The `beams` largest of a prompt's are kept, largest
 * first, of equal ones the lowest (b, v) first; NaN counts as largest.  Finite values of one
 * beam are in the order of their logits, also where fp64 does not resolve it.  A row whose log sum
 * is not finite (a NaN or +inf among its logits, or nothing but -inf) gives NaN, and so
 * does a score of NaN or +inf.  Kept candidate m of prompt i:
 *   score_out[i][m] its value, token[i][m] = v, src[i][m] = i * beams + b (where beam b's
 *   sequence lives, for zoact_cache_fork, if beams_in <= beams), hist_out[i][m] = hist[i][b], then v.
 * Values are compared in fp64 from fp32 sums and rounded once.  logits [n * beams_in][ldl]
 * in dtype (F32 or BF16, aligned to its type), score, score_out fp32, hist
 * [n][beams_in][ld_hist], hist_out [n][beams][ld_hist_out], token, src int32 [n * beams]
 * (token and src may be NULL); 0 <= length <= ld_hist, length < ld_hist_out.  Outputs must
 * not overlap inputs.  1 <= beams_in, beams <= ZOACT_BEAMS_MAX, beams <= vocab <= 2^30,
 * n * beams_in <= 65535, length < 2^31.  ws: zoact_beam_workspace_bytes() bytes, 16-byte aligned. */
enum { ZOACT_BEAMS_MAX = 64 };
typedef struct {
  int32_t n;
  int32_t beams_in;
  int32_t beams;
  int32_t eos;           /* -1: no candidate ends */
  int64_t vocab;
  int64_t length;
  const float* score;    /* [n][beams_in]             */
  const int32_t* hist;   /* NULL allowed if length == 0 */
  int64_t ld_hist;
  float* score_out;      /* [n][beams]                */
  int32_t* hist_out;
  int64_t ld_hist_out;
  int32_t* token;        /* [n][beams] or NULL        */
  int32_t* src;          /* [n][beams] or NULL        */
} zoact_beams;
size_t zoact_beam_workspace_bytes(int32_t n, int32_t beams_in, int32_t beams, int64_t vocab);
zoact_status zoact_beam_select(const zoact_beams* b, const void* logits, int64_t ldl, int32_t dtype, void* ws,
                               size_t ws_bytes, zoact_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* ZOACT_PACKED_H */
