/* Rows that leave the 4-bit paged KV cache (sm_103a): what attention every cached row has had, the choice of those
 * that stay, and their moving together, in place.
 *
 * The paper admits a session only if its whole context fits (section V-D).  A user that is cut to a budget of rows
 * goes on beyond it: the first and the last rows stay, and of the others those that queries have looked at most.
 * Keys keep the rotation of the position that they were appended at, so a row may lie at any slot; new
 * tokens are rotated by their true position (kfl_kv4_append_at).
 *
 * Conventions as in kafila_kv4.h.
 */
#ifndef KAFILA_KV4_EVICT_H
#define KAFILA_KV4_EVICT_H

#include "kafila_kv4.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Attention weight per cached row: device fp32 at data + layer * layer_stride + user * user_stride + head *
 * head_stride + slot (strides in elements; a KV head's slots contiguous, max_pages * page_tokens of them).  Different
 * layers, users and heads do not overlap.  Slots behind a user's length hold 0: new rows start from there
 * (kfl_kv4_keep sees to it; the caller zeroes the buffer first, and a user's slots when kfl_kv4_free ends it).  What
 * kfl_kv4_fork gives a user is weighed anew by nobody: the caller copies the source's slots, all of them, to the
 * destination's (of all pairs at once, as the rows are). */
typedef struct {
  float *data;
  int64_t layer_stride, user_stride, head_stride;
} kfl_kv4_mass;

/* Adds to every cached row of one layer the weight that the query rows of its KV head give it:
 *   mass[user][head][t] += sum over the sequence's tokens i that see t, and the head's query heads j, of
 *                          exp(scale q_ij k_t - lse_ij)
 * q, lse (what kfl_kv4_attend or _attend_tree wrote), users, q_start, n_seqs, n_tokens, max_q, scale, window and
 * workspace as in kfl_kv4_attend: a sequence's tokens are its user's last ones, token i sees the rows up to its own.  A row of
 * q whose lse is -inf (it saw nothing) adds nothing.  n_seqs at most 1024; a user named again is reported
 * (KFL_BAD_USER) and its later sequences are skipped.  Rows on a page out of range are reported and keep what they have.
 * Precision: scores from the exact codes with fp32 sums, weights and their sums in fp32, always in the same order.  The
 * error of a weight grows with the numbers in its exponent: it is within 2^-19 (M + |lse_ij|) + 2^-22 of itself, M =
 * |scale| sum_c (16 s_c + |c_c|) |q_c| with the scales and centres of the key's channels, and a sum of r weights within
 * r 2^-24 of itself more; the mass that it is added to is rounded to fp32.  Measured with normal keys and queries, lse
 * below 12: 1e-7 of 64 bits, up to 1e-6 (2-norm).
 * Errors: KFL_ERR_ARG, KFL_ERR_RANGE (layer, sequences, query rows), KFL_ERR_CUDA. */
int kfl_kv4_weights(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *q, const float *lse,
                    const kfl_kv4_mass *mass, const int32_t *users, const int32_t *q_start, int n_seqs, int n_tokens,
                    int max_q, float scale, int window, void *workspace, size_t workspace_bytes, int32_t *status,
                    void *cuda_stream);

/* The rows that stay of each of n users (device int32 users[n], up to 1024) cut to `budget` rows, for every layer and KV
 * head on its own: of L rows the first `first`, the last `recent`, and of those between the budget - first - recent with
 * the greatest mass (ties to the lowest slot; NaN counts as greater than all numbers); all of them if L <= budget.
 *   rows    device int32 [n_layers][n][n_kv_heads][budget]: slots, ascending; -1 behind the last
 *   counts  device int32 [n]: min(L, budget)
 * A user out of range is reported: its rows are -1, its count 0.  Nothing of the cache changes: kfl_kv4_keep does
 * that.  first + recent at most budget, budget at least 1 and at most 2^26, max_pages * page_tokens at most 2^26.
 * Errors: KFL_ERR_ARG, KFL_ERR_RANGE (more than 1024 users), KFL_ERR_CUDA. */
int kfl_kv4_select(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const kfl_kv4_mass *mass, const int32_t *users,
                   int n, int budget, int first, int recent, int32_t *rows, int32_t *counts, int32_t *status,
                   void *cuda_stream);

/* Slots that stay: device int32 at data + layer * layer_stride + i * seq_stride + head * head_stride + j (strides in
 * elements, 0 where all are alike), j < most. */
typedef struct {
  const int32_t *data;
  int64_t layer_stride, seq_stride, head_stride;
  int most;
} kfl_kv4_rows;

/* Cuts users[i] (device int32 [n], up to 1024) to its rows below first[i] (NULL: 0) and the counts[i] rows of its list,
 * in the list's order: slot first + j gets the row of slot list[j], for every layer and KV head by its own list; mass (NULL:
 * none) moves with the rows and is 0 behind them.  length becomes first + counts; pages behind it are
 * given back.  Moved in place: a list's entry j is at least first + j and below the length (as in every ascending list
 * of different slots); another one is reported (KFL_BAD_POSITION) and its row, and mass, stay what the slot held.
 * Pages that other users hold too are not written: the user gets new ones (free before the call, lowest first) for
 * those that rows move in.  From the first user on that there is no room for, those that need new pages are left as they
 * were (KFL_NO_PAGES), also where the free ones would do for a later one of them.  Left as it was is also one whose
 * first or count is negative, whose count is above `most` or whose rows would be more than its length
 * (KFL_BAD_POSITION), that is named again (KFL_BAD_USER), or with a page out of range (KFL_BAD_PAGE).
 * A user that loses nothing is not touched.  workspace: kfl_kv4_pages_workspace_bytes, its contents of no account.
 * Errors: KFL_ERR_ARG, KFL_ERR_RANGE (more than 1024 users), KFL_ERR_CUDA. */
int kfl_kv4_keep(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const int32_t *users, const kfl_kv4_rows *rows,
                 const int32_t *first, const int32_t *counts, const kfl_kv4_mass *mass, int n, void *workspace,
                 int32_t *status, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* KAFILA_KV4_EVICT_H */
