/* A KV cache in 4 bits, in pages that users share (sm_103a): what writes it, the attention that reads it, and
 * the copying, forking, compacting and freeing of its pages.
 *
 * The paper reserves the cache of every declared user at the declared context (section V-C, lim(i)) and admits
 * a session only if that fits (section V-D).  Pages of 4-bit rows hold the same tokens in 0.28 of the bf16
 * bytes, and only as many as there are tokens; users that go on from a common prompt hold its pages together.
 *
 * The caller owns every buffer (pool, tables, workspaces); the calls allocate nothing, wait for nothing and
 * can be captured.  Calls on one pool are ordered by the caller's stream or events.
 *
 * A cached row (one token, one KV head) is coded in groups of 64 channels.  With lo, hi the group's ends:
 *   scale = fp16((hi - lo) / 15), centre = fp16(lo + 8 scale)
 *   code = clamp(rint((x - centre) / scale) + 8, 0, 15)      (8 if scale is 0)
 *   value = centre + (code - 8) scale
 * (1 / scale is rounded to fp32 first.)  The error of a value is at most half a step beside the rounding
 * of scale and centre to fp16.  A group with a value that is not finite or larger than 32768 in magnitude
 * reads as NaN throughout: scale and centre are stored as NaN.
 *
 * Conventions as in kafila_stage.h; types, rows of heads and the status word as in kafila_rope.h.
 */
#ifndef KAFILA_KV4_H
#define KAFILA_KV4_H

#include <stddef.h>
#include <stdint.h>

#include "kafila_rope.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The pool: device memory [n_pages][n_layers][n_kv_heads] of blocks, 16-byte aligned.  A block holds
 * page_tokens tokens of one head of one layer, page_tokens * head_dim * 9 / 8 bytes:
 *   K codes [token][head_dim / 2] bytes (channel 2 j in the low half of byte j, 2 j + 1 in the high half),
 *   V codes the same, K parameters [token][head_dim / 64] pairs of fp16 (scale, centre), V parameters.
 * page_tokens 16, 32, 64 or 128; head_dim 64 or 128; n_kv_heads up to 256; n_pages up to 2^20. */
typedef struct {
  void *pages;
  int n_pages, page_tokens, n_layers, n_kv_heads, head_dim;
} kfl_kv4_pool;

/* Who holds which pages (device int32, all layers alike):
 *   table   [n_users][max_pages]: user u's pages in order of position, -1 behind the last
 *   lengths [n_users]: cached tokens; a user holds ceil(length / page_tokens) pages
 *   refs    [n_pages]: how many users hold the page, 0 for a free one */
typedef struct {
  int32_t *table, *lengths, *refs;
  int n_users, max_pages;
} kfl_kv4_map;

/* Bytes of one page over all layers and heads.  Errors: KFL_ERR_ARG. */
int kfl_kv4_page_bytes(const kfl_kv4_pool *pool, size_t *out);

/* Codes n_tokens rows of k and v (n_heads = n_kv_heads, the same type; any of the three) of one layer into
 * the pages: row t to user users[t] at positions[t] (device int32; users NULL: row t to user t).  With rope
 * (NULL: none) k is rotated first, in fp32, by the row's position.  The pages are those of the table: a position
 * behind them (or a user or page out of range) is reported in status and not written.  Rows of one call are
 * distinct places; a page that several users hold is written for all of them (kfl_kv4_fork leaves no
 * such page to be written).  Lengths are kfl_kv4_reserve's to change.
 * Errors: KFL_ERR_ARG, KFL_ERR_RANGE (layer, n_tokens * n_kv_heads of 2^31 and more), KFL_ERR_CUDA. */
int kfl_kv4_append(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *k,
                   const kfl_heads *v, const int32_t *users, const int32_t *positions, int n_tokens,
                   const kfl_rope_plan *rope, int32_t *status, void *cuda_stream);

/* The same for rows whose place is not their position (drafted trees, users that rows were taken from): row t to slot
 * slots[t] of its user, k rotated by positions[t] (device int32 [n_tokens]; rope is needed).  A slot behind the user's
 * pages, or a position outside the rotation's table, is reported in status and not written. */
int kfl_kv4_append_at(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *k,
                      const kfl_heads *v, const int32_t *users, const int32_t *slots, const int32_t *positions,
                      int n_tokens, const kfl_rope_plan *rope, int32_t *status, void *cuda_stream);

/* The values that the cache holds for the rows (users[t], positions[t]) of one layer, rounded to the outputs'
 * type.  Rows out of range are reported in status and not written. */
int kfl_kv4_read(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const int32_t *users,
                 const int32_t *positions, int n_tokens, const kfl_heads *k_out, const kfl_heads *v_out,
                 int32_t *status, void *cuda_stream);

/* Attention over the cached rows of one layer, softmax(scale q k^T) v, for n_seqs sequences:
 *   users     device int32 [n_seqs]: whose pages (NULL: sequence s is user s)
 *   q_start   device int32 [n_seqs + 1]: sequence s's tokens are rows [q_start[s], q_start[s + 1]) of q and out
 *             (NULL: one token each, n_tokens = n_seqs).  Each has at most max_q tokens, all n_tokens together.
 * They are the user's last tokens, already appended: token i of c stands at position length - c + i and sees
 * the positions up to its own, with window > 0 only the last `window` of them.  A token that sees nothing (a
 * user without rows, more tokens than rows) gets zeros, and -inf in lse.  What lies outside a token's
 * view does not reach its output, NaN included.
 *   q, out    bf16 or fp16, the same type and number of heads: a multiple of n_kv_heads, query head h reading
 *             KV head h / (n_heads / n_kv_heads), at most 128 heads per KV head; out does not overlap q
 *   scale     of the scores (normally 1 / sqrt(head_dim))
 *   lse       NULL, or device fp32 [n_tokens][n_heads]: the natural log of the sum of exp(scores)
 *   max_pages * page_tokens at most 2^26; a sequence's query rows per KV head at most 2^30.  Prompts that see more
 *             than 2^31 tiles (of 256 rows by 64 keys, per KV head, summed over 512 neighbouring sequences: one
 *             prompt of 2^22 tokens of 8 heads per KV head) are reported (KFL_BAD_POSITION) and not computed
 *   workspace device memory of kfl_kv4_attend_workspace_bytes for the same sizes (or larger ones), 16-byte
 *             aligned, zeroed before its first use and left as it has to be found.  Calls that may overlap
 *             (other streams, no ordering) need one each; after KFL_TIMED_OUT it is zeroed again.
 * A page out of range is reported in status and its rows count as not cached.
 * Precision: fp16 products with fp32 sums; softmax weights rounded to fp16; sums and softmax statistics in fp32.
 * The cached values enter exactly, as codes (few query rows per KV head) or as sums of two fp16 numbers (many, fp16
 * outputs), or rounded to fp16 (many, bf16 outputs).  Root mean square error of the outputs against 64 bits,
 * their own rounding among it: 1.7e-3 with bf16, 2.9e-4 with fp16.
 * Errors: KFL_ERR_ARG, KFL_ERR_RANGE (layer, query rows), KFL_ERR_CUDA. */
int kfl_kv4_attend(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *q,
                   const kfl_heads *out, float *lse, const int32_t *users, const int32_t *q_start, int n_seqs,
                   int n_tokens, int max_q, float scale, int window, void *workspace, size_t workspace_bytes,
                   int32_t *status, void *cuda_stream);
int kfl_kv4_attend_workspace_bytes(const kfl_kv4_pool *pool, int n_heads, int n_seqs, int n_tokens, int max_q,
                                   size_t *out);

/* ---- pages.  n lists up to 1024 users; lists are device int32.  workspace: device memory of
 * kfl_kv4_pages_workspace_bytes, 16-byte aligned, its contents of no account.  Free pages are given out lowest
 * number first, in the order of the list. ---- */
int kfl_kv4_pages_workspace_bytes(const kfl_kv4_pool *pool, size_t *out);

/* Room for n_new[i] >= 0 more tokens of user users[i]: gives it the pages that it lacks and adds n_new[i] to its
 * length.  From the first user on that the pool has no room for, those that need a page are left as
 * they were (KFL_NO_PAGES); so is one whose table row is too short.  A last page that other users hold too is
 * not split: kfl_kv4_fork never shares one that is not full. */
int kfl_kv4_reserve(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const int32_t *users, const int32_t *n_new,
                    int n, void *workspace, int32_t *status, void *cuda_stream);

/* User dst[i] goes on from where src[i] is, for all i at once (beams change places in one call): gives back what
 * it held, holds src[i]'s full pages together with it, and gets a copy of a last page that is not full.  dst
 * names each user once; src[i] = dst[i] changes nothing.  New pages are taken before old ones are given
 * back.  Pairs that find no page are left as they were (KFL_NO_PAGES). */
int kfl_kv4_fork(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const int32_t *src, const int32_t *dst, int n,
                 void *workspace, int32_t *status, void *cuda_stream);

/* Gives the users' pages back (those that nobody else holds become free), empties their rows and lengths. */
int kfl_kv4_free(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const int32_t *users, int n, int32_t *status,
                 void *cuda_stream);

/* Moves the live pages together: with L pages in use, those numbered L and up go to the free ones below L, lowest
 * to lowest.  table_out and refs_out ([n_users][max_pages], [n_pages]; the map's own or other buffers) get the new
 * numbers, n_live (device int32, may be NULL) L.  Pages from L on are free afterwards. */
int kfl_kv4_compact(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int32_t *table_out, int32_t *refs_out,
                    int32_t *n_live, void *workspace, int32_t *status, void *cuda_stream);

/* Copies page src[i] to page dst[i] (device int32 [n], any n), all layers and heads.  No page is named as a
 * destination twice, or as both source and destination. */
int kfl_kv4_copy_pages(const kfl_kv4_pool *pool, const int32_t *src, const int32_t *dst, int n, int32_t *status,
                       void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* KAFILA_KV4_H */
