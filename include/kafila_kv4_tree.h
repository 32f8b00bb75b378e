/* Trees of drafted tokens over the 4-bit paged KV cache (sm_103a): what a step has to know of a tree, and the
 * attention of its nodes.  The accepted path's rows are brought together by kfl_kv4_keep (kafila_kv4_evict.h).
 *
 * A sequence's drafted tokens are the nodes of a tree (or of several: a node without a parent hangs on the
 * cached context).  A node sees the whole context, its ancestors and itself.  Nodes are appended like other tokens,
 * node i of c at slot length - c + i, but stand at position (context) + (number of ancestors), which k is rotated by
 * (kfl_kv4_append_at).
 *
 * Conventions as in kafila_kv4.h.
 */
#ifndef KAFILA_KV4_TREE_H
#define KAFILA_KV4_TREE_H

#include "kafila_kv4.h"

#ifdef __cplusplus
extern "C" {
#endif

#define KFL_KV4_TREE_MOST 1024 /* nodes of a sequence */

/* Views and positions of n_seqs trees:
 *   parents    device int32 [n_tokens]: the node's parent, counted within its sequence, below its own place; -1: none.
 *              Another value is reported in status (KFL_BAD_POSITION) and counts as none.
 *   q_start    device int32 [n_seqs + 1]: sequence s's nodes are [q_start[s], q_start[s + 1]), at most max_q (NULL: one
 *              each, n_tokens = n_seqs).  A sequence that does not fit is reported (KFL_BAD_POSITION), its rows not written.
 *   first      device int32 [n_seqs]: position of a node without ancestors (NULL: 0)
 *   views      device uint32 [n_tokens][ceil(max_q / 32)]: bit j % 32 of word j / 32 is set if the node sees node j
 *   positions  device int32 [n_tokens], may be NULL: first + number of ancestors
 * Enqueued on cuda_stream, returns without waiting.
 * Errors: KFL_ERR_ARG, KFL_ERR_RANGE (max_q above KFL_KV4_TREE_MOST), KFL_ERR_CUDA. */
int kfl_kv4_tree(const int32_t *parents, const int32_t *q_start, const int32_t *first, int n_seqs, int n_tokens,
                 int max_q, uint32_t *views, int32_t *positions, int32_t *status, void *cuda_stream);

/* The same for attention with a sliding window of `window` positions (0: none): a node sees itself and the window - 1 nodes
 * before it on its path.  kfl_kv4_attend_tree with these views and the same window is the sliding window: each node
 * sees the rows that its token would see behind its path alone.  (With kfl_kv4_tree's views a node sees all of its path,
 * however short the window.)  Positions count all ancestors. */
int kfl_kv4_tree_window(const int32_t *parents, const int32_t *q_start, const int32_t *first, int n_seqs, int n_tokens,
                        int max_q, int window, uint32_t *views, int32_t *positions, int32_t *status, void *cuda_stream);

/* kfl_kv4_attend for trees: token i of c of a sequence sees the rows below length - c and, of the last c, those whose
 * bit is set in its row of `views` ([n_tokens][ceil(max_q / 32)], kfl_kv4_tree's, kfl_kv4_tree_window's or any others; bits
 * from c on count for nothing).  With window > 0 a token that sees b of the last c sees only the last max(0, window - b) rows of the others:
 * window rows in all, or all its b if those are more (a sliding window: kfl_kv4_tree_window's views).  A token that sees nothing gets zeros, and -inf in lse.
 * Arguments, workspace, precision and errors otherwise as kfl_kv4_attend's; max_q up to KFL_KV4_TREE_MOST
 * (KFL_ERR_RANGE). */
int kfl_kv4_attend_tree(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *q,
                        const kfl_heads *out, float *lse, const int32_t *users, const int32_t *q_start,
                        const uint32_t *views, int n_seqs, int n_tokens, int max_q, float scale, int window,
                        void *workspace, size_t workspace_bytes, int32_t *status, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* KAFILA_KV4_TREE_H */
