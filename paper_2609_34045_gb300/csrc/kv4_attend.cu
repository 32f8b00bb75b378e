// Attention over the 4-bit paged KV cache (include/kafila_kv4.h): kfl_kv4_attend.
//
// Few query rows per KV head (a decode step's group, some drafted tokens) go to the kernel that streams the cache, sixteen
// rows at a time (kv4_attend_few.cu), more to the one that multiplies 128 rows at a time (kv4_attend_prompt.cu).
#include <math.h>

#include <algorithm>

#include "../../include/kafila_kv4_tree.h"
#include "kv4_attend.cuh"

namespace kfl {
namespace {

// Which kernel: the first reads and decodes a tile once for every sixteen rows, the second once for all, at a larger cost
// to begin with.  us, heads of 128, 8 KV heads, first against second:
//   sequences x keys      24 rows        32 rows        48 rows        64 rows
//    1 x 1000            14.3   23.1    14.5   23.7    14.7   24.8    14.9   28.8
//    4 x 3000            21.2   33.3    21.4   33.7    24.6   35.0    29.8   37.8
//    8 x 4096            33.4   56.5    33.8   57.5    45.4   59.6    55.8   65.1
//    8 x 8192            55.4   76.8    55.9   76.8    76.6   79.6    99.7   85.2
//   16 x 8192            99.5    121    99.8    122     141    124
//   64 x 4096             186    253     186    254     274    257
// The contexts' lengths are on the device: the third and fourth sixteen rows go by what the tables could hold.  These
// times are of tables that just fit; the same calls with tables of 131072 keys a user take the second kernel (4 x 3000, 48 rows:
// 34.8 us for 24.4; 1 x 1000, 64 rows: 28.7 for 14.8).
bool is_few(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int n_seqs, int64_t rows) {
  if (rows <= 32) return true;
  return rows <= FEW_ROWS && n_seqs <= 65536 &&
         (int64_t)n_seqs * pool->n_kv_heads * map->max_pages * pool->page_tokens <= (rows <= 48 ? 1 << 19 : 1 << 18);
}

int check_attend(const char *me, const kfl_kv4_pool *pool, int n_heads, int n_seqs, int n_tokens, int max_q,
                 bool bytes) {
  const int rc = check_pool(pool, bytes, me);
  if (rc != KFL_OK) return rc;
  if (n_heads < 1 || n_heads % pool->n_kv_heads || n_heads / pool->n_kv_heads > 128)
    return bad_arg(me, "the query heads are a multiple of n_kv_heads, at most 128 per KV head");
  if (n_seqs < 0 || n_tokens < 0 || max_q < 1) return bad_arg(me, "n_seqs, n_tokens and max_q are not negative");
  return KFL_OK;
}

}  // namespace
}  // namespace kfl

using namespace kfl;

extern "C" int kfl_kv4_attend_workspace_bytes(const kfl_kv4_pool *pool, int n_heads, int n_seqs, int n_tokens,
                                              int max_q, size_t *out) {
  const char *me = "kfl_kv4_attend_workspace_bytes";
  const int rc = check_attend(me, pool, n_heads, n_seqs, n_tokens, max_q, false);
  if (rc != KFL_OK) return rc;
  if (!out) return bad_arg(me, "NULL pointer");
  const int64_t rows = (int64_t)max_q * (n_heads / pool->n_kv_heads);
  *out = TICKET_BYTES +
         (rows <= 32 ? attend_few_partials(pool->head_dim, few_cols(rows))
                     : std::max(attend_few_partials(pool->head_dim, 16), attend_prompt_partials(pool->head_dim, rows)));
  return KFL_OK;
}

// views NULL: each token sees the rows up to its own.
static int attend(const char *me, const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *q,
                  const kfl_heads *out, float *lse, const int32_t *users, const int32_t *q_start, const uint32_t *views,
                  int n_seqs, int n_tokens, int max_q, float scale, int window, void *workspace, size_t workspace_bytes,
                  int32_t *status, void *cuda_stream) {
  if (!heads_valid(q, n_tokens) || !heads_valid(out, n_tokens)) return bad_arg(me, "q and out are needed");
  int rc = check_attend(me, pool, q->n_heads, n_seqs, n_tokens, max_q, true);
  if (rc == KFL_OK) rc = check_map(map, me);
  if (rc == KFL_OK) rc = check_layer(pool, layer, me);
  if (rc != KFL_OK) return rc;
  if (q->n_heads != out->n_heads || q->dtype != out->dtype || q->dtype == KFL_DT_FP32)
    return bad_arg(me, "q and out have the same heads and are both bf16 or both fp16");
  if (!std::isfinite(scale) || window < 0) return bad_arg(me, "scale is finite, window not negative");
  if (!q_start && n_tokens != n_seqs) return bad_arg(me, "without q_start every sequence has one token");
  size_t need = 0;
  rc = kfl_kv4_attend_workspace_bytes(pool, q->n_heads, n_seqs, n_tokens, max_q, &need);
  if (rc != KFL_OK) return rc;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15) || workspace_bytes < need)
    return bad_arg(me, "a 16-byte aligned workspace of kfl_kv4_attend_workspace_bytes is needed");
  if (n_seqs == 0 || n_tokens == 0) return KFL_OK;
  if (((int64_t)map->max_pages * pool->page_tokens) > (1 << 26)) return bad_arg(me, "max_pages * page_tokens is at most 2^26");
  AttendParams p = {};
  p.pool = pool_of(*pool), p.map = map_of(*map), p.layer = layer;
  p.q = view_of(*q), p.out = view_of(*out);
  p.q_wide = rows_aligned16(*q), p.out_wide = rows_aligned16(*out), p.bf16 = q->dtype == KFL_DT_BF16;
  p.lse = lse, p.users = users, p.q_start = q_start;
  p.views = views, p.words = (max_q + 31) / 32;
  p.n_seqs = n_seqs, p.n_tokens = n_tokens, p.max_q = q_start ? max_q : 1;
  p.n_heads = q->n_heads, p.group = q->n_heads / pool->n_kv_heads;
  p.group_inv = (65536 + p.group - 1) / p.group;
  p.scale = scale, p.status = status;
  // (a window that no context fills is none; the kernels take it off places below 2^26, in 32 bits)
  p.window = window >= map->max_pages * pool->page_tokens ? 0 : window;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const int64_t rows = (int64_t)p.max_q * p.group;
  if (std::min(rows, (int64_t)n_tokens * p.group) > (1 << 30)) {
    bad_arg(me, "more than 2^30 query rows of a sequence per KV head");
    return KFL_ERR_RANGE;
  }
  const bool few = is_few(pool, map, n_seqs, rows);
  p.most_blocks = few ? (int)((rows + few_cols(rows) - 1) / few_cols(rows)) : 0;
  p.tickets = static_cast<unsigned *>(workspace);
  p.partials = reinterpret_cast<float *>(static_cast<char *>(workspace) + TICKET_BYTES);
  int dev = 0, n_sm = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev);
  for (int s0 = 0; e == cudaSuccess && s0 < n_seqs; s0 += FEW_SEQS) {
    p.seq0 = s0, p.n_seqs = std::min(FEW_SEQS, n_seqs - s0);
    p.users = users ? users + s0 : nullptr, p.q_start = q_start ? q_start + s0 : nullptr;
    e = few ? launch_attend_few(p, few_cols(rows), n_sm, s) : launch_attend_prompt(p, n_sm, s);
  }
  return cuda_result(e, me);
}

extern "C" int kfl_kv4_attend(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *q,
                              const kfl_heads *out, float *lse, const int32_t *users, const int32_t *q_start,
                              int n_seqs, int n_tokens, int max_q, float scale, int window, void *workspace,
                              size_t workspace_bytes, int32_t *status, void *cuda_stream) {
  return attend("kfl_kv4_attend", pool, map, layer, q, out, lse, users, q_start, nullptr, n_seqs, n_tokens, max_q, scale, window,
                workspace, workspace_bytes, status, cuda_stream);
}

extern "C" int kfl_kv4_attend_tree(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *q,
                                   const kfl_heads *out, float *lse, const int32_t *users, const int32_t *q_start,
                                   const uint32_t *views, int n_seqs, int n_tokens, int max_q, float scale, int window,
                                   void *workspace, size_t workspace_bytes, int32_t *status, void *cuda_stream) {
  const char *me = "kfl_kv4_attend_tree";
  if (max_q > KFL_KV4_TREE_MOST) {
    bad_arg(me, "a sequence has at most 1024 nodes");
    return KFL_ERR_RANGE;
  }
  if ((!views && n_tokens > 0) || (reinterpret_cast<uintptr_t>(views) & 3)) return bad_arg(me, "views are needed");
  return attend(me, pool, map, layer, q, out, lse, users, q_start, views, n_seqs, n_tokens, max_q, scale, window, workspace,
                workspace_bytes, status, cuda_stream);
}
