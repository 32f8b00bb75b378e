// The attention weight of cached rows (include/kafila_kv4_evict.h): kfl_kv4_weights.
#include <math.h>

#include <algorithm>

#include "kv4_weights.cuh"

using namespace kfl;

extern "C" int kfl_kv4_weights(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *q,
                               const float *lse, const kfl_kv4_mass *mass, const int32_t *users, const int32_t *q_start,
                               int n_seqs, int n_tokens, int max_q, float scale, int window, void *workspace,
                               size_t workspace_bytes, int32_t *status, void *cuda_stream) {
  const char *me = "kfl_kv4_weights";
  if (!heads_valid(q, n_tokens)) return bad_arg(me, "q is needed");
  int rc = check_pool(pool, true, me);
  if (rc == KFL_OK) rc = check_map(map, me);
  if (rc == KFL_OK) rc = check_layer(pool, layer, me);
  if (rc != KFL_OK) return rc;
  if (q->dtype == KFL_DT_FP32) return bad_arg(me, "q is bf16 or fp16");
  if (!std::isfinite(scale) || window < 0) return bad_arg(me, "scale is finite, window not negative");
  if (!q_start && n_tokens != n_seqs) return bad_arg(me, "without q_start every sequence has one token");
  size_t need = 0;
  rc = kfl_kv4_attend_workspace_bytes(pool, q->n_heads, n_seqs, n_tokens, max_q, &need);  // (checks heads and counts)
  if (rc != KFL_OK) return rc;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15) || workspace_bytes < need)
    return bad_arg(me, "a 16-byte aligned workspace of kfl_kv4_attend_workspace_bytes is needed");
  if (n_seqs > WEIGHT_SEQS) {
    bad_arg(me, "more than 1024 sequences in one call");
    return KFL_ERR_RANGE;
  }
  if (n_seqs == 0 || n_tokens == 0) return KFL_OK;
  if (!mass_valid(mass) || !lse || (reinterpret_cast<uintptr_t>(lse) & 3)) return bad_arg(me, "lse and mass are needed");
  if (((int64_t)map->max_pages * pool->page_tokens) > (1 << 26)) return bad_arg(me, "max_pages * page_tokens is at most 2^26");
  WeightParams p = {};
  p.pool = pool_of(*pool), p.map = map_of(*map), p.layer = layer;
  p.q = view_of(*q), p.q_wide = rows_aligned16(*q), p.bf16 = q->dtype == KFL_DT_BF16;
  p.lse = lse, p.mass = view_of(*mass), p.all_users = users;
  p.n_tokens = n_tokens, p.max_q = q_start ? max_q : 1;
  p.n_heads = q->n_heads, p.group = q->n_heads / pool->n_kv_heads;
  p.scale = scale, p.status = status;
  // (a window that no context fills is none; the kernels take it off places below 2^26, in 32 bits)
  p.window = window >= map->max_pages * pool->page_tokens ? 0 : window;
  const int64_t rows = (int64_t)std::min(p.max_q, n_tokens) * p.group;
  if (rows > (1 << 30)) {
    bad_arg(me, "more than 2^30 query rows of a sequence per KV head");
    return KFL_ERR_RANGE;
  }
  p.tickets = static_cast<unsigned *>(workspace);
  p.partials = reinterpret_cast<float *>(static_cast<char *>(workspace) + TICKET_BYTES);
  // The streaming kernel takes up to 32 query rows per KV head at once, and twice as many in two launches; the other one's time is
  // that of its 256-key tiles, much the same up to 128 rows: little as long as every SM has one at most (by what the tables could
  // hold: the lengths are on the device).  us in a graph, heads of 128, 8 KV heads, bf16:
  //   sequences x keys   streaming: 8 rows   16     32     48     64   |   the other: 72    128    256
  //    1 x 1000                    5.6      7.0    9.3   16.9   18.2              11.0   10.7   12.0
  //    4 x 3000                    6.4      8.2   10.7   19.1   21.1              21.8   19.9   23.7
  //    8 x 8192                   12.7     17.0   23.7   40.9   47.0              73.4   62.1   80.3
  //   32 x 4096                   21.1     28.9   41.6   74.4   83.0               143    124    159
  const int64_t tiles = (int64_t)n_seqs * pool->n_kv_heads * (((int64_t)map->max_pages * pool->page_tokens + 255) / 256);
  const bool few = rows <= WEIGHT_COLS || (rows <= 2 * WEIGHT_COLS && tiles > 152);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  int dev = 0, n_sm = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev);
  for (int s0 = 0; e == cudaSuccess && s0 < n_seqs; s0 += FEW_SEQS) {
    p.seq0 = s0, p.n_seqs = std::min(FEW_SEQS, n_seqs - s0);
    p.users = users ? users + s0 : nullptr, p.q_start = q_start ? q_start + s0 : nullptr;
    if (few)
      for (p.row0 = 0; e == cudaSuccess && p.row0 < rows; p.row0 += WEIGHT_COLS)
        e = launch_weights_few(p, weight_cols(rows - p.row0), n_sm, s);
    else
      e = launch_weights_many(p, n_sm, s);
  }
  return cuda_result(e, me);
}
