// Attention over the 4-bit paged KV cache (include/kafila_kv4.h): kfl_kv4_attend.
//
// A warp per query row (token, head): 32 keys at a time, a lane's key's score from its codes, the running maximum and
// sum of the softmax, then each lane's channels of the weighted values.
#include <math.h>

#include <algorithm>

#include "kv4_attend.cuh"

namespace kfl {
namespace {

template <class T>
__global__ void __launch_bounds__(128) kv4_attend_kernel(const AttendParams p) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ float s_q[4][128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hd = p.pool.head_dim;
  const int s = blockIdx.y / p.max_q, i = blockIdx.y % p.max_q;
  const int head = blockIdx.x * 4 + warp;
  if (head >= p.n_heads) return;
  const int first = p.q_start ? p.q_start[s] : s, count = (p.q_start ? p.q_start[s + 1] : s + 1) - first;
  if (i >= count || first < 0 || first + i >= p.n_tokens) return;
  const int64_t t = first + i;
  const int user = p.users ? p.users[s] : s;
  const bool known = user >= 0 && user < p.map.n_users;
  if (!known && lane == 0) report(p.status, KFL_BAD_USER);
  const int length = known ? min(max(0, p.map.lengths[user]), p.map.max_pages << p.pool.log2_tokens) : 0;
  const int end = length - count + i + 1;  // keys below it are seen
  const int begin = p.window > 0 ? max(0, end - p.window) : 0;
  const T *q = reinterpret_cast<const T *>(p.q.row(t, head));
  for (int c = lane; c < hd; c += 32) s_q[warp][c] = to_f32(q[c]) * p.scale;
  __syncwarp();
  float top = -INFINITY, sum = 0.f, acc[4] = {};
  for (int k0 = begin; k0 < end; k0 += 32) {
    const int key = k0 + lane;
    const uint8_t *block = nullptr;
    int slot = 0;
    if (key < end) {
      const int page = p.map.table[(int64_t)user * p.map.max_pages + (key >> p.pool.log2_tokens)];
      if (page < 0 || page >= p.pool.n_pages)
        report(p.status, KFL_BAD_PAGE);
      else
        block = p.pool.block(page, p.layer, head / p.group), slot = key & (p.pool.page_tokens() - 1);
    }
    float score = -INFINITY;
    const int groups = hd / KV4_GROUP;
    if (block) {
      score = 0.f;
      for (int g = 0; g < groups; ++g) {
        const __half2 par = *reinterpret_cast<const __half2 *>(block + 2 * p.pool.code_bytes() + (slot * groups + g) * 4);
        for (int w = 0; w < 8; ++w) {
          const uint32_t codes = *reinterpret_cast<const uint32_t *>(block + slot * (hd / 2) + g * 32 + w * 4);
          for (int j = 0; j < 8; ++j)
            score = fmaf(fmaf((float)((int)((codes >> (4 * j)) & 15) - 8), __low2float(par), __high2float(par)),
                         s_q[warp][g * 64 + w * 8 + j], score);
        }
      }
    }
    float m = score;
    for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    const float now = fmaxf(top, m);
    const float base = now == -INFINITY ? 0.f : now;
    const float keep = expf(top - base);
    const float weight = block ? expf(score - base) : 0.f;
    top = now;
    sum *= keep;
    for (int c = 0; c < 4; ++c) acc[c] *= keep;
    for (int j = 0; j < 32; ++j) {
      const uint64_t at = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(block), j);
      const float w = __shfl_sync(0xffffffffu, weight, j);
      const int sl = __shfl_sync(0xffffffffu, slot, j);
      if (!at) continue;
      const uint8_t *b = reinterpret_cast<const uint8_t *>(at);
      sum += w;
      for (int c = 0; c < hd / 32; ++c) {
        const int ch = lane + 32 * c;
        const int byte = b[p.pool.code_bytes() + sl * (hd / 2) + ch / 2];
        const __half2 par = *reinterpret_cast<const __half2 *>(b + 2 * p.pool.code_bytes() + p.pool.param_bytes() +
                                                               (sl * groups + ch / KV4_GROUP) * 4);
        acc[c] = fmaf(w, fmaf((float)((ch & 1 ? byte >> 4 : byte & 15) - 8), __low2float(par), __high2float(par)), acc[c]);
      }
    }
  }
  T *out = reinterpret_cast<T *>(p.out.row(t, head));
  for (int c = 0; c < hd / 32; ++c) out[lane + 32 * c] = from_f32<T>(sum == 0.f ? 0.f : acc[c] / sum);
  if (p.lse && lane == 0) p.lse[t * p.n_heads + head] = sum == 0.f ? -INFINITY : top + logf(sum);
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

// The workspace: tickets (zero between calls), then partial results.
size_t ticket_bytes(const kfl_kv4_pool *pool, int n_seqs) {
  return ((size_t)std::min(n_seqs, FEW_SEQS) * pool->n_kv_heads * 4 + 127) / 128 * 128;
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
  const int cols = (int)std::min<int64_t>((int64_t)max_q * (n_heads / pool->n_kv_heads), FEW_ROWS);
  *out = ticket_bytes(pool, n_seqs) + attend_few_partials(pool->head_dim, cols);
  return KFL_OK;
}

extern "C" int kfl_kv4_attend(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *q,
                              const kfl_heads *out, float *lse, const int32_t *users, const int32_t *q_start,
                              int n_seqs, int n_tokens, int max_q, float scale, int window, void *workspace,
                              size_t workspace_bytes, int32_t *status, void *cuda_stream) {
  const char *me = "kfl_kv4_attend";
  if (!heads_valid(q) || !heads_valid(out)) return bad_arg(me, "q and out are needed");
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
  p.n_seqs = n_seqs, p.n_tokens = n_tokens, p.max_q = q_start ? max_q : 1;
  p.n_heads = q->n_heads, p.group = q->n_heads / pool->n_kv_heads;
  p.scale = scale, p.window = window, p.status = status;
  p.tickets = static_cast<unsigned *>(workspace);
  p.partials = reinterpret_cast<float *>(static_cast<char *>(workspace) + ticket_bytes(pool, n_seqs));
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const int64_t rows = (int64_t)p.max_q * p.group;
  if (rows <= FEW_ROWS) {
    int dev = 0, n_sm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev);
    for (int s0 = 0; e == cudaSuccess && s0 < n_seqs; s0 += FEW_SEQS) {
      p.seq0 = s0, p.n_seqs = std::min(FEW_SEQS, n_seqs - s0);
      p.users = users ? users + s0 : nullptr, p.q_start = q_start ? q_start + s0 : nullptr;
      e = launch_attend_few(p, (int)rows, n_sm, s);
    }
    return cuda_result(e, me);
  }
  const dim3 grid((q->n_heads + 3) / 4, n_seqs * p.max_q);
  const cudaError_t e = q->dtype == KFL_DT_BF16 ? launch_chained(kv4_attend_kernel<__nv_bfloat16>, grid, 128, 0, s, p)
                                                : launch_chained(kv4_attend_kernel<__half>, grid, 128, 0, s, p);
  return cuda_result(e, me);
}
