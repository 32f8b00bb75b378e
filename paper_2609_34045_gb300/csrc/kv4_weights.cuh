// Attention weights of cached rows: what the entry point hands to the kernels.
#pragma once

#include "../../include/kafila_kv4_evict.h"
#include "kv4_attend.cuh"

namespace kfl {

constexpr int WEIGHT_SEQS = 1024;  // sequences of a call
constexpr int WEIGHT_COLS = 32;    // most query rows per KV head of one launch of the streaming kernel

struct MassView {
  float *data;
  int64_t layer_stride, user_stride, head_stride;
  __device__ __forceinline__ float *row(int layer, int user, int head) const {
    return data + layer * layer_stride + user * user_stride + head * head_stride;
  }
};
inline MassView view_of(const kfl_kv4_mass &m) { return {m.data, m.layer_stride, m.user_stride, m.head_stride}; }
inline bool mass_valid(const kfl_kv4_mass *m) { return m && m->data && (reinterpret_cast<uintptr_t>(m->data) & 3) == 0; }

struct WeightParams {
  Kv4Pool pool;
  Kv4Map map;
  int layer;
  HeadsView q;
  int q_wide, bf16;
  const float *lse;
  MassView mass;
  const int32_t *all_users;           // the call's list, or NULL
  const int32_t *users, *q_start;     // from sequence seq0 on
  int seq0, n_seqs, n_tokens, max_q, n_heads, group;
  int row0;  // streaming kernel: query rows [row0, row0 + its columns) of a KV head
  float scale;
  int window;
  unsigned *tickets;
  float *partials;
  int32_t *status;
};

// A sequence as the kernels' lists hold it: (user, length, first token, tokens); no tokens where there is nothing to do.
// again: an earlier sequence of the call has the user.
__device__ __forceinline__ int4 weight_sequence(const WeightParams &p, int s, bool again, bool tell) {
  const int user = p.users ? p.users[s] : p.seq0 + s;
  const int first = p.q_start ? p.q_start[s] : p.seq0 + s;
  int count = p.q_start ? p.q_start[s + 1] - first : 1, length = 0, bad = 0;
  if (first < 0 || count < 0 || count > p.max_q || first > p.n_tokens - count) bad |= KFL_BAD_POSITION, count = 0;
  if (user < 0 || user >= p.map.n_users || again)
    bad |= KFL_BAD_USER, count = 0;
  else
    length = min(max(0, p.map.lengths[user]), p.map.max_pages << p.pool.log2_tokens);
  if (bad && tell) report(p.status, bad);
  return make_int4(user, length, first, length > 0 ? count : 0);
}
// Whether an earlier sequence of the call has the same user.
__device__ __forceinline__ bool named_earlier(const WeightParams &p, int s) {
  if (!p.all_users) return false;
  const int user = p.users[s];
  bool again = false;
#pragma unroll 8
  for (int j = 0; j < p.seq0 + s; ++j) again |= p.all_users[j] == user;
  return again;
}

inline int weight_cols(int64_t rows) { return rows <= 8 ? 8 : rows <= 16 ? 16 : 32; }
cudaError_t launch_weights_few(const WeightParams &p, int cols, int n_sm, cudaStream_t s);
cudaError_t launch_weights_many(const WeightParams &p, int n_sm, cudaStream_t s);

}  // namespace kfl
