// Attention over the 4-bit paged KV cache: what its entry point hands to the kernels.
#pragma once

#include "kv4.cuh"
#include "prefill.cuh"  // SmemOptIn

namespace kfl {

constexpr int FEW_ROWS = 16;     // most query rows per KV head of the few-row kernel
constexpr int FEW_SEQS = 512;    // sequences of one of its launches (their places lie in shared memory)
constexpr int FEW_BLOCKS = 152;  // most blocks of one of its launches

struct AttendParams {
  Kv4Pool pool;
  Kv4Map map;
  int layer;
  HeadsView q, out;
  int q_wide, out_wide, bf16;
  float *lse;
  const int32_t *users, *q_start;
  int seq0, n_seqs, n_tokens, max_q, n_heads, group;
  float scale;
  int window;
  unsigned *tickets;  // [n_seqs][n_kv_heads], zero between launches
  float *partials;
  int32_t *status;
};

// Bytes of the few-row kernel's partial results for `cols` query rows per KV head.
size_t attend_few_partials(int head_dim, int cols);
cudaError_t launch_attend_few(const AttendParams &p, int cols, int n_sm, cudaStream_t s);

}  // namespace kfl
