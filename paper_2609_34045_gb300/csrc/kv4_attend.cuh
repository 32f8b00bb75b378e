// Attention over the 4-bit paged KV cache: what its entry point hands to the kernels.
#pragma once

#include "kv4.cuh"
#include "prefill.cuh"  // SmemOptIn

namespace kfl {

constexpr int FEW_ROWS = 64;     // most query rows per KV head of the few-row kernel, in blocks of 8 or 16
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
  unsigned group_inv;  // 2^16 / group, rounded up
  int most_blocks;    // few rows: of a KV head's query rows, in blocks of few_cols
  unsigned *tickets;  // zero between launches: [n_seqs][n_kv_heads][most_blocks], many rows: [FEW_BLOCKS]
  float *partials;
  int32_t *status;
};

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

// Waits for an mbarrier phase for two seconds at most (by the clock: a poll may itself be held for microseconds).
__device__ __forceinline__ bool wait_2s(uint32_t bar, uint32_t parity) {
  for (int i = 0; i < 64; ++i)
    if (mbar_try_wait(bar, parity)) return true;
  const unsigned long long until = global_ns() + 2000000000ull;
  while (!mbar_try_wait(bar, parity))
    if (global_ns() > until) return false;
  return true;
}

// Query rows of a KV head that the few-row kernel works on at once.
inline int few_cols(int64_t rows) { return rows <= 8 ? 8 : 16; }
// Bytes of its partial results.
size_t attend_few_partials(int head_dim, int cols);
cudaError_t launch_attend_few(const AttendParams &p, int cols, int n_sm, cudaStream_t s);


// Query rows of a KV head that share a decoded tile in the many-row kernel.
inline int prompt_rows(int64_t rows) { return rows > 128 ? 256 : 128; }
size_t attend_prompt_partials(int head_dim, int64_t rows);
cudaError_t launch_attend_prompt(const AttendParams &p, int n_sm, cudaStream_t s);

}  // namespace kfl
