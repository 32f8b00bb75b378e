// Attention over the 4-bit paged KV cache: what its entry point hands to the kernels.
#pragma once

#include "kv4.cuh"
#include "prefill.cuh"  // SmemOptIn

namespace kfl {

constexpr int FEW_ROWS = 64;     // most query rows per KV head of the few-row kernel, in blocks of 8 or 16
constexpr int FEW_SEQS = 512;    // sequences of one of its launches (their places lie in shared memory)
constexpr int FEW_BLOCKS = 152;  // most blocks of one of its launches

// The workspace: tickets (zero between calls), then partial results.  The tickets' part is the same for every call, so
// that no call's partial results lie where another one's tickets are.
constexpr size_t TICKET_BYTES = (size_t)FEW_SEQS * KV4_MOST_HEADS * ((FEW_ROWS + 15) / 16) * 4;
static_assert(TICKET_BYTES >= FEW_BLOCKS * 4 && TICKET_BYTES % 128 == 0, "tickets");

struct AttendParams {
  Kv4Pool pool;
  Kv4Map map;
  int layer;
  HeadsView q, out;
  int q_wide, out_wide, bf16;
  float *lse;
  const int32_t *users, *q_start;
  const uint32_t *views;  // trees: which of the last tokens each token sees, [n_tokens][words]; else NULL
  int words;
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

// Trees.  Rows of context that a token which sees `nodes` of the last tokens still sees with a window.
__device__ __forceinline__ int tree_nodes(const AttendParams &p, int token, int count) {
  const uint32_t *view = p.views + (int64_t)token * p.words;
  int n = 0;
  for (int w = 0; 32 * w < count; ++w) n += __popc(view[w] & (count - 32 * w >= 32 ? 0xffffffffu : (1u << (count - 32 * w)) - 1));
  return n;
}
// Which of the 32 keys from key0 on a token sees, a bit each; its sequence has `count` nodes from key `base` on (below 0
// where a user has fewer rows than nodes: those nodes' keys are not there).
__device__ __forceinline__ uint32_t tree_view(const AttendParams &p, int token, int key0, int base, int count) {
  const uint32_t *view = p.views + (int64_t)token * p.words;
  const int node0 = key0 - base, w = node0 >> 5;  // (of the context: negative)
  const auto word = [&](int i) { return i < 0 ? 0xffffffffu : i < p.words ? view[i] : 0u; };
  uint32_t seen = __funnelshift_r(word(w), word(w + 1), node0 & 31);
  if (node0 + 32 > count) seen &= node0 >= count ? 0u : (1u << (count - node0)) - 1;
  if (p.window > 0 && node0 < 0) {
    const int begin = base - max(0, p.window - tree_nodes(p, token, count)) - key0;  // (at most the nodes' own start)
    if (begin >= 32)
      seen = 0;
    else if (begin > 0)
      seen &= ~((1u << begin) - 1);
  }
  return seen;
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
