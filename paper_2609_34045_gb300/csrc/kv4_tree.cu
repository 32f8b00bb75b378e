// Trees of drafted tokens (include/kafila_kv4_tree.h): kfl_kv4_tree, kfl_kv4_tree_window.
//
// A node's view is its own bit and those of its ancestors, of the nearest ones with a window.  A parent stands before its children, so the walk upwards
// passes the nodes in descending order: a thread per node writes its words from the last to the first, each once, and
// keeps none of them.  Parents lie in shared memory; the walk is a chain of its loads, some 30 clocks a step.  4 to 132 bytes
// a node: nothing but latency, 1.5 us in a graph for four trees of 8, 2.8 for 64 of up to 128.
#include "../../include/kafila_kv4_tree.h"
#include "heads.cuh"

namespace kfl {
namespace {

constexpr int TREE_THREADS = 128;

struct TreeParams {
  const int32_t *parents, *q_start, *first;
  int n_tokens, max_q, words;
  int window;  // nodes of a view (none: as many as there can be)
  uint32_t *views;
  int32_t *positions, *status;
};

__global__ void __launch_bounds__(TREE_THREADS) kv4_tree_kernel(const TreeParams p) {
  __shared__ int parent[KFL_KV4_TREE_MOST];
  pdl_launch_dependents();
  pdl_wait();
  const int s = blockIdx.x;
  const int begin = p.q_start ? p.q_start[s] : s, count = p.q_start ? p.q_start[s + 1] - begin : 1;
  if (begin < 0 || count < 0 || count > p.max_q || begin > p.n_tokens - count) {
    if (threadIdx.x == 0) report(p.status, KFL_BAD_POSITION);
    return;
  }
  const int first = p.first ? p.first[s] : 0;
  for (int i = threadIdx.x; i < count; i += TREE_THREADS) {
    int up = p.parents[begin + i];
    if (up < -1 || up >= i) {
      report(p.status, KFL_BAD_POSITION);
      up = -1;
    }
    parent[i] = up;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += TREE_THREADS) {
    uint32_t *view = p.views + (int64_t)(begin + i) * p.words;
    int at = i, seen = 0;
    for (int w = p.words - 1; w >= 0; --w) {
      uint32_t bits = 0;
      for (; at >= 32 * w; at = parent[at], ++seen) bits |= seen < p.window ? 1u << (at & 31) : 0u;  // (-1 is below every word)
      view[w] = bits;
    }
    if (p.positions) p.positions[begin + i] = first + seen - 1;
  }
}

}  // namespace
}  // namespace kfl

using namespace kfl;

static int tree(const char *me, const int32_t *parents, const int32_t *q_start, const int32_t *first, int n_seqs, int n_tokens,
                int max_q, int window, uint32_t *views, int32_t *positions, int32_t *status, void *cuda_stream) {
  if (n_seqs < 0 || n_tokens < 0 || max_q < 1) return bad_arg(me, "n_seqs, n_tokens and max_q are not negative");
  if (max_q > KFL_KV4_TREE_MOST) {
    bad_arg(me, "a sequence has at most 1024 nodes");
    return KFL_ERR_RANGE;
  }
  if (window < 0) return bad_arg(me, "the window is not negative");
  if (!q_start && n_tokens != n_seqs) return bad_arg(me, "without q_start every sequence has one node");
  if (n_seqs == 0 || n_tokens == 0) return KFL_OK;
  if (!parents || !views) return bad_arg(me, "parents and views are needed");
  TreeParams p = {};
  p.parents = parents, p.q_start = q_start, p.first = first;
  p.n_tokens = n_tokens, p.max_q = q_start ? max_q : 1, p.words = (max_q + 31) / 32;
  p.window = window > 0 ? window : KFL_KV4_TREE_MOST;
  p.views = views, p.positions = positions, p.status = status;
  return cuda_result(launch_chained(kv4_tree_kernel, n_seqs, TREE_THREADS, 0, static_cast<cudaStream_t>(cuda_stream), p), me);
}

extern "C" int kfl_kv4_tree(const int32_t *parents, const int32_t *q_start, const int32_t *first, int n_seqs, int n_tokens,
                            int max_q, uint32_t *views, int32_t *positions, int32_t *status, void *cuda_stream) {
  return tree("kfl_kv4_tree", parents, q_start, first, n_seqs, n_tokens, max_q, 0, views, positions, status, cuda_stream);
}

extern "C" int kfl_kv4_tree_window(const int32_t *parents, const int32_t *q_start, const int32_t *first, int n_seqs,
                                   int n_tokens, int max_q, int window, uint32_t *views, int32_t *positions, int32_t *status,
                                   void *cuda_stream) {
  return tree("kfl_kv4_tree_window", parents, q_start, first, n_seqs, n_tokens, max_q, window, views, positions, status,
              cuda_stream);
}
