// The 4-bit paged KV cache on the device (include/kafila_kv4.h): where a row lies, and what the entry points
// check alike.
#pragma once

#include "../../include/kafila_kv4.h"
#include "heads.cuh"

namespace kfl {

constexpr int KV4_GROUP = 64;          // channels that share a scale and a centre
constexpr int KV4_MOST_HEADS = 256;    // KV heads of a pool
constexpr float KV4_LIMIT = 32768.f;   // a group with a larger magnitude reads as NaN

struct Kv4Pool {
  uint8_t *pages;
  int n_pages, log2_tokens, n_layers, n_kv_heads, head_dim;
  __host__ __device__ int page_tokens() const { return 1 << log2_tokens; }
  __host__ __device__ int code_bytes() const { return (head_dim / 2) << log2_tokens; }    // K or V codes of a block
  __host__ __device__ int param_bytes() const { return (head_dim / 16) << log2_tokens; }  // K or V parameters
  __host__ __device__ int block_bytes() const { return 2 * (code_bytes() + param_bytes()); }
  __host__ __device__ size_t page_bytes() const { return (size_t)n_layers * n_kv_heads * block_bytes(); }
  __device__ uint8_t *block(int page, int layer, int head) const {
    return pages + (((size_t)page * n_layers + layer) * n_kv_heads + head) * (size_t)block_bytes();
  }
};

struct Kv4Map {
  int32_t *table, *lengths, *refs;
  int n_users, max_pages;
};

inline int log2_page(int tokens) {
  return tokens == 16 ? 4 : tokens == 32 ? 5 : tokens == 64 ? 6 : tokens == 128 ? 7 : -1;
}

// need_pages: the call touches the pages' bytes.
inline int check_pool(const kfl_kv4_pool *p, bool need_pages, const char *where) {
  if (!p) return bad_arg(where, "no pool");
  if (log2_page(p->page_tokens) < 0) return bad_arg(where, "page_tokens is 16, 32, 64 or 128");
  if (p->head_dim != 64 && p->head_dim != 128) return bad_arg(where, "head_dim is 64 or 128");
  if (p->n_kv_heads < 1 || p->n_kv_heads > KV4_MOST_HEADS) return bad_arg(where, "n_kv_heads is 1..256");
  if (p->n_layers < 1 || p->n_layers > (1 << 16)) return bad_arg(where, "n_layers is 1..65536");
  if (p->n_pages < 1 || p->n_pages > (1 << 20)) return bad_arg(where, "n_pages is 1..2^20");
  if (need_pages && (!p->pages || (reinterpret_cast<uintptr_t>(p->pages) & 15)))
    return bad_arg(where, "the pages are 16-byte aligned device memory");
  return KFL_OK;
}
inline int check_map(const kfl_kv4_map *m, const char *where) {
  if (!m || !m->table || !m->lengths || !m->refs) return bad_arg(where, "table, lengths and refs are needed");
  if (m->n_users < 1 || m->max_pages < 1 || m->max_pages > (1 << 24) ||
      (int64_t)m->n_users * m->max_pages > (int64_t)1 << 31)
    return bad_arg(where, "n_users and max_pages (at most 2^24) are positive, their product at most 2^31");
  return KFL_OK;
}
inline int check_layer(const kfl_kv4_pool *p, int layer, const char *where) {
  if (layer >= 0 && layer < p->n_layers) return KFL_OK;
  bad_arg(where, "layer outside [0, n_layers)");
  return KFL_ERR_RANGE;
}
inline Kv4Pool pool_of(const kfl_kv4_pool &p) {
  return {static_cast<uint8_t *>(p.pages), p.n_pages, log2_page(p.page_tokens), p.n_layers, p.n_kv_heads, p.head_dim};
}
inline Kv4Map map_of(const kfl_kv4_map &m) { return {m.table, m.lengths, m.refs, m.n_users, m.max_pages}; }

}  // namespace kfl
