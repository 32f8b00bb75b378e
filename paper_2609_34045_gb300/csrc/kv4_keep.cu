// Rows of a user's cache brought together in place (include/kafila_kv4_evict.h): kfl_kv4_keep.
//
// A plan kernel (one block) checks the users and gives those whose rows move inside pages that others hold too their new
// pages, lowest first.  The moving is a second kernel over all (user, layer, KV head): slot first + j gets the row of slot list[j].
// Since list[j] >= first + j, a walk in ascending slots may read and write the same pages: what a chunk of rows
// writes lies behind all that later chunks read, and within a chunk every row is loaded before one is stored.  The last
// block to be done with a user writes its table row, its counts of holders and its length.
//
// What bounds it.  The kept rows' bytes, read and written (9/8 head_dim each way), through rows of 64 and 8 bytes: eight users of
// 8192 rows cut to half, 14 layers of 4 heads of 128, 134 us with the reservation after it, of which the moving takes some 120: 428 MB
// read and 237 MB written, 5.6 TB/s.  Read is what lines of 128 bytes of codes come to, two rows in each (191 bytes a kept row for its
// 128), with sectors of parameters (30), masses (8) and the lists (4): 427 MB; in sectors of 32 bytes all through it would be 312.  (Two
// chunks ahead instead of one: the same.)  With a few rows (accepted drafts) the chain of round trips, plan, list, page, row: 11 us with the reservation.  The next chunk's rows are under way, and the one
// after's addresses looked up, while a chunk is stored.
#include <algorithm>

#include "kv4_weights.cuh"

namespace kfl {
namespace {

constexpr int KEEP_THREADS = 256, KEEP_MOST = 1024, KEEP_PLAN = 1024;
constexpr int KEEP_CHUNK = KEEP_THREADS / 4;  // rows: four threads each

struct KeepParams {
  Kv4Pool pool;
  Kv4Map map;
  const int32_t *users, *first, *counts;
  kfl_kv4_rows rows;
  MassView mass;
  int n;
  // the workspace (kfl_kv4_pages_workspace_bytes), three parts of n_pages + 1024 places
  int32_t *fresh, *tickets;   // new pages, user after user; [n] blocks that are done with a user
  int32_t *place, *n_fresh;   // the new pages' places in their user's row of the table, ascending; [n] how many
  int32_t *start;             // [n]: where a user's are in both lists, -1: it is not touched
  int32_t *status;
};

// What is asked of user i: the slots from `first` on get `count` rows.  Pages from `begin` on change, of `held` those
// from `need` on go.
struct Cut {
  int user, first, count, length, begin, need, held;
};
__device__ __forceinline__ Cut cut_of(const KeepParams &p, int i) {
  Cut c;
  const int P = p.pool.log2_tokens;
  c.user = p.users[i], c.first = p.first ? p.first[i] : 0, c.count = p.counts[i], c.length = 0;
  if (c.user >= 0 && c.user < p.map.n_users) c.length = min(max(0, p.map.lengths[c.user]), p.map.max_pages << P);
  c.begin = c.first >> P;
  c.need = (int)(((int64_t)c.first + c.count + p.pool.page_tokens() - 1) >> P);
  c.held = (int)(((int64_t)c.length + p.pool.page_tokens() - 1) >> P);
  return c;
}

__global__ void __launch_bounds__(KEEP_PLAN) kv4_keep_plan_kernel(const KeepParams p) {
  __shared__ int user[KEEP_MOST], news[KEEP_MOST], at[KEEP_MOST];
  __shared__ int3 pages[KEEP_MOST];  // (begin, need, held)
  __shared__ int sums[32];
  pdl_launch_dependents();
  pdl_wait();
  const int i = threadIdx.x, warp = i >> 5, lane = i & 31;
  Cut c = {};
  if (i < p.n) c = cut_of(p, i), user[i] = c.user;
  __syncthreads();
  // ---- which users change at all
  if (i < p.n) {
    bool again = false;
    for (int j = 0; j < i; ++j) again |= user[j] == c.user;
    int bad = 0;
    if (c.user < 0 || c.user >= p.map.n_users || again)
      bad = KFL_BAD_USER;
    else if (c.first < 0 || c.count < 0 || c.count > p.rows.most || (int64_t)c.first + c.count > c.length)
      bad = KFL_BAD_POSITION;
    if (bad) report(p.status, bad);
    news[i] = bad || c.first + c.count == c.length ? -1 : 0;
    pages[i] = make_int3(c.begin, c.need, c.held);
  }
  __syncthreads();
  // ---- the pages that rows move into and others hold too, a warp per user
  for (int k = warp; k < p.n; k += KEEP_PLAN / 32) {
    if (news[k] < 0) continue;
    const int3 c = pages[k];
    const int32_t *row = p.map.table + (int64_t)user[k] * p.map.max_pages;
    int n = 0;
    bool bad = false;
#pragma unroll 4
    for (int j = c.x + lane; j < c.z; j += 32) {
      const int page = row[j];
      if (page < 0 || page >= p.pool.n_pages)
        bad = true;
      else
        n += j < c.y && p.map.refs[page] > 1;
    }
    n = __reduce_add_sync(0xffffffffu, n);
    bad = __any_sync(0xffffffffu, bad);
    if (lane == 0) {
      if (bad) report(p.status, KFL_BAD_PAGE);
      news[k] = bad ? -1 : min(n, p.pool.n_pages + 1);
    }
  }
  __syncthreads();
  // ---- their places among the new pages (more than there are do not fit, however many: the sum stays below 2^31)
  const auto scan = [&](int v, int &total) {
    int s = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, s, off);
      if (lane >= off) s += o;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = s;
    __syncthreads();
    int w = sums[lane];
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, w, off);
      if (lane >= off) w += o;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    return s - v + (warp ? before : 0);
  };
  const int mine = i < p.n ? news[i] : -1;
  int total;
  const int offset = scan(max(mine, 0), total);
  // ---- free pages, lowest first, as many as are wanted
  const int want = min(total, p.pool.n_pages);
  int found = 0;
  for (int base = 0; base < p.pool.n_pages && found < want; base += KEEP_PLAN * 4) {
    int r[4], free = 0, here;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      r[j] = base + 4 * i + j < p.pool.n_pages ? p.map.refs[base + 4 * i + j] : 1;
      free += r[j] == 0;
    }
    int rank = found + scan(free, here);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (r[j] == 0) {
        if (rank < want) p.fresh[rank] = base + 4 * i + j;
        ++rank;
      }
    found += here;
  }
  found = min(found, want);
  const bool fits = mine >= 0 && (mine == 0 || offset + mine <= found);
  if (mine >= 0 && !fits) report(p.status, KFL_NO_PAGES);
  if (i < p.n) {
    at[i] = fits ? offset : -1;
    p.start[i] = at[i], p.n_fresh[i] = fits ? mine : 0, p.tickets[i] = 0;
  }
  __syncthreads();
  // ---- which places they take
  for (int k = warp; k < p.n; k += KEEP_PLAN / 32) {
    if (at[k] < 0 || news[k] == 0) continue;
    const int3 c = pages[k];
    const int32_t *row = p.map.table + (int64_t)user[k] * p.map.max_pages;
    int to = at[k];
    for (int j0 = c.x; j0 < c.y; j0 += 32) {
      const int j = j0 + lane;
      const unsigned shared = __ballot_sync(0xffffffffu, j < c.y && p.map.refs[row[min(j, c.y - 1)]] > 1);
      if (shared >> lane & 1) p.place[to + __popc(shared & ((1u << lane) - 1))] = j;
      to += __popc(shared);
    }
  }
}

// A row's bytes, a quarter in each of four threads: 16 of its K codes and 16 of its V codes (head_dim 128), or 16 of either (64);
// in the first two threads also its parameters (K, V), in the third its mass.
template <int HD>
struct RowPart {
  uint4 a, b;
  uint2 par;
  float mass;
};
template <int HD>
__device__ __forceinline__ size_t codes_at(const Kv4Pool &pool, int page, int layer, int head, int slot, int sub) {
  const size_t block = (((size_t)page * pool.n_layers + layer) * pool.n_kv_heads + head) * (size_t)pool.block_bytes();
  if (HD == 128) return block + slot * 64 + sub * 16;                                      // (V's are code_bytes on)
  return block + (sub >> 1) * pool.code_bytes() + slot * 32 + (sub & 1) * 16;
}
template <int HD>
__device__ __forceinline__ size_t params_at(const Kv4Pool &pool, int page, int layer, int head, int slot, int which) {
  const size_t block = (((size_t)page * pool.n_layers + layer) * pool.n_kv_heads + head) * (size_t)pool.block_bytes();
  return block + 2 * pool.code_bytes() + which * pool.param_bytes() + slot * (HD / 16);
}

template <int HD>
__global__ void __launch_bounds__(KEEP_THREADS) kv4_keep_kernel(const KeepParams p) {
  __shared__ int last;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, sub = tid & 3, P = p.pool.log2_tokens, heads = p.pool.n_kv_heads;
  const int64_t per_user = (int64_t)p.pool.n_layers * heads, items = per_user * p.n;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t row_of = item / heads;
    const int head = (int)(item - row_of * heads), layer = (int)(row_of / p.n), i = (int)(row_of - (int64_t)layer * p.n);
    const int start = p.start[i];
    if (start < 0) continue;
    const Cut c = cut_of(p, i);
    const int n_fresh = p.n_fresh[i], stop = c.first + c.count;
    const int32_t *row = p.map.table + (int64_t)c.user * p.map.max_pages;
    const int32_t *place = p.place + start, *fresh = p.fresh + start;
    const int32_t *list = p.rows.data + layer * p.rows.layer_stride + i * p.rows.seq_stride + head * p.rows.head_stride;
    float *mass = p.mass.data ? p.mass.row(layer, c.user, head) : nullptr;
    // the page that holds the page place j afterwards
    const auto page_for = [&](int j) {
      if (n_fresh == 0) return row[j];
      int lo = 0, hi = n_fresh;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (place[mid] < j)
          lo = mid + 1;
        else
          hi = mid;
      }
      return lo < n_fresh && place[lo] == j ? fresh[lo] : row[j];
    };
    // (what stands before the first row goes along into a new page)
    const int s0 = n_fresh > 0 && place[0] == c.begin ? c.begin << P : c.first;
    const int mask = p.pool.page_tokens() - 1;
    // a thread's row of a chunk: its slot, the slot that it comes from, then both pages (a page of -1: nothing moves)
    struct Move {
      int to, from, to_page, from_page;
    };
    const auto look = [&](int chunk) {  // the list's entry
      Move m;
      m.to = s0 + chunk * KEEP_CHUNK + (tid >> 2);
      m.to_page = m.from_page = -1;
      if (m.to >= stop) m.to = -1;
      m.from = m.to < c.first ? m.to : list[m.to - c.first];
      return m;
    };
    const auto locate = [&](Move &m) {
      if (m.to < 0) return;
      if (m.from < m.to || m.from >= c.length) {
        if (sub == 0) report(p.status, KFL_BAD_POSITION);
        m.from = m.to;
      }
      m.from_page = row[m.from >> P];
      m.to_page = page_for(m.to >> P);
      if (m.from_page == m.to_page && m.from == m.to) m.to = -1;
    };
    const auto load = [&](const Move &m, RowPart<HD> &r) {
      if (m.to < 0) return;
      const int slot = m.from & mask;
      const uint8_t *at = p.pool.pages + codes_at<HD>(p.pool, m.from_page, layer, head, slot, sub);
      r.a = *reinterpret_cast<const uint4 *>(at);
      if (HD == 128) r.b = *reinterpret_cast<const uint4 *>(at + p.pool.code_bytes());
      if (sub < 2) {
        const uint8_t *par = p.pool.pages + params_at<HD>(p.pool, m.from_page, layer, head, slot, sub);
        if (HD == 128)
          r.par = *reinterpret_cast<const uint2 *>(par);
        else
          r.par.x = *reinterpret_cast<const uint32_t *>(par);
      } else if (sub == 2 && mass) {
        r.mass = mass[m.from];
      }
    };
    const auto store = [&](const Move &m, const RowPart<HD> &r) {
      if (m.to < 0) return;
      const int slot = m.to & mask;
      uint8_t *at = p.pool.pages + codes_at<HD>(p.pool, m.to_page, layer, head, slot, sub);
      *reinterpret_cast<uint4 *>(at) = r.a;
      if (HD == 128) *reinterpret_cast<uint4 *>(at + p.pool.code_bytes()) = r.b;
      if (sub < 2) {
        uint8_t *par = p.pool.pages + params_at<HD>(p.pool, m.to_page, layer, head, slot, sub);
        if (HD == 128)
          *reinterpret_cast<uint2 *>(par) = r.par;
        else
          *reinterpret_cast<uint32_t *>(par) = r.par.x;
      } else if (sub == 2 && mass) {
        mass[m.to] = r.mass;
      }
    };
    // ---- chunk after chunk: stored, the next one's rows loaded, the one after's pages and the one after that's entries
    // looked up.  (Loads of the next chunk are from slots at or behind its own: no store of this one reaches them)
    const int chunks = (stop - s0 + KEEP_CHUNK - 1) / KEEP_CHUNK;
    Move now = look(0), next = look(1), later = look(2);
    RowPart<HD> r, r_next;
    locate(now);
    load(now, r);
    locate(next);
    for (int k = 0; k < chunks; ++k) {
      const Move after = look(k + 3);
      load(next, r_next);
      locate(later);
      __syncthreads();  // (every thread has loaded this chunk's rows)
      store(now, r);
      now = next, next = later, later = after, r = r_next;
    }
    __syncthreads();
    if (mass)
      for (int s = stop + tid; s < c.length; s += KEEP_THREADS) mass[s] = 0.f;
    if (tid == 0) last = atom_add_acq_rel(reinterpret_cast<unsigned *>(p.tickets + i), 1u) == (unsigned)(per_user - 1);
    __syncthreads();
    if (last) {
      int32_t *to = p.map.table + (int64_t)c.user * p.map.max_pages;
      for (int j = tid; j < n_fresh; j += KEEP_THREADS) {
        atomicSub(p.map.refs + to[place[j]], 1);
        to[place[j]] = fresh[j];
        p.map.refs[fresh[j]] = 1;
      }
      for (int j = c.need + tid; j < c.held; j += KEEP_THREADS) {
        atomicSub(p.map.refs + to[j], 1);
        to[j] = -1;
      }
      if (tid == 0) p.map.lengths[c.user] = stop;
    }
    __syncthreads();  // (before `last` is written again)
  }
}

}  // namespace
}  // namespace kfl

using namespace kfl;

extern "C" int kfl_kv4_keep(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const int32_t *users,
                            const kfl_kv4_rows *rows, const int32_t *first, const int32_t *counts,
                            const kfl_kv4_mass *mass, int n, void *workspace, int32_t *status, void *cuda_stream) {
  const char *me = "kfl_kv4_keep";
  int rc = check_pool(pool, true, me);
  if (rc == KFL_OK) rc = check_map(map, me);
  if (rc != KFL_OK) return rc;
  if (n < 0) return bad_arg(me, "n is not negative");
  if (n > KEEP_MOST) {
    bad_arg(me, "more than 1024 users in one call");
    return KFL_ERR_RANGE;
  }
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return bad_arg(me, "a 16-byte aligned workspace is needed");
  if ((int64_t)map->max_pages * pool->page_tokens > (1 << 26)) return bad_arg(me, "max_pages * page_tokens is at most 2^26");
  if (n == 0) return KFL_OK;
  if (!users || !counts || !rows || rows->most < 0 || (rows->most > 0 && !rows->data))
    return bad_arg(me, "users, rows and counts are needed");
  if (mass && !mass_valid(mass)) return bad_arg(me, "a mass has aligned data");
  KeepParams p = {};
  p.pool = pool_of(*pool), p.map = map_of(*map);
  p.users = users, p.first = first, p.counts = counts, p.rows = *rows, p.n = n, p.status = status;
  if (mass) p.mass = view_of(*mass);
  const size_t part = (size_t)pool->n_pages + KEEP_MOST;
  int32_t *ws = static_cast<int32_t *>(workspace);
  p.fresh = ws, p.tickets = ws + pool->n_pages;
  p.place = ws + part, p.n_fresh = p.place + pool->n_pages;
  p.start = ws + 2 * part;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = launch_chained(kv4_keep_plan_kernel, 1, KEEP_PLAN, 0, s, p);
  if (e != cudaSuccess) return cuda_result(e, me);
  const unsigned grid = (unsigned)std::min<int64_t>((int64_t)pool->n_layers * pool->n_kv_heads * n, 152 * 8);
  return cuda_result(pool->head_dim == 128 ? launch_chained(kv4_keep_kernel<128>, grid, KEEP_THREADS, 0, s, p)
                                           : launch_chained(kv4_keep_kernel<64>, grid, KEEP_THREADS, 0, s, p),
                     me);
}
