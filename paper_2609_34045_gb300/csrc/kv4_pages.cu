// Pages of the 4-bit KV cache (include/kafila_kv4.h): reserving, forking, freeing, compacting, copying.
//
// Counting and table work is small and ordered (pages are given out lowest number first, so that a call's
// result is the same every time): one block of 1024 threads does a call's whole plan, a pass over refs being one
// coalesced read with a running count.  The pages' bytes, which are what a fork or a compaction costs, are moved by
// a second kernel over all SMs from the plan's list of moves: a compaction that moves 407 pages of 516 KB takes 76 us, 5.5 TB/s
// with its plan; eight beams' forks 11 us, of which the plan's chain of round trips is 6.
#include <algorithm>

#include "kv4.cuh"

namespace kfl {
namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_MOST = 1024;    // users of one call
constexpr int PLAN_LIST = 4096;    // new pages of one call that are listed in shared memory; more go through the workspace
constexpr int SCAN_PER_THREAD = 16;
constexpr int COPY_THREADS = 256;

// Workspace (int32): the number of moves, then source pages, destination pages, references of the moved pages;
// new numbers of the pages.
struct PagesWorkspace {
  int32_t *base;
  int n_pages;
  __host__ __device__ int list() const { return n_pages + PLAN_MOST; }
  __host__ __device__ int32_t *count() const { return base; }
  __host__ __device__ int32_t *src() const { return base + 4; }
  __host__ __device__ int32_t *dst() const { return src() + list(); }
  __host__ __device__ int32_t *moved_refs() const { return dst() + list(); }
  __host__ __device__ size_t bytes() const { return (size_t)(4 + 3 * (size_t)list()) * 4; }
};

struct PlanParams {
  Kv4Pool pool;
  Kv4Map map;
  const int32_t *users, *other;  // reserve: users, n_new; fork: src, dst; free: users
  int n;
  int32_t *table_out, *refs_out, *n_live;  // compact
  PagesWorkspace ws;
  int32_t *status;
};

// Exclusive sum over the block of one value per thread (all threads call); total: the sum.
__device__ __forceinline__ int block_scan(int v, int &total) {
  __shared__ int sums[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, s, off);
    if (lane >= off) s += o;
  }
  __syncthreads();  // (the sums of an earlier call have been read)
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
}

// One thread's run of refs in a pass of the whole block: SCAN_PER_THREAD neighbours from `at` (0 behind the end is
// told apart by the caller through n).
__device__ __forceinline__ void load_refs(const int32_t *refs, int at, int n, bool wide, int (&r)[SCAN_PER_THREAD]) {
  if (wide && at + SCAN_PER_THREAD <= n) {
#pragma unroll
    for (int i = 0; i < SCAN_PER_THREAD; i += 4) {
      const int4 q = *reinterpret_cast<const int4 *>(refs + at + i);
      r[i] = q.x, r[i + 1] = q.y, r[i + 2] = q.z, r[i + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < SCAN_PER_THREAD; ++i) r[i] = at + i < n ? refs[at + i] : 1;
  }
}

// The `want` lowest free pages into list[0..); returns how many there are (at most want).  r: the references of the
// thread's run in the first pass, loaded by the caller ahead of what it waits for in between.
__device__ int find_free(const int32_t *refs, int n_pages, int want, int32_t *list, int (&r)[SCAN_PER_THREAD]) {
  const bool wide = (reinterpret_cast<uintptr_t>(refs) & 15) == 0;
  int found = 0;
  for (int base = 0; base < n_pages && found < want; base += PLAN_THREADS * SCAN_PER_THREAD) {
    const int at = base + threadIdx.x * SCAN_PER_THREAD;
    int mine = 0, total;
    if (base > 0) load_refs(refs, at, n_pages, wide, r);
#pragma unroll
    for (int i = 0; i < SCAN_PER_THREAD; ++i) mine += r[i] == 0;
    int rank = found + block_scan(mine, total);
#pragma unroll
    for (int i = 0; i < SCAN_PER_THREAD; ++i)
      if (r[i] == 0) {
        if (rank < want) list[rank] = at + i;
        ++rank;
      }
    found += total;
  }
  __syncthreads();
  return min(found, want);
}
__device__ __forceinline__ void load_first_refs(const PlanParams &p, int (&r)[SCAN_PER_THREAD]) {
  load_refs(p.map.refs, threadIdx.x * SCAN_PER_THREAD, p.pool.n_pages, (reinterpret_cast<uintptr_t>(p.map.refs) & 15) == 0, r);
}

// Whether an earlier entry of the call's list (in shared memory) names the same user.
__device__ __forceinline__ bool named_before(const int *users, int i) {
  const int u = users[i];
  for (int j = 0; j < i; ++j)
    if (users[j] == u) return true;
  return false;
}

__global__ void __launch_bounds__(PLAN_THREADS) kv4_reserve_kernel(const PlanParams p) {
  __shared__ int s_user[PLAN_MOST], s_held[PLAN_MOST], s_end[PLAN_MOST], s_list[PLAN_LIST];
  pdl_launch_dependents();
  pdl_wait();
  const int i = threadIdx.x, P = p.pool.log2_tokens;
  int first_refs[SCAN_PER_THREAD];
  load_first_refs(p, first_refs);
  if (i < p.n) s_user[i] = p.users[i];
  __syncthreads();
  int need = 0, held = 0, length = 0, user = -1;
  if (i < p.n) {
    user = s_user[i];
    const int add = p.other[i];
    if (user < 0 || user >= p.map.n_users || add < 0 || named_before(s_user, i)) {
      report(p.status, KFL_BAD_USER);
      user = -1;
    } else {
      length = p.map.lengths[user];
      const int64_t to = (int64_t)length + add;
      if (length < 0 || to > (int64_t)p.map.max_pages << P || to > 0x7fffffff) {
        report(p.status, KFL_NO_PAGES);
        user = -1;
      } else {
        held = (int)(((int64_t)length + p.pool.page_tokens() - 1) >> P);
        need = (int)((to + p.pool.page_tokens() - 1) >> P) - held;
        length = (int)to;
      }
    }
  }
  int total;
  // (more pages than the pool has do not fit however many they are: the sum stays below 2^31)
  need = min(need, p.pool.n_pages + 1);
  const int offset = block_scan(need, total);
  const int want = min(total, p.pool.n_pages);
  int32_t *list = want <= PLAN_LIST ? s_list : p.ws.src();
  const int found = find_free(p.map.refs, p.pool.n_pages, want, list, first_refs);
  const bool fits = user >= 0 && (need == 0 || offset + need <= found);
  if (user >= 0 && !fits) report(p.status, KFL_NO_PAGES);
  if (fits) p.map.lengths[user] = length;
  if (i < p.n) {
    s_user[i] = fits ? user : -1;
    s_held[i] = held - offset;
    s_end[i] = offset + need;
  }
  __syncthreads();
  // page of rank r: the first user whose pages end behind it
  for (int r = i; r < found; r += PLAN_THREADS) {
    int lo = 0, hi = p.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_end[mid] > r)
        hi = mid;
      else
        lo = mid + 1;
    }
    if (s_user[lo] < 0) continue;
    const int page = list[r];
    p.map.table[(int64_t)s_user[lo] * p.map.max_pages + s_held[lo] + r] = page;
    p.map.refs[page] = 1;
  }
}

__global__ void __launch_bounds__(256) kv4_free_kernel(const PlanParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int i = blockIdx.x, user = p.users[i];
  bool again = false;
  for (int j = threadIdx.x; j < i; j += blockDim.x) again |= p.users[j] == user;
  if (__syncthreads_or(again) || user < 0 || user >= p.map.n_users) {
    if (threadIdx.x == 0) report(p.status, KFL_BAD_USER);
    return;
  }
  int32_t *row = p.map.table + (int64_t)user * p.map.max_pages;
  for (int j = threadIdx.x; j < p.map.max_pages; j += blockDim.x) {
    const int page = row[j];
    if (page == -1) continue;
    row[j] = -1;
    if (page < 0 || page >= p.pool.n_pages)
      report(p.status, KFL_BAD_PAGE);
    else
      atomicSub(p.map.refs + page, 1);
  }
  if (threadIdx.x == 0) p.map.lengths[user] = 0;
}

// The pairs' rows in steps of 32 columns: a step's old entries are all read before one of its new ones is written,
// so that a user may be source and destination at once; columns do not hang on one another.
__global__ void __launch_bounds__(PLAN_THREADS) kv4_fork_kernel(const PlanParams p) {
  __shared__ int s_src[PLAN_MOST], s_dst[PLAN_MOST], s_full[PLAN_MOST], s_new[PLAN_MOST], s_list[PLAN_MOST];
  __shared__ int s_columns, s_count;
  pdl_launch_dependents();
  pdl_wait();
  const int i = threadIdx.x, P = p.pool.log2_tokens;
  int first_refs[SCAN_PER_THREAD];
  load_first_refs(p, first_refs);
  if (i == 0) s_columns = s_count = 0;
  if (i < p.n) s_dst[i] = p.other[i];
  __syncthreads();
  int src = -1, dst = -1, length = 0, full = 0, need = 0, columns = 0;
  if (i < p.n) {
    src = p.users[i], dst = s_dst[i];
    if (src < 0 || src >= p.map.n_users || dst < 0 || dst >= p.map.n_users || named_before(s_dst, i)) {
      report(p.status, KFL_BAD_USER);
      dst = -1;
    } else if (src == dst) {
      dst = -1;
    } else {
      // (max_pages 2^24 of 128 tokens are 2^31 of them)
      const int64_t most = (int64_t)p.map.max_pages << P;
      length = (int)min((int64_t)max(0, p.map.lengths[src]), most);
      full = length >> P;
      need = (length & (p.pool.page_tokens() - 1)) != 0;
      const int64_t before = min((int64_t)max(0, p.map.lengths[dst]), most);
      columns = max(full + need, (int)((before + p.pool.page_tokens() - 1) >> P));
    }
  }
  int total;
  const int rank = block_scan(need, total);
  const int found = find_free(p.map.refs, p.pool.n_pages, total, s_list, first_refs);
  int page = -1;
  if (dst >= 0 && need) {
    if (rank >= found) {
      report(p.status, KFL_NO_PAGES);
      dst = -1, columns = 0;
    } else {
      page = s_list[rank];
      p.map.refs[page] = 1;
      const int end = p.map.table[(int64_t)src * p.map.max_pages + full];
      if (end < 0 || end >= p.pool.n_pages) {
        report(p.status, KFL_BAD_PAGE);
      } else {
        const int at = atomicAdd(&s_count, 1);
        p.ws.src()[at] = end, p.ws.dst()[at] = page;
      }
    }
  }
  if (i < p.n) {
    s_src[i] = src;
    s_full[i] = full;
    s_new[i] = page;
  }
  __syncthreads();  // (every thread has read s_dst, refs and the old rows' ends)
  if (i < p.n) s_dst[i] = dst;
  atomicMax(&s_columns, columns);
  __syncthreads();
  if (i == 0) *p.ws.count() = s_count;
  const int warp = i >> 5, lane = i & 31;
  for (int c0 = 0; c0 < s_columns; c0 += 32) {
    const int c = c0 + lane;
    int entry[PLAN_MOST / 32];
#pragma unroll
    for (int k = 0; k < PLAN_MOST / 32; ++k) {
      const int j = warp + 32 * k;
      entry[k] = -1;
      if (j >= p.n || s_dst[j] < 0 || c >= p.map.max_pages) continue;
      if (c < s_full[j])
        entry[k] = p.map.table[(int64_t)s_src[j] * p.map.max_pages + c];
      else if (c == s_full[j])
        entry[k] = s_new[j];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PLAN_MOST / 32; ++k) {
      const int j = warp + 32 * k;
      if (j >= p.n || s_dst[j] < 0 || c >= p.map.max_pages) continue;
      int32_t *at = p.map.table + (int64_t)s_dst[j] * p.map.max_pages + c;
      const int old = *at;
      if (old >= 0 && old < p.pool.n_pages) atomicSub(p.map.refs + old, 1);
      if (c < s_full[j] && entry[k] >= 0 && entry[k] < p.pool.n_pages) atomicAdd(p.map.refs + entry[k], 1);
      if (entry[k] != old) *at = entry[k];
    }
  }
  if (dst >= 0) p.map.lengths[dst] = length;
}

__global__ void __launch_bounds__(PLAN_THREADS) kv4_compact_kernel(const PlanParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int32_t *refs = p.map.refs;
  const int n = p.pool.n_pages;
  const bool wide = (reinterpret_cast<uintptr_t>(refs) & 15) == 0;
  int live = 0;
  for (int at = threadIdx.x * SCAN_PER_THREAD; at < n; at += PLAN_THREADS * SCAN_PER_THREAD) {
    int r[SCAN_PER_THREAD];
    load_refs(refs, at, n, wide, r);
#pragma unroll
    for (int i = 0; i < SCAN_PER_THREAD; ++i) live += at + i < n && r[i] != 0;
  }
  int n_live;
  block_scan(live, n_live);
  // holes below n_live and live pages from it on: as many of one as of the other
  int holes = 0, moved = 0;
  for (int base = 0; base < n; base += PLAN_THREADS * SCAN_PER_THREAD) {
    const int at = base + threadIdx.x * SCAN_PER_THREAD;
    int r[SCAN_PER_THREAD], mine = 0, total;
    load_refs(refs, at, n, wide, r);
    // both counts in one sum: a pass has 16384 pages
#pragma unroll
    for (int i = 0; i < SCAN_PER_THREAD; ++i)
      if (at + i < n) mine += at + i < n_live ? r[i] == 0 : (r[i] != 0) << 15;
    const int before = block_scan(mine, total);
    int hole = holes + (before & 0x7fff), source = moved + (before >> 15);
#pragma unroll
    for (int i = 0; i < SCAN_PER_THREAD; ++i) {
      if (at + i >= n) break;
      if (at + i < n_live ? r[i] == 0 : r[i] != 0) {
        if (at + i < n_live) {
          p.ws.dst()[hole++] = at + i;
        } else {
          p.ws.moved_refs()[source] = r[i];
          p.ws.src()[source++] = at + i;
        }
      }
    }
    holes += total & 0x7fff, moved += total >> 15;
  }
  __syncthreads();
  // (the counts' own buffer may be the one that was read: every read is done)
  if (p.refs_out != p.map.refs)
    for (int i = threadIdx.x; i < n; i += PLAN_THREADS) p.refs_out[i] = i < n_live ? refs[i] : 0;
  __syncthreads();
  for (int i = threadIdx.x; i < moved; i += PLAN_THREADS) {
    p.refs_out[p.ws.src()[i]] = 0;
    p.refs_out[p.ws.dst()[i]] = p.ws.moved_refs()[i];
  }
  if (threadIdx.x == 0) {
    *p.ws.count() = moved;
    if (p.n_live) *p.n_live = n_live;
  }
}

// A page's new number: its place among the moved ones (ascending), or its old one.
__device__ __forceinline__ int renumber(int page, const int32_t *src, const int32_t *dst, int moved) {
  if (moved == 0 || page < src[0]) return page;
  int lo = 0, hi = moved - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (src[mid] <= page)
      lo = mid;
    else
      hi = mid - 1;
  }
  return src[lo] == page ? dst[lo] : page;
}

struct CopyParams {
  Kv4Pool pool;
  const int32_t *src, *dst, *count;  // count NULL: n
  int n;
  // compaction: the table's entries under their new numbers
  const int32_t *table;
  int32_t *table_out;
  int64_t n_entries;
  int32_t *status;
};

// Moves, in units of one block's 16 KB: four 16-byte loads of a thread in flight, then their stores.
constexpr int COPY_AHEAD = 4;
constexpr int COPY_UNIT = COPY_THREADS * COPY_AHEAD * 16;

__global__ void __launch_bounds__(COPY_THREADS) kv4_copy_kernel(const CopyParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int n = p.count ? *p.count : p.n;
  for (int64_t i = (int64_t)blockIdx.x * COPY_THREADS + threadIdx.x; i < p.n_entries;
       i += (int64_t)gridDim.x * COPY_THREADS) {
    const int page = p.table[i];
    p.table_out[i] = page >= 0 ? renumber(page, p.src, p.dst, n) : page;
  }
  const size_t bytes = p.pool.page_bytes();
  const int units = (int)((bytes + COPY_UNIT - 1) / COPY_UNIT);
  for (int64_t w = blockIdx.x; w < (int64_t)n * units; w += gridDim.x) {
    const int move = (int)(w / units);
    const int from = p.src[move], to = p.dst[move];
    if (from < 0 || from >= p.pool.n_pages || to < 0 || to >= p.pool.n_pages) {
      if (threadIdx.x == 0) report(p.status, KFL_BAD_PAGE);
      continue;
    }
    const size_t at = (size_t)(w % units) * COPY_UNIT + threadIdx.x * 16;
    const uint8_t *src = p.pool.pages + from * bytes;
    uint8_t *dst = p.pool.pages + to * bytes;
    uint4 v[COPY_AHEAD];
#pragma unroll
    for (int j = 0; j < COPY_AHEAD; ++j)
      if (at + j * COPY_THREADS * 16 < bytes) v[j] = __ldcs(reinterpret_cast<const uint4 *>(src + at + j * COPY_THREADS * 16));
#pragma unroll
    for (int j = 0; j < COPY_AHEAD; ++j)
      if (at + j * COPY_THREADS * 16 < bytes) __stcs(reinterpret_cast<uint4 *>(dst + at + j * COPY_THREADS * 16), v[j]);
  }
}

cudaError_t launch_copy(const CopyParams &p, int64_t most_moves, cudaStream_t s) {
  const int64_t units = (int64_t)((p.pool.page_bytes() + COPY_UNIT - 1) / COPY_UNIT);
  const int64_t work = std::max(most_moves * units, (p.n_entries + COPY_THREADS - 1) / COPY_THREADS);
  const unsigned grid = (unsigned)std::min<int64_t>(std::max<int64_t>(work, 1), 152 * 8);
  return launch_chained(kv4_copy_kernel, grid, COPY_THREADS, 0, s, p);
}

int check_lists(const char *me, const kfl_kv4_pool *pool, const kfl_kv4_map *map, bool bytes, const int32_t *a,
                const int32_t *b, int n) {
  int rc = check_pool(pool, bytes, me);
  if (rc == KFL_OK) rc = check_map(map, me);
  if (rc != KFL_OK) return rc;
  if (n < 0 || (n > 0 && (!a || !b))) return bad_arg(me, "lists are needed");
  if (n > PLAN_MOST) {
    bad_arg(me, "more than 1024 users in one call");
    return KFL_ERR_RANGE;
  }
  return KFL_OK;
}
int check_workspace(const char *me, const void *workspace) {
  if (workspace && (reinterpret_cast<uintptr_t>(workspace) & 15) == 0) return KFL_OK;
  return bad_arg(me, "a 16-byte aligned workspace is needed");
}

PlanParams plan_of(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const int32_t *a, const int32_t *b, int n,
                   void *workspace, int32_t *status) {
  PlanParams p = {};
  p.pool = pool_of(*pool), p.map = map_of(*map);
  p.users = a, p.other = b, p.n = n;
  p.ws = {static_cast<int32_t *>(workspace), pool->n_pages};
  p.status = status;
  return p;
}

}  // namespace
}  // namespace kfl

using namespace kfl;

extern "C" int kfl_kv4_pages_workspace_bytes(const kfl_kv4_pool *pool, size_t *out) {
  const int rc = check_pool(pool, false, "kfl_kv4_pages_workspace_bytes");
  if (rc != KFL_OK) return rc;
  if (!out) return bad_arg("kfl_kv4_pages_workspace_bytes", "NULL pointer");
  *out = (PagesWorkspace{nullptr, pool->n_pages}.bytes() + 15) / 16 * 16;
  return KFL_OK;
}

extern "C" int kfl_kv4_reserve(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const int32_t *users,
                               const int32_t *n_new, int n, void *workspace, int32_t *status, void *cuda_stream) {
  const char *me = "kfl_kv4_reserve";
  int rc = check_lists(me, pool, map, false, users, n_new, n);
  if (rc == KFL_OK) rc = check_workspace(me, workspace);
  if (rc != KFL_OK || n == 0) return rc;
  const PlanParams p = plan_of(pool, map, users, n_new, n, workspace, status);
  return cuda_result(launch_chained(kv4_reserve_kernel, 1, PLAN_THREADS, 0, static_cast<cudaStream_t>(cuda_stream), p), me);
}

extern "C" int kfl_kv4_free(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const int32_t *users, int n,
                            int32_t *status, void *cuda_stream) {
  const char *me = "kfl_kv4_free";
  const int rc = check_lists(me, pool, map, false, users, users, n);
  if (rc != KFL_OK || n == 0) return rc;
  const PlanParams p = plan_of(pool, map, users, nullptr, n, nullptr, status);
  return cuda_result(launch_chained(kv4_free_kernel, n, 256, 0, static_cast<cudaStream_t>(cuda_stream), p), me);
}

extern "C" int kfl_kv4_fork(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const int32_t *src, const int32_t *dst,
                            int n, void *workspace, int32_t *status, void *cuda_stream) {
  const char *me = "kfl_kv4_fork";
  int rc = check_lists(me, pool, map, true, src, dst, n);
  if (rc == KFL_OK) rc = check_workspace(me, workspace);
  if (rc != KFL_OK || n == 0) return rc;
  const PlanParams p = plan_of(pool, map, src, dst, n, workspace, status);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = launch_chained(kv4_fork_kernel, 1, PLAN_THREADS, 0, s, p);
  if (e != cudaSuccess) return cuda_result(e, me);
  CopyParams c = {};
  c.pool = p.pool, c.src = p.ws.src(), c.dst = p.ws.dst(), c.count = p.ws.count(), c.status = status;
  return cuda_result(launch_copy(c, n, s), me);
}

extern "C" int kfl_kv4_compact(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int32_t *table_out,
                               int32_t *refs_out, int32_t *n_live, void *workspace, int32_t *status,
                               void *cuda_stream) {
  const char *me = "kfl_kv4_compact";
  int rc = check_lists(me, pool, map, true, nullptr, nullptr, 0);
  if (rc == KFL_OK) rc = check_workspace(me, workspace);
  if (rc != KFL_OK) return rc;
  if (!table_out || !refs_out) return bad_arg(me, "table_out and refs_out are needed");
  PlanParams p = plan_of(pool, map, nullptr, nullptr, 0, workspace, status);
  p.table_out = table_out, p.refs_out = refs_out, p.n_live = n_live;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = launch_chained(kv4_compact_kernel, 1, PLAN_THREADS, 0, s, p);
  if (e != cudaSuccess) return cuda_result(e, me);
  CopyParams c = {};
  c.pool = p.pool, c.src = p.ws.src(), c.dst = p.ws.dst(), c.count = p.ws.count(), c.status = status;
  c.table = map->table, c.table_out = table_out, c.n_entries = (int64_t)map->n_users * map->max_pages;
  return cuda_result(launch_copy(c, pool->n_pages / 2 + 1, s), me);
}

extern "C" int kfl_kv4_copy_pages(const kfl_kv4_pool *pool, const int32_t *src, const int32_t *dst, int n,
                                  int32_t *status, void *cuda_stream) {
  const char *me = "kfl_kv4_copy_pages";
  const int rc = check_pool(pool, true, me);
  if (rc != KFL_OK) return rc;
  if (n < 0 || (n > 0 && (!src || !dst))) return bad_arg(me, "lists are needed");
  if (n == 0) return KFL_OK;
  CopyParams c = {};
  c.pool = pool_of(*pool), c.src = src, c.dst = dst, c.n = n, c.status = status;
  return cuda_result(launch_copy(c, n, static_cast<cudaStream_t>(cuda_stream)), me);
}
