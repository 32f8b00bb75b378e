// The rows that stay of a cache that is cut (include/kafila_kv4_evict.h): kfl_kv4_select.
//
// The K greatest of a row of masses, ties to the lowest slot, out in ascending order.  A mass becomes a 32-bit key that
// orders like it; up to three passes over the keys (11, 11 and 10 bits) count how many have each value of the next bits, and so
// narrow down the K-th greatest key T, until a value's keys are all wanted; a last pass writes the slots with a key above T,
// and the first ones with T itself, each to the place that a running count gives it.
//
// What bounds it.  4 bytes a row in and 4 bytes a kept row out; some 30 instructions a key, and a chain of ten barriers.  The
// keys are read from memory once and stay in registers (a row longer than the registers of eight blocks: in shared memory, and
// are read again behind it).  A long row, of which there are too few to fill the SMs, is shared by a cluster of up to
// eight blocks, whose counts meet in distributed shared memory.
#include <algorithm>

#include "kv4_weights.cuh"
#include "prefill.cuh"

namespace kfl {
namespace {

constexpr int SEL_THREADS = 512, SEL_WARPS = SEL_THREADS / 32;
constexpr int SEL_BINS = 2048;
constexpr int SEL_ROOM = 40960;  // keys of a block in shared memory at most; more are read again
constexpr int SEL_USERS = 1024;

struct SelectParams {
  Kv4Pool pool;
  Kv4Map map;
  MassView mass;
  const int32_t *users;
  int n, budget, first, recent;
  int32_t *rows, *counts, *status;
  int room, cluster;  // keys in shared memory (PER 0), blocks of a row
  int64_t items;      // layers * n * heads
};

// Keys order as the masses do (NaN above all, both zeros alike).
__device__ __forceinline__ uint32_t mass_key(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint32_t ld_cluster(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ uint4 ld_cluster4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

// Exclusive sum over the block of one value per thread; total: the sum.
__device__ __forceinline__ int scan_block(int v, int &total, int *sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, s, off);
    if (lane >= off) s += o;
  }
  if (lane == 31) sums[warp] = s;
  __syncthreads();
  int w = lane < SEL_WARPS ? sums[lane] : 0;
#pragma unroll
  for (int off = 1; off < SEL_WARPS; off <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, w, off);
    if (lane >= off) w += o;
  }
  total = __shfl_sync(0xffffffffu, w, SEL_WARPS - 1);
  const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
  return s - v + (warp ? before : 0);
}

// PER: keys of a thread, in registers; 0: any number, in shared memory and behind it.
template <int PER>
__global__ void __launch_bounds__(SEL_THREADS) kv4_select_kernel(const SelectParams p) {
  extern __shared__ uint32_t keys[];  // [room]
  __shared__ alignas(16) uint32_t hist[2][SEL_BINS];  // by turns: the last pass's counts are read while the next one's are made
  __shared__ int sums[SEL_WARPS], above[SEL_WARPS], ties[SEL_WARPS];
  __shared__ int found[3];   // the bin, how many of it are wanted, how many there are
  __shared__ int totals[2];  // of this block: above the threshold, at it
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = p.cluster > 1 ? (int)cluster_ctarank() : 0, C = p.cluster;
  const int heads = p.pool.n_kv_heads;
  *reinterpret_cast<uint4 *>(&hist[0][4 * tid]) = *reinterpret_cast<uint4 *>(&hist[1][4 * tid]) = make_uint4(0, 0, 0, 0);
  pdl_launch_dependents();
  pdl_wait();
  const auto sync = [&]() {
    if (C > 1)
      cluster_sync_all();
    else
      __syncthreads();
  };
  for (int64_t item = blockIdx.x / C; item < p.items; item += gridDim.x / C) {
    const int64_t row_of = item / heads;
    const int head = (int)(item - row_of * heads), layer = (int)(row_of / p.n), i = (int)(row_of - (int64_t)layer * p.n);
    const int user = p.users[i];
    const bool known = user >= 0 && user < p.map.n_users;
    const int length = known ? min(max(0, p.map.lengths[user]), p.map.max_pages << p.pool.log2_tokens) : 0;
    int32_t *out = p.rows + item * p.budget;
    if (layer == 0 && head == 0 && rank == 0 && tid == 0) {
      p.counts[i] = min(length, p.budget);
      if (!known) report(p.status, KFL_BAD_USER);
    }
    if (length <= p.budget) {  // (the whole cluster alike)
      for (int j = rank * SEL_THREADS + tid; j < p.budget; j += C * SEL_THREADS) out[j] = j < length ? j : -1;
      continue;
    }
    const int m = length - p.first - p.recent, K = p.budget - p.first - p.recent;
    // ---- this block's slice of the m rows between, a run of whole 32s for each warp
    const float *mass = p.mass.row(layer, user, head) + p.first;
    const int seg = ((m + C * SEL_WARPS - 1) / (C * SEL_WARPS) + 31) / 32 * 32;
    const int w0 = (int)min(((int64_t)rank * SEL_WARPS + warp) * seg, (int64_t)m), w1 = min(w0 + seg, m);
    uint32_t mine[PER > 0 ? PER : 1];
    const int begin = (int)min((int64_t)rank * SEL_WARPS * seg, (int64_t)m);
    const auto stored = [&](int j) { return j - begin < p.room ? keys[j - begin] : mass_key(mass[j]); };
    // every key of this thread: f(slot less `first`, key, whether there is one)
    const auto each = [&](auto f) {
      if constexpr (PER > 0) {
#pragma unroll
        for (int k = 0; k < PER; ++k)
          if (32 * k < seg) f(w0 + 32 * k + lane, mine[k], w0 + 32 * k + lane < w1);
      } else {
        for (int j0 = w0; j0 < w1; j0 += 32) f(j0 + lane, j0 + lane < w1 ? stored(j0 + lane) : 0u, j0 + lane < w1);
      }
    };
    if (K > 0) {
      if constexpr (PER > 0) {
        float v[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) v[k] = w0 + 32 * k + lane < w1 ? mass[w0 + 32 * k + lane] : 0.f;
#pragma unroll
        for (int k = 0; k < PER; ++k) mine[k] = mass_key(v[k]);
      } else {
#pragma unroll 8
        for (int j = w0 + lane; j < min(w1, begin + p.room); j += 32) keys[j - begin] = mass_key(mass[j]);
        __syncwarp();
      }
    }
    for (int j = rank * SEL_THREADS + tid; j < p.first + p.recent; j += C * SEL_THREADS)
      out[j < p.first ? j : K + j] = j < p.first ? j : m + j;
    if (K == 0) continue;
    uint32_t T = 0;
    int want = K;
    bool all = false;  // of the last bin
    __syncthreads();   // (the counts are zero)
#pragma unroll 1
    for (int pass = 0; pass < 3 && !all; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
      uint32_t *counts = hist[pass & 1];
      each([&](int, uint32_t k, bool is) {
        if (is && (pass == 0 || k >> (shift + bits) == T >> (shift + bits))) atomicAdd(&counts[k >> shift & ((1u << bits) - 1)], 1u);
      });
      sync();
      // four bins a thread, of all blocks; the one in which the `want`-th greatest lies
      const uint32_t at = smem_addr(&counts[4 * tid]);
      uint4 b = *reinterpret_cast<const uint4 *>(&counts[4 * tid]);
      for (int r = 1; r < C; ++r) {
        const uint4 o = ld_cluster4(map_to_rank(at, (rank + r) & (C - 1)));
        b.x += o.x, b.y += o.y, b.z += o.z, b.w += o.w;
      }
      int total;
      const int own = b.x + b.y + b.z + b.w, before = scan_block(own, total, sums);
      int greater = total - before - own;
      if (greater < want && greater + own >= want) {
        const int four[4] = {(int)b.x, (int)b.y, (int)b.z, (int)b.w};
#pragma unroll
        for (int j = 3; j >= 0; --j) {
          if (greater < want && greater + four[j] >= want) found[0] = 4 * tid + j, found[1] = want - greater, found[2] = four[j];
          greater += four[j];
        }
      }
      // the other counts are free: every block has been here since it read them (zero again for the next pass, or row)
      *reinterpret_cast<uint4 *>(&hist[(pass & 1) ^ 1][4 * tid]) = make_uint4(0, 0, 0, 0);
      __syncthreads();
      T |= (uint32_t)found[0] << shift;
      want = found[1];
      all = want == found[2];
    }
    // (all of the last bin: its keys are those from T on, whatever their other bits)
    if (all && T > 0) --T, want = 0;
    // ---- how many of each warp's run are above T, and at it
    int g = 0, t = 0;
    each([&](int, uint32_t k, bool is) { g += is && k > T, t += is && k == T; });
    g = __reduce_add_sync(0xffffffffu, g), t = __reduce_add_sync(0xffffffffu, t);
    if (lane == 0) above[warp] = g, ties[warp] = t;
    __syncthreads();
    if (C > 1 && warp == 0) {
      const int a = __reduce_add_sync(0xffffffffu, lane < SEL_WARPS ? above[lane] : 0);
      const int b = __reduce_add_sync(0xffffffffu, lane < SEL_WARPS ? ties[lane] : 0);
      if (lane == 0) totals[0] = a, totals[1] = b;
    }
    int g0 = lane < warp ? above[lane] : 0, t0 = lane < warp ? ties[lane] : 0;
    sync();
    if (C > 1 && lane < rank) {
      g0 += ld_cluster(map_to_rank(smem_addr(&totals[0]), lane));
      t0 += ld_cluster(map_to_rank(smem_addr(&totals[1]), lane));
    }
    g0 = __reduce_add_sync(0xffffffffu, g0), t0 = __reduce_add_sync(0xffffffffu, t0);
    // ---- the slots, each at its place
    each([&](int j, uint32_t k, bool is) {
      const unsigned over = __ballot_sync(0xffffffffu, is && k > T), at = __ballot_sync(0xffffffffu, is && k == T);
      const unsigned below = (1u << lane) - 1;
      const int tie = t0 + __popc(at & below);
      if ((over >> lane & 1) || ((at >> lane & 1) && tie < want)) out[p.first + g0 + __popc(over & below) + min(tie, want)] = p.first + j;
      g0 += __popc(over), t0 += __popc(at);
    });
    // the counts of the last pass, too, for the next row (the others have read them, and the totals)
    sync();
    *reinterpret_cast<uint4 *>(&hist[0][4 * tid]) = *reinterpret_cast<uint4 *>(&hist[1][4 * tid]) = make_uint4(0, 0, 0, 0);
  }
}

template <int PER>
cudaError_t launch(const SelectParams &p, cudaStream_t s) {
  const size_t smem = PER > 0 ? 0 : (size_t)p.room * 4;
  if (PER == 0) {
    static SmemOptIn opt_in;
    const cudaError_t e = opt_in(reinterpret_cast<const void *>(&kv4_select_kernel<PER>), SEL_ROOM * 4);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.cluster, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(std::min<int64_t>(p.items, 1 << 20) * p.cluster)), cfg.blockDim = dim3(SEL_THREADS);
  cfg.dynamicSmemBytes = smem, cfg.stream = s;
  cfg.attrs = attr, cfg.numAttrs = p.cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kv4_select_kernel<PER>, p);
}

}  // namespace
}  // namespace kfl

using namespace kfl;

extern "C" int kfl_kv4_select(const kfl_kv4_pool *pool, const kfl_kv4_map *map, const kfl_kv4_mass *mass,
                              const int32_t *users, int n, int budget, int first, int recent, int32_t *rows,
                              int32_t *counts, int32_t *status, void *cuda_stream) {
  const char *me = "kfl_kv4_select";
  int rc = check_pool(pool, false, me);
  if (rc == KFL_OK) rc = check_map(map, me);
  if (rc != KFL_OK) return rc;
  if (n < 0) return bad_arg(me, "n is not negative");
  if (n > SEL_USERS) {
    bad_arg(me, "more than 1024 users in one call");
    return KFL_ERR_RANGE;
  }
  if (budget < 1 || budget > (1 << 26) || first < 0 || recent < 0 || first > budget || recent > budget - first)
    return bad_arg(me, "budget is 1..2^26, first and recent are not negative and together at most budget");
  if ((int64_t)map->max_pages * pool->page_tokens > (1 << 26)) return bad_arg(me, "max_pages * page_tokens is at most 2^26");
  if (n == 0) return KFL_OK;
  if (!mass_valid(mass) || !users || !rows || !counts) return bad_arg(me, "mass, users, rows and counts are needed");
  SelectParams p = {};
  p.pool = pool_of(*pool), p.map = map_of(*map), p.mass = view_of(*mass);
  p.users = users, p.n = n, p.budget = budget, p.first = first, p.recent = recent;
  p.rows = rows, p.counts = counts, p.status = status;
  p.items = (int64_t)pool->n_layers * n * pool->n_kv_heads;
  // blocks of a row: as many as leave a thread no more than 8 keys, while the rows do not fill the SMs twice; else as few
  // as hold the keys in registers, 32 a thread at most
  const int64_t most = std::max<int64_t>((int64_t)map->max_pages * pool->page_tokens - first - recent, 1);
  const auto per_thread = [&]() { return (most + (int64_t)p.cluster * SEL_THREADS - 1) / (p.cluster * SEL_THREADS); };
  p.cluster = 1;
  while (p.cluster < 8 && per_thread() > (p.items * p.cluster < 2 * 152 ? 8 : 32)) p.cluster *= 2;
  const int64_t per = per_thread();
  p.room = SEL_ROOM;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return cuda_result(per <= 8 ? launch<8>(p, s) : per <= 16 ? launch<16>(p, s) : per <= 32 ? launch<32>(p, s) : launch<0>(p, s), me);
}
