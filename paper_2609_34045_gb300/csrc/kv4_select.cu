// The rows that stay of a cache that is cut (include/kafila_kv4_evict.h): kfl_kv4_select.
//
// The K greatest of a row of masses, ties to the lowest slot, out in ascending order.  A mass becomes a 32-bit key that
// orders like it; up to three passes over the keys (11, 11 and 10 bits) count how many have each value of the next bits, and so
// narrow down the K-th greatest key T, until a value's keys are all wanted; a last pass writes the slots with a key above T,
// and the first ones with T itself, each to the place that a running count gives it.
//
// What bounds it.  4 bytes a row in and 4 bytes a kept row out; the instructions a key (some 40), and a chain of ten barriers: 896 rows
// of up to 8192 keys 20 us (in two waves: five blocks an SM are 760), four rows of 4096 keys 4.4, eight of 131072 16.3 (two thousand clocks each to load, to count a pass, and
// twice that to read the other blocks' counts).  The
// keys are read from memory once and stay in shared memory, neighbours with one thread, so that a place in the output costs a
// thread one sum over the block and not a vote a key (128 instructions a key with the votes).  (A row longer than the shared
// memory of eight blocks is read again in each pass.)  A long row, of which there are too few to fill the SMs, is shared by a
// cluster of up to eight blocks, whose counts meet in distributed shared memory.
#include <algorithm>
#include <type_traits>

#include "attn_core.cuh"  // cp_async16
#include "kv4_weights.cuh"
#include "prefill.cuh"

namespace kfl {
namespace {

constexpr int SEL_BINS = 2048;
constexpr int SEL_BYTES = 192 << 10;  // of keys in a block's shared memory
constexpr int SEL_USERS = 1024;

struct SelectParams {
  Kv4Pool pool;
  Kv4Map map;
  MassView mass;
  const int32_t *users;
  int n, budget, first, recent;
  int32_t *rows, *counts, *status;
  int cluster;    // blocks of a row
  int room;       // keys of a thread that fit shared memory
  int wide;       // rows of masses start on 16 bytes
  int log2_cluster;
};

// Keys order as the masses do.  The sum makes both zeros one, and of every NaN the positive one, above all numbers.  No
// mass has a key below 2^22.
__device__ __forceinline__ uint32_t mass_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
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

// One more in a count of shared memory, if so (predicated: a branch a key costs more).
__device__ __forceinline__ void count_if(uint32_t at, bool so) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p red.shared.add.u32 [%0], 1;\n\t}" ::"r"(at), "r"((uint32_t)so) : "memory");
}

// Sum of one value per thread over the threads before this one; total: over the block.
template <int WARPS>
__device__ __forceinline__ uint32_t scan_block(uint32_t v, uint32_t &total, uint32_t *sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t s = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, s, off);
    if (lane >= off) s += o;
  }
  if (lane == 31) sums[warp] = s;
  __syncthreads();
  const uint32_t w = lane < WARPS ? sums[lane] : 0;
  total = __reduce_add_sync(0xffffffffu, w);
  return s - v + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
}

// A thread's keys of n (at most 2^26) for 2^log2_threads: an odd multiple of four, so that the threads of a warp read theirs
// from different banks.
__host__ __device__ inline int keys_per_thread(int n, int log2_threads) {
  return ((((n - 1) >> log2_threads) + 4) & ~3) | 4;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 5 : 1) kv4_select_kernel(const SelectParams p) {
  extern __shared__ __align__(16) uint32_t keys[];  // [thread][per]
  constexpr int WARPS = THREADS / 32, BINS = SEL_BINS / THREADS, LOG2 = THREADS == 256 ? 8 : 9;
  // of clusters by turns: the last pass's counts are read by other blocks while the next one's are made
  constexpr int TURNS = THREADS == 512 ? 2 : 1;
  __shared__ alignas(16) uint32_t hist[TURNS][SEL_BINS];
  __shared__ uint32_t sums[2][WARPS];
  __shared__ int found[3];        // the bin, how many of it are wanted, how many there are
  __shared__ uint32_t totals[2];  // of this block: above the threshold, at it
  const int tid = threadIdx.x;
  const int rank = p.cluster > 1 ? (int)cluster_ctarank() : 0, C = p.cluster;
  const int heads = p.pool.n_kv_heads;
  const auto clear = [&](uint32_t *counts) {
#pragma unroll
    for (int j = 0; j < BINS; j += 4) *reinterpret_cast<uint4 *>(&counts[BINS * tid + j]) = make_uint4(0, 0, 0, 0);
  };
  clear(hist[0]), clear(hist[TURNS - 1]);
  pdl_launch_dependents();
  pdl_wait();
  const auto sync = [&]() {
    if (C > 1)
      cluster_sync_all();
    else
      __syncthreads();
  };
  const unsigned in_layer = blockIdx.x >> p.log2_cluster;  // (user of the list, head)
  const int i = in_layer / heads, head = in_layer - i * heads;
  const int user = p.users[i];
  for (int layer = blockIdx.y; layer < p.pool.n_layers; layer += gridDim.y) {
    const bool known = user >= 0 && user < p.map.n_users;
    const int length = known ? min(max(0, p.map.lengths[user]), p.map.max_pages << p.pool.log2_tokens) : 0;
    int32_t *out = p.rows + (((int64_t)layer * p.n + i) * heads + head) * p.budget;
    if (layer == 0 && head == 0 && rank == 0 && tid == 0) {
      p.counts[i] = min(length, p.budget);
      if (!known) report(p.status, KFL_BAD_USER);
    }
    if (length <= p.budget) {  // (the whole cluster alike)
      for (int j = rank * THREADS + tid; j < p.budget; j += C * THREADS) out[j] = j < length ? j : -1;
      continue;
    }
    const int stop = length - p.recent, K = p.budget - p.first - p.recent;
    // ---- this thread's slots, of those from `first` (rounded down to four) to `stop`: `per` neighbours
    const float *mass = p.mass.row(layer, user, head);
    const int first4 = p.first & ~3;
    const int per = keys_per_thread(stop - first4, LOG2 + p.log2_cluster);
    const int s0 = min(first4 + (rank * THREADS + tid) * per, stop);  // (below 2^27)
    const bool stays = per <= p.room;
    const bool inner = __all_sync(0xffffffffu, s0 >= p.first && s0 + per <= stop);  // all of this warp's are in question
    const auto key_of = [&](int s, float v) { return s >= p.first && s < stop ? mass_key(v) : 0u; };
    if (stays && K > 0) {  // the masses as they are, a warp's together, its lanes side by side
      const int lane = tid & 31, sw = min(first4 + (rank * THREADS + tid - lane) * per, stop);
      float *to = reinterpret_cast<float *>(keys) + (tid - lane) * per;
      for (int o = 4 * lane; o < 32 * per; o += 128) {
        if (p.wide) {  // (a row's slots are a multiple of 16: what is read behind `stop` is there)
          if (sw + o < stop) cp_async16(to + o, mass + sw + o);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (sw + o + j < stop) to[o + j] = mass[sw + o + j];
        }
      }
      cp_async_commit();
    }
    // every key of this thread: f(slot, key); the first time they are made
    const auto each = [&](auto f, auto made) {
      if (stays) {
#pragma unroll 4
        for (int q = 0; q < per; q += 4) {
          uint4 *at = reinterpret_cast<uint4 *>(keys + tid * per + q);
          uint4 k = *at;
          if constexpr (!decltype(made)::value) {
            if (inner)
              k = {mass_key(__uint_as_float(k.x)), mass_key(__uint_as_float(k.y)), mass_key(__uint_as_float(k.z)),
                   mass_key(__uint_as_float(k.w))};
            else
              k = {key_of(s0 + q, __uint_as_float(k.x)), key_of(s0 + q + 1, __uint_as_float(k.y)),
                   key_of(s0 + q + 2, __uint_as_float(k.z)), key_of(s0 + q + 3, __uint_as_float(k.w))};
            *at = k;
          }
          f(s0 + q, k.x), f(s0 + q + 1, k.y), f(s0 + q + 2, k.z), f(s0 + q + 3, k.w);
        }
      } else {
#pragma unroll 4
        for (int q = 0; q < per; ++q) f(s0 + q, s0 + q < stop ? key_of(s0 + q, mass[s0 + q]) : 0u);
      }
    };
    const std::true_type made;
    for (int j = rank * THREADS + tid; j < p.first + p.recent; j += C * THREADS)
      out[j < p.first ? j : K + j] = j < p.first ? j : length - p.first - p.recent + j;
    if (K == 0) continue;
    uint32_t T = 0;
    int want = K;
    bool all = false;  // of the last bin
    cp_async_wait<0>();
    __syncthreads();  // (and the counts are zero)
    const auto narrow = [&](auto which) {
      constexpr int PASS = decltype(which)::value, SHIFT = PASS == 0 ? 21 : PASS == 1 ? 10 : 0;
      uint32_t *counts = hist[PASS & (TURNS - 1)];
      const uint32_t base = smem_addr(counts);
      // (keys of no slot, 0, fall into the first bin, which is never the one)
      each(
          [&](int, uint32_t k) {
            const uint32_t x = k ^ T;  // (T: the bits so far)
            if constexpr (PASS == 0)
              asm volatile("red.shared.add.u32 [%0], 1;" ::"r"(base + (x >> SHIFT) * 4) : "memory");
            else
              count_if(base + (x >> SHIFT) * 4, x < 1u << (SHIFT + (PASS == 1 ? 11 : 10)));
          },
          std::integral_constant<bool, (PASS > 0)>());
      sync();
      // a run of bins a thread, of all blocks; the one in which the `want`-th greatest lies
      uint4 b[BINS / 4];
#pragma unroll
      for (int j = 0; j < BINS / 4; ++j) b[j] = *reinterpret_cast<const uint4 *>(&counts[BINS * tid + 4 * j]);
      if constexpr (THREADS == 512) {  // (clusters: all blocks' counts under way together)
        if (C > 1) {
          uint4 o[7];
#pragma unroll
          for (int r = 1; r < 8; ++r)
            if (r < C) o[r - 1] = ld_cluster4(map_to_rank(base + BINS * tid * 4, (rank + r) & (C - 1)));
#pragma unroll
          for (int r = 1; r < 8; ++r)
            if (r < C) b[0].x += o[r - 1].x, b[0].y += o[r - 1].y, b[0].z += o[r - 1].z, b[0].w += o[r - 1].w;
        }
      }
      uint32_t own = 0, total;
#pragma unroll
      for (int j = 0; j < BINS / 4; ++j) own += b[j].x + b[j].y + (b[j].z + b[j].w);
      const uint32_t before = scan_block<WARPS>(own, total, sums[0]);
      int greater = (int)(total - before - own);
      if (greater < want && greater + (int)own >= want) {
#pragma unroll
        for (int j = BINS - 1; j >= 0; --j) {
          const int here = j % 4 == 3 ? b[j / 4].w : j % 4 == 2 ? b[j / 4].z : j % 4 == 1 ? b[j / 4].y : b[j / 4].x;
          if (greater < want && greater + here >= want) found[0] = BINS * tid + j, found[1] = want - greater, found[2] = here;
          greater += here;
        }
      }
      // zero again for the next pass: the other counts, free since every block has been here after it read them; or these, each
      // thread its own
      clear(hist[TURNS == 2 ? (PASS & 1) ^ 1 : 0]);
      __syncthreads();
      T |= (uint32_t)found[0] << SHIFT;
      want = found[1];
      all = want == found[2];
    };
    narrow(std::integral_constant<int, 0>());
    if (!all) narrow(std::integral_constant<int, 1>());
    if (!all) narrow(std::integral_constant<int, 2>());
    // (all of the last bin: its keys are those from T on, whatever their other bits)
    if (all) --T, want = 0;
    // ---- each thread's places: how many before it are above T, and at it
    uint32_t g = 0, t = 0, g0, t0 = 0, all_g, all_t = 0;
    each([&](int, uint32_t k) { g += k > T; }, made);
    if (want > 0) each([&](int, uint32_t k) { t += k == T; }, made);
    g0 = scan_block<WARPS>(g, all_g, sums[1]);
    if (want > 0) t0 = scan_block<WARPS>(t, all_t, sums[0]);
    if (C > 1) {
      if (tid == 0) totals[0] = all_g, totals[1] = all_t;
      cluster_sync_all();
      const int lane = tid & 31;
      const uint32_t a = lane < rank ? ld_cluster(map_to_rank(smem_addr(&totals[0]), lane)) : 0;
      const uint32_t b = lane < rank ? ld_cluster(map_to_rank(smem_addr(&totals[1]), lane)) : 0;
      g0 += __reduce_add_sync(0xffffffffu, a), t0 += __reduce_add_sync(0xffffffffu, b);
    }
    // ---- the slots: those above T, and of those at it the first `want`
    const uint32_t most = want;
    int32_t *to = out + p.first + g0 + min(t0, most);
    if (want == 0) {
      each(
          [&](int s, uint32_t k) {
            if (k > T) *to++ = s;
          },
          made);
    } else {
      uint32_t left = t0 < most ? most - t0 : 0;  // ties that are still wanted
      each(
          [&](int s, uint32_t k) {
            const bool tie = k == T && left > 0;
            if (k > T || tie) *to++ = s;
            left -= tie;
          },
          made);
    }
    // (the others have read this block's counts and totals)
    sync();
    if (TURNS == 2) clear(hist[0]), clear(hist[TURNS - 1]);
  }
}

template <int THREADS>
cudaError_t launch(SelectParams p, int most, cudaStream_t s) {
  static SmemOptIn opt_in;
  const cudaError_t e = opt_in(reinterpret_cast<const void *>(&kv4_select_kernel<THREADS>), SEL_BYTES);
  if (e != cudaSuccess) return e;
  p.room = std::min(keys_per_thread(most, (THREADS == 256 ? 8 : 9) + p.log2_cluster), SEL_BYTES / (4 * THREADS));
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.cluster, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.n * p.pool.n_kv_heads * p.cluster, std::min(p.pool.n_layers, 65535)), cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = (size_t)p.room * THREADS * 4, cfg.stream = s, cfg.attrs = attr, cfg.numAttrs = p.cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kv4_select_kernel<THREADS>, p);
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
  p.wide = ((reinterpret_cast<uintptr_t>(mass->data) | (uintptr_t)(4 * (mass->layer_stride | mass->user_stride | mass->head_stride))) & 15) == 0;
  // Rows for every SM: a block of 256 threads each, if 36 keys a thread hold them (a table is often a page longer than a round
  // number of rows).  Fewer, or longer ones: blocks of 512 threads, and clusters of them while a thread has more than 12 keys and
  // all are at work at once, or where one block's shared memory does not hold a row.  us in a graph, by rows x length:
  //                  256 threads   512   2 x 512   4 x 512   8 x 512
  //     4 x  4096       5.0        4.5     5.8       6.6       8.7
  //    64 x  4096       6.0        5.3     6.8      13.4      41.9
  //   256 x  4096       7.6        9.1    22.3      49.8
  //   896 x  4096      14.0       24.4    64.1
  //     8 x 16384                  9.9     9.7       9.7      11.6
  //   128 x 16384                 10.1    17.7      32.0      80.3
  //     8 x 65536                 (171)   16.4      12.1      11.9
  //   224 x 65536                 (406)   54.5      85.6     180.9
  const int most = map->max_pages * pool->page_tokens;
  const int64_t items = (int64_t)pool->n_layers * n * pool->n_kv_heads;
  p.cluster = 1;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (items >= 152 && keys_per_thread(most, 8) <= 36) return cuda_result(launch<256>(p, most, s), me);
  while (p.cluster < 8 &&
         keys_per_thread(most, 9 + p.log2_cluster) > (items * p.cluster * 2 <= 152 ? 12 : SEL_BYTES / (4 * 512)))
    p.cluster *= 2, ++p.log2_cluster;
  return cuda_result(launch<512>(p, most, s), me);
}
