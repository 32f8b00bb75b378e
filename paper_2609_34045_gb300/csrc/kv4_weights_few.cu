// The attention weight that few query rows of a KV head give its cached rows (include/kafila_kv4_evict.h).
//
// Mathematics.  With the log-sum-exp of every query row j known, a key's weights need no maximum and no other key:
//   mass_t += sum_j 2^(x_tj - log2(e) lse_j),  x_tj = scale log2(e) sum_g [ s_tg sum_c (u_tc - 8) q_jc + c_tg sum_c q_jc ]
// (g: groups of 64 channels).  The codes enter the products as they are, a nibble with zeros around it being an fp16
// u 2^-24 or u 2^-20, and the 8 too many come off through the accumulator's start value.  Every step is exact but the
// fp32 sums, the exponential (2^-22) and the weights' sum.
//
// What bounds it.  Half the cache's bytes (K): 0.28 bytes per cached element, 2 flops per query row: HBM, if the codes' instructions
// keep up.  32 users at 412 to 8192 keys, 64/8 heads of 128 (88 MB): 20.3 us in a graph, 4.3 TB/s; some 500 instructions a tile at half
// the issue slots, and about 6 us before the first tile and after the last.  (16 warps of 128 registers: 21.1; 14: 24.9; slots
// of three tiles: the same.)
//
// Layout.  S^T = K Q^T with m16n8k16, keys in M, 8 query rows in N (two or four such column blocks).  A key's weights lie in
// four lanes, which sum them; every cached row belongs to one warp, so nothing is merged and the order of the sums
// is always the same.
//
// Work split.  The tiles (64 keys of one sequence and KV head) of all sequences form one list, a unit more for each
// (sequence, head), whose query rows take about a tile's time; warps take equal pieces and stream them through
// slots of their own (bulk copies of the pages' K parts), with no barrier between warps.
#include <algorithm>
#include <type_traits>

#include "kv4_stream.cuh"
#include "kv4_weights.cuh"

namespace kfl {
namespace {

constexpr int LOG_TILE = 6, TILE = 1 << LOG_TILE;  // keys

template <int HD, int NT>
struct Weigh {
  static constexpr int WARPS = NT <= 2 ? 12 : 8;
  static constexpr int THREADS = WARPS * 32;
  static constexpr int UNROLL = NT == 1 ? 4 : 2;  // groups of 16 keys in a body
  static constexpr int GROUPS = HD / KV4_GROUP;
  static constexpr int CODES = TILE * HD / 2, PARAMS = TILE * HD / 16;
  static constexpr int TILE_BYTES = CODES + PARAMS;
  static constexpr int SLOTS = 4;
  static constexpr int RING_BYTES = WARPS * SLOTS * TILE_BYTES;
  static constexpr int SMEM = RING_BYTES + FEW_SEQS * 16 + (FEW_SEQS + 4) * 4 + WARPS * SLOTS * 8;
  static_assert(SMEM <= 232448, "shared memory of a block");
};

struct Cursor {
  int seq, head, tile, n_tiles, first_tile;
  int user, length, first, count;
};

// Tiles of a sequence for a KV head: none if it has no query rows here.
__device__ __forceinline__ int tiles_of(const int4 &v, const WeightParams &p, int &first_tile) {
  first_tile = p.window > 0 ? max(0, v.y - v.w + 1 - p.window) / TILE : 0;
  return v.w * p.group > p.row0 ? max(0, (v.y + TILE - 1) / TILE - first_tile) : 0;
}

__device__ __forceinline__ void enter_sequence(Cursor &c, const int4 *info, const WeightParams &p) {
  const int4 v = info[c.seq];
  c.user = v.x, c.length = v.y, c.first = v.z, c.count = v.w;
  c.n_tiles = tiles_of(v, p, c.first_tile);
}

// The tile of unit `flat` of the list, -1 for what comes before a segment's first (a segment of n tiles is n + 1 units).
__device__ __forceinline__ void locate_tile(Cursor &c, int64_t flat, const int4 *info, const int *prefix, const WeightParams &p) {
  int lo = 0, hi = p.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if ((int64_t)prefix[mid + 1] * p.pool.n_kv_heads > flat)
      hi = mid;
    else
      lo = mid + 1;
  }
  c.seq = lo;
  enter_sequence(c, info, p);
  const int rest = (int)(flat - (int64_t)prefix[lo] * p.pool.n_kv_heads);  // (below 256 heads * 2^20)
  c.head = rest / (c.n_tiles + 1);
  c.tile = rest - c.head * (c.n_tiles + 1) - 1;
}

__device__ __forceinline__ void next_tile(Cursor &c, const int4 *info, const WeightParams &p) {
  if (++c.tile < c.n_tiles) return;
  c.tile = 0;
  if (++c.head < p.pool.n_kv_heads) return;
  c.head = 0;
  do {
    if (++c.seq >= p.n_seqs) return;
    enter_sequence(c, info, p);
  } while (c.n_tiles <= 0);
}

template <int HD, int NT, bool BF16>
__global__ void __launch_bounds__(Weigh<HD, NT>::THREADS, 1) kv4_weights_few_kernel(const WeightParams p) {
  using F = Weigh<HD, NT>;
  constexpr int G = F::GROUPS, W = F::WARPS, UNROLL = F::UNROLL;
  extern __shared__ __align__(128) uint8_t smem[];
  int4 *info = reinterpret_cast<int4 *>(smem + F::RING_BYTES);
  int *prefix = reinterpret_cast<int *>(info + FEW_SEQS);
  uint64_t *bars = reinterpret_cast<uint64_t *>(prefix + FEW_SEQS + 4);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
  const int heads = p.pool.n_kv_heads, lp = p.pool.log2_tokens;
  pdl_launch_dependents();
  if (lane < F::SLOTS) mbar_init(smem_addr(bars + warp * F::SLOTS + lane), 1);  // (each warp its own)
  fence_mbar_init();
  pdl_wait();

  // ---- the list of tiles: each sequence's, summed.  Up to 32 sequences every warp makes the whole list, alike
  const auto units_of = [&](int s, bool again) {
    const int4 v = weight_sequence(p, s, again, blockIdx.x == 0 && p.row0 == 0);
    info[s] = v;
    int first_tile;
    const int n = tiles_of(v, p, first_tile);
    return n > 0 ? n + 1 : 0;
  };
  const auto warp_sum = [&](int v) {  // up to and with this lane's
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, v, off);
      if (lane >= off) v += o;
    }
    return v;
  };
  if (lane == 0) prefix[0] = 0;
  if (p.n_seqs <= 32 && p.seq0 == 0) {
    const unsigned same = __match_any_sync(0xffffffffu, p.users && lane < p.n_seqs ? p.users[lane] : -1 - lane);
    const int sum = warp_sum(lane < p.n_seqs ? units_of(lane, (same & ((1u << lane) - 1)) != 0) : 0);
    if (lane < p.n_seqs) prefix[lane + 1] = sum;
    __syncwarp();
  } else {
    for (int s = tid; s < p.n_seqs; s += F::THREADS) prefix[s + 1] = units_of(s, named_earlier(p, s));
    __syncthreads();
    if (warp == 0) {
      int before = 0;
      for (int s0 = 0; s0 < p.n_seqs; s0 += 32) {
        const int sum = warp_sum(s0 + lane < p.n_seqs ? prefix[s0 + lane + 1] : 0);
        if (s0 + lane < p.n_seqs) prefix[s0 + lane + 1] = before + sum;
        before += __shfl_sync(0xffffffffu, sum, 31);
      }
    }
    __syncthreads();
  }
  const int64_t total = (int64_t)prefix[p.n_seqs] * heads;
  const int64_t shares = (int64_t)gridDim.x * W, mine = (int64_t)blockIdx.x + (int64_t)warp * gridDim.x;
  // (neighbouring pieces to different SMs: a short list is spread over all of them)
  const int64_t quota = max((total + shares - 1) / shares, (int64_t)2);
  int64_t w0 = min(mine * quota, total);
  const int64_t w1 = min(w0 + quota, total);
  if (w0 >= w1) return;

  const uint32_t ring = smem_addr(smem) + warp * F::SLOTS * F::TILE_BYTES;
  const uint32_t bar0 = smem_addr(bars + warp * F::SLOTS);
  const int lb = min(lp, LOG_TILE);  // log2 of a page's tokens in a tile
  const int block_bytes = p.pool.block_bytes();
  const size_t page_bytes = p.pool.page_bytes();
  const uint8_t *layer_pages = p.pool.pages + (size_t)p.layer * heads * block_bytes;
  const uint64_t policy = policy_evict_normal();

  // ---- copies: codes and parameters of every page in a tile, a lane each
  Cursor fetch;
  locate_tile(fetch, w0, info, prefix, p);
  if (fetch.tile < 0) fetch.tile = 0, ++w0;
  if (w0 >= w1) return;  // (only the start of a segment whose tiles are another warp's)
  int64_t fetch_flat = w0;
  unsigned fetch_slot = 0;
  int fetch_page = -2;  // (behind the sequence's end)
  const bool copies = lane < (2 * TILE >> lb);
  const int part = lane & 1, block = lane >> 1;  // codes or parameters, of which page
  const int32_t *fetch_row = p.map.table + (int64_t)fetch.user * p.map.max_pages;
  const auto load_page = [&]() {
    const int key = (fetch.first_tile + fetch.tile) * TILE + (block << lb);
    fetch_page = copies && key < fetch.length ? fetch_row[key >> lp] : -2;
  };
  constexpr unsigned ALL = (1u << TILE / 16) - 1;
  unsigned valid[F::SLOTS] = {};  // which 16 keys of a slot's tile are there, a bit each
  bool dead = false;              // a wait gave up: no more copies, nothing is added
  const auto issue = [&]() {
    const uint32_t bar = bar0 + fetch_slot * 8, dst = ring + fetch_slot * F::TILE_BYTES;
    const bool there = fetch_page >= 0 && fetch_page < p.pool.n_pages;
    if (fetch_page != -2 && !there) report(p.status, KFL_BAD_PAGE);
    const unsigned lanes = __ballot_sync(0xffffffffu, there);
    unsigned have = 0;
#pragma unroll
    for (int i = 0; i < TILE / 16; ++i) have |= (lanes >> ((16 * i >> lb) * 2) & 1) << i;
    if (lane == 0) mbar_arrive_expect_tx(bar, __popc(have) * (F::TILE_BYTES / (TILE / 16)));
    __syncwarp();
    if (there) {
      const int size = part ? F::PARAMS : F::CODES, bytes = size >> (LOG_TILE - lb);
      const int more = lp - LOG_TILE, nth = more > 0 ? (fetch.first_tile + fetch.tile) & ((1 << more) - 1) : 0;
      const uint8_t *src = layer_pages + (unsigned)fetch_page * page_bytes + (unsigned)(fetch.head * block_bytes) +
                           (part ? 2 * p.pool.code_bytes() : 0) + nth * size;
      bulk_g2s(dst + (part ? F::CODES : 0) + block * bytes, src, bytes, bar, policy);
    }
#pragma unroll
    for (int i = 0; i < F::SLOTS; ++i)
      if (i == (int)fetch_slot) valid[i] = have;
    fetch_slot = fetch_slot + 1 == F::SLOTS ? 0 : fetch_slot + 1;
    const int seq = fetch.seq;
    fetch_flat += fetch.tile + 1 == fetch.n_tiles ? 2 : 1;
    if (fetch_flat < w1) {
      next_tile(fetch, info, p);
      if (fetch.seq != seq) fetch_row = p.map.table + (int64_t)fetch.user * p.map.max_pages;
      load_page();
    }
  };
  Cursor at = fetch;
  load_page();

  uint32_t q[NT][G][2][2][2];  // B fragments: [group][word of a lane][half of its pairs][register]
  float2 qs[NT][G], seed[NT][G], cf[NT], nl[NT];  // (columns 2 tig and 2 tig + 1)
  int end[NT][2];  // keys below it are seen
  bool without = false, absent = false;  // a row of this lane's saw nothing; a column is no row, or such a one
  unsigned slot = 0, phase = 0;
  float *mass = nullptr;
  const float log2_scale = fabsf(p.scale) * 1.44269504089f;
  const int key_lane = (gid >> 1) + 4 * (gid & 1);  // matrix row gid is this key of 16, row gid + 8 key_lane + 8
  for (int64_t flat = w0; flat < w1;) {
    if (flat == w0 || at.tile == 0) {
      // ---- a new (sequence, head): its query rows as fp16 (a power of two per row brings the largest to [2^14, 2^15): exact
      // but for the smallest of fp16)
      uint32_t raw[NT][G][8];
      const int rows = at.count * p.group - p.row0;  // (or more than there are columns)
      without = absent = false;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int row = p.row0 + min(n * 8 + gid, rows - 1), t = row / p.group;
        const bool there = n * 8 + gid < rows;
        const uint16_t *e =
            reinterpret_cast<const uint16_t *>(p.q.row((int64_t)at.first + t, at.head * p.group + row - t * p.group)) + tig * 16;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          if (!there) {
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[n][g][i] = 0;
          } else if (p.q_wide) {
            const uint4 a = *reinterpret_cast<const uint4 *>(e + 64 * g), b = *reinterpret_cast<const uint4 *>(e + 64 * g + 8);
            raw[n][g][0] = a.x, raw[n][g][1] = a.y, raw[n][g][2] = a.z, raw[n][g][3] = a.w;
            raw[n][g][4] = b.x, raw[n][g][5] = b.y, raw[n][g][6] = b.z, raw[n][g][7] = b.w;
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[n][g][i] = e[64 * g + 2 * i] | ((uint32_t)e[64 * g + 2 * i + 1] << 16);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int col = n * 8 + 2 * tig + c, row = p.row0 + min(col, rows - 1), t = row / p.group;
          const float lse = p.lse[((int64_t)at.first + t) * p.n_heads + at.head * p.group + row - t * p.group];
          // (a row that saw nothing adds nothing, and rows that are not there neither)
          const bool counts = col < rows && lse != -INFINITY;
          without = without || (col < rows && !counts);
          absent = absent || !counts;
          (c ? nl[n].y : nl[n].x) = counts ? lse * -1.44269504089f : -INFINITY;
          end[n][c] = counts ? at.length - at.count + t + 1 : -1;
        }
      if (flat == w0) issue();
      mass = p.mass.row(p.layer, at.user, at.head);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        // (magnitudes of either type order as their bits)
        uint32_t big2 = 0;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int i = 0; i < 8; ++i) big2 = __vmaxu2(big2, raw[n][g][i] & 0x7FFF7FFFu);
        uint32_t big1 = max(big2 & 0xffff, big2 >> 16);
        big1 = max(big1, __shfl_xor_sync(0xffffffffu, big1, 1));
        big1 = max(big1, __shfl_xor_sync(0xffffffffu, big1, 2));
        float inv;
        const float unit = xchunk_scale(BF16 ? bf16_to_f32((uint16_t)big1) : f16_to_f32((uint16_t)big1), &inv);
        inv = p.scale > 0.f ? inv : p.scale < 0.f ? -inv : 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float even[4] = {}, odd[4] = {};  // sums over the channels, as products with ones: in the accumulators' columns
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                // (odd channels' codes are 16 times the even ones': a sixteenth of the query)
                const uint32_t two = __byte_perm(raw[n][g][4 * j + h], raw[n][g][4 * j + h + 2], k ? 0x7632 : 0x5410);
                const float lo = BF16 ? bf16_lo(two) : half_lo(two), hi = BF16 ? bf16_hi(two) : half_hi(two);
                const float r = k ? inv * 0.0625f : inv;
                q[n][g][j][h][k] = pack_half2(lo * r, hi * r);
              }
              mma16816(even, 0x3C003C00u, 0x3C003C00u, 0, 0, q[n][g][j][h][0], q[n][g][j][h][1]);
              mma16816(odd, 0, 0, 0x3C003C00u, 0x3C003C00u, q[n][g][j][h][0], q[n][g][j][h][1]);
            }
          qs[n][g] = {LOW * fmaf(16.f, odd[0], even[0]), LOW * fmaf(16.f, odd[1], even[1])};
          seed[n][g] = {-8.f * qs[n][g].x, -8.f * qs[n][g].y};
        }
        const float factor = unit * log2_scale * (1.f / LOW);  // (columns of the accumulators: 2 tig, 2 tig + 1)
        cf[n] = {__shfl_sync(0xffffffffu, factor, 8 * tig), __shfl_sync(0xffffffffu, factor, 8 * tig + 4)};
        if (nl[n].x == -INFINITY) cf[n].x = 0.f;  // (no score makes up for it)
        if (nl[n].y == -INFINITY) cf[n].y = 0.f;
      }
      if (flat == w0)
#pragma unroll
        for (int i = 1; i < F::SLOTS; ++i)
          if (fetch_flat < w1) issue();
    }

    // ---- one tile.  A lane keeps the sums of two keys, of the 16 keys that bear its place's number
    const int tile0 = (at.first_tile + at.tile) * TILE;
    const int key_a = tile0 + 16 * tig + key_lane, key_b = key_a + 8;
    float old_a = 0.f, old_b = 0.f;
    if (key_a < at.length) old_a = mass[key_a];
    if (key_b < at.length) old_b = mass[key_b];
    if (!dead && !wait_2s(bar0 + slot * 8, phase)) {
      dead = true, fetch_flat = w1;
      if (lane == 0) report(p.status, KFL_TIMED_OUT);
      for (int i = 0; i < F::SLOTS; ++i) wait_2s(bar0 + i * 8, i < (int)slot ? phase ^ 1 : phase);
    }
    dead = __any_sync(0xffffffffu, dead);
    if (dead) return;  // (its own copies have landed or been waited for)
    unsigned have = 0;
#pragma unroll
    for (int i = 0; i < F::SLOTS; ++i)
      if (i == (int)slot) have = valid[i];
    const bool partly = __any_sync(0xffffffffu, without) || tile0 + TILE > at.length - at.count + 1 + p.row0 / p.group || have != ALL ||
                        (p.window > 0 && tile0 < at.length - p.window);
    float2 sum[TILE / 16] = {};  // of the lane's columns, for its two keys of every 16
    const auto weigh = [&](auto careful) {
      constexpr bool CAREFUL = decltype(careful)::value;
#pragma unroll(CAREFUL ? 1 : UNROLL)
      for (int st = 0; st < TILE / 16; ++st) {
        const uint32_t kb = ring + slot * F::TILE_BYTES + 16 * st * (HD / 2);
        const uint32_t kp = ring + slot * F::TILE_BYTES + F::CODES + 16 * st * (G * 4);
        uint2 kw[2][G];
        float ks[2][G], kc[2][G];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int g = 0; g < G; ++g) kw[h][g] = lds64(kb + (key_lane + 8 * h) * (HD / 2) + g * 32 + tig * 8);
          const uint32_t off = (key_lane + 8 * h) * (G * 4);
          uint32_t pk[G];
          if constexpr (G == 2) {
            const uint2 a = lds64(kp + off);
            pk[0] = a.x, pk[G - 1] = a.y;
          } else {
            pk[0] = lds32(kp + off);
          }
#pragma unroll
          for (int g = 0; g < G; ++g) ks[h][g] = half_lo(pk[g]), kc[h][g] = half_hi(pk[g]);
        }
        float2 x[NT][2];  // of a key, both columns
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float acc[NT][4];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t lo = j ? kw[0][g].y : kw[0][g].x, hi = j ? kw[1][g].y : kw[1][g].x;
            uint32_t a0, a1, a2, a3, a4, a5, a6, a7;
            code_pairs(lo, a0, a2), code_pairs(hi, a1, a3);
            code_pairs(lo >> 8, a4, a6), code_pairs(hi >> 8, a5, a7);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              if (j == 0) {
                const float from[4] = {seed[n][g].x, seed[n][g].y, seed[n][g].x, seed[n][g].y};
                mma16816(acc[n], a0, a1, a2, a3, q[n][g][j][0][0], q[n][g][j][0][1], from);
              } else {
                mma16816(acc[n], a0, a1, a2, a3, q[n][g][j][0][0], q[n][g][j][0][1]);
              }
              mma16816(acc[n], a4, a5, a6, a7, q[n][g][j][1][0], q[n][g][j][1][1]);
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              x[n][h] = fma2({ks[h][g], ks[h][g]}, {acc[n][2 * h], acc[n][2 * h + 1]},
                             fma2({kc[h][g], kc[h][g]}, qs[n][g], g == 0 ? float2{0.f, 0.f} : x[n][h]));
        }
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float2 w = fma2(x[n][h], cf[n], nl[n]);
            w = {ex2(w.x), ex2(w.y)};
            if (CAREFUL) {
              const int key = tile0 + 16 * st + key_lane + 8 * h;
              const auto sees = [&](int e) { return key < e && (p.window == 0 || key >= e - p.window) && (have >> st & 1); };
              w = {sees(end[n][0]) ? w.x : 0.f, sees(end[n][1]) ? w.y : 0.f};
            }
            s[h] += w.x + w.y;  // (in the same order: what is seen does not hang on what is not)
          }
#pragma unroll
        for (int i = 0; i < TILE / 16; ++i)  // (not by index: the sums stay in registers)
          if (i == st) sum[i] = {s[0], s[1]};
      }
    };
    bool again = partly;
    if (!partly) {
      weigh(std::false_type());
      // (a key that is no number has no weight for columns that are no rows)
      if (__any_sync(0xffffffffu, absent)) {
        float all = 0.f;
#pragma unroll
        for (int st = 0; st < TILE / 16; ++st) all += sum[st].x + sum[st].y;
        again = __any_sync(0xffffffffu, all != all);
      }
    }
    if (again) weigh(std::true_type());
    // sums over the four lanes of a key, in two exchanges: each lane ends with the 16 keys of its own number
    float2 half[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 mine = tig & 2 ? sum[2 + i] : sum[i], other = tig & 2 ? sum[i] : sum[2 + i];
      half[i] = {mine.x + __shfl_xor_sync(0xffffffffu, other.x, 2), mine.y + __shfl_xor_sync(0xffffffffu, other.y, 2)};
    }
    const float2 mine = tig & 1 ? half[1] : half[0], other = tig & 1 ? half[0] : half[1];
    const float sum_a = mine.x + __shfl_xor_sync(0xffffffffu, other.x, 1), sum_b = mine.y + __shfl_xor_sync(0xffffffffu, other.y, 1);
    __syncwarp();  // (every lane has read the slot)
    if (fetch_flat < w1) issue();
    if (++slot == F::SLOTS) slot = 0, phase ^= 1;
    if (have >> tig & 1) {
      if (key_a < at.length) mass[key_a] = old_a + sum_a;
      if (key_b < at.length) mass[key_b] = old_b + sum_b;
    }
    flat += at.tile + 1 == at.n_tiles ? 2 : 1;
    if (flat < w1) next_tile(at, info, p);
  }
}

template <int HD, int NT, bool BF16>
cudaError_t launch(const WeightParams &p, int n_sm, cudaStream_t s) {
  using F = Weigh<HD, NT>;
  static SmemOptIn opt_in;
  const void *kernel = reinterpret_cast<const void *>(&kv4_weights_few_kernel<HD, NT, BF16>);
  const cudaError_t e = opt_in(kernel, F::SMEM);
  if (e != cudaSuccess) return e;
  // as many blocks as the longest contexts could fill with two tiles a warp's share and one warp each
  const int64_t most = (int64_t)p.n_seqs * p.pool.n_kv_heads * (((int64_t)p.map.max_pages << p.pool.log2_tokens) / TILE + 2);
  const unsigned grid = (unsigned)std::min<int64_t>(n_sm, (most + 1) / 2);
  return launch_chained(kv4_weights_few_kernel<HD, NT, BF16>, grid, F::THREADS, F::SMEM, s, p);
}

template <int HD, bool BF16>
cudaError_t launch_cols(const WeightParams &p, int cols, int n_sm, cudaStream_t s) {
  return cols <= 8 ? launch<HD, 1, BF16>(p, n_sm, s) : cols <= 16 ? launch<HD, 2, BF16>(p, n_sm, s) : launch<HD, 4, BF16>(p, n_sm, s);
}

}  // namespace

cudaError_t launch_weights_few(const WeightParams &p, int cols, int n_sm, cudaStream_t s) {
  if (p.pool.head_dim == 128) return p.bf16 ? launch_cols<128, true>(p, cols, n_sm, s) : launch_cols<128, false>(p, cols, n_sm, s);
  return p.bf16 ? launch_cols<64, true>(p, cols, n_sm, s) : launch_cols<64, false>(p, cols, n_sm, s);
}

}  // namespace kfl
