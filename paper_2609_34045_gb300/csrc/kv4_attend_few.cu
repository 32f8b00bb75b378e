// Attention over the 4-bit paged KV cache for few query rows per KV head (decode steps, drafts), eight or sixteen at once.
//
// Mathematics.  For a KV head's query rows (token, head of its group) j and its keys t:
//   x_tj = scale log2(e) sum_g [ s_tg sum_c (u_tc - 8) q_jc + c_tg sum_c q_jc ]        (g: groups of 64 channels)
//   o_j = sum_t 2^(x_tj - m_j) [ s'_tg (u'_tc - 8) + c'_tg ] / sum_t 2^(x_tj - m_j)
// The codes enter the matrix products as they are, a nibble with zeros around it being an fp16 u 2^-24 or u 2^-20.  For
// the scores the 8 too many are taken off by the accumulator's start value -8 sum q; for the values the weights
// 2^(x - m) s' are the fp16 operand and 8 times their own sum (a product with ones) is taken off at the end.  (An
// offset as large as the 64 of a nibble set in the mantissa of a normal fp16 would be lost to the matrix unit's
// truncation: 3e-8 of the sum at every step, always downwards, made 131072 keys 4.4e-3 wrong.)  The scales so cost one
// factor per key and group, not per element, a group that reads as NaN reaches exactly the rows that see it, and
// codes behind a user's end (any bits) are finite.
//
// What bounds it.  0.56 bytes per cached element and 4 flops per query row: HBM, if the elements' arithmetic
// keeps up.  At 6.77 TB/s an SM gets 42 elements a clock, its logic units do 64 operations: 0.6 (K) and 0.75 (V) per
// element for the nibbles and some 0.4 for the rest.  Measured: 32 users at 412 to 8192 keys, 64/8 heads of 128 (160 MB)
// 41 us; one user at 131072 keys (151 MB) 40 us, 3.8 TB/s: 25 us of tiles, which 12 warps of 168 registers work off at
// about 0.88 of the copy rate, 4 us before them (list, queries) and 10 after (partial results, merges), most of it code
// that runs once.
//
// Layout.  S^T = K Q^T and O^T = V^T P^T with m16n8k16: keys and channels fill M = 16, the query rows N = 8, nothing
// is padded at 8 rows.  The matrix unit's k order is ours to choose, so a lane's K words hold whole fragments
// in natural byte order, and V's pairs of tokens come together by one byte permute per eight codes.
//
// Work split.  The tiles (64 keys of one sequence, KV head and sixteen query rows) of all sequences form one list, with a
// place more for each segment (sequence, head, rows), whose start and end cost a warp as much as a tile; one
// block per SM takes an equal piece, its warps equal pieces of that.  A warp streams its tiles through two slots of its own
// (bulk copies of whole page blocks), with no barrier between warps until the end.  What a warp holds of a
// segment that it does not own alone is merged within the block, then over blocks by the last to arrive, which brings their
// parts to shared memory together; every sum is taken in list order, so results do not depend on arrival.
#include <algorithm>
#include <type_traits>

#include "attn_core.cuh"  // cp_async16
#include "kv4_attend.cuh"

namespace kfl {
namespace {

constexpr int LOG_TILE = 6, TILE = 1 << LOG_TILE;  // keys
constexpr float WEIGHT_UNIT = 2048.f;  // fp16 weights: 2^(x - m) times this, at most WEIGHT_MOST times as much
constexpr float WEIGHT_MOST = 16.f;
// Groups of 16 keys that are worked on at once: 1, 2 and 4 took 54, 51 and 58 us for 32 ragged users, of which 10 have gone
// since at the start and the end (more steps; more code than the instruction cache next to the scheduler holds)
constexpr int SUB = 2;

template <int HD, int NT>
struct Few {
  // 12 warps of at most 168 registers (11: 2 us more for 32 ragged users; 16 spill in the tile loop); with 16 query rows 8 warps of
  // 255.  At head_dim 128 both keep 16 bytes of a thread in local memory
  static constexpr int WARPS = NT == 1 ? 12 : 8;
  static constexpr int THREADS = WARPS * 32;
  static constexpr int COLS = 8 * NT;
  static constexpr int GROUPS = HD / KV4_GROUP;
  static constexpr int TILE_BYTES = TILE * HD * 9 / 8;
  static constexpr int SLOTS = HD == 128 ? 2 : 3;
  static constexpr int COL = HD + 4;                    // floats from column to column of a partial result: other banks
  static constexpr int PARTIAL = COLS * COL + 2 * COLS;  // floats: [col][channel], then [col] (max, sum)
  static constexpr int RING_BYTES = WARPS * SLOTS * TILE_BYTES;
  static constexpr int SMEM = RING_BYTES + FEW_SEQS * 16 + (FEW_SEQS + 4) * 4 + WARPS * SLOTS * 8 + (8 * WARPS + 8) * 4;
  static_assert(PARTIAL % 4 == 0, "copied in 16 bytes");
  static_assert(PARTIAL * 4 <= TILE_BYTES, "a slot holds a warp's partial result");
  static_assert(SMEM <= 232448, "shared memory of a block");
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same from a start value of its own.
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1, const float (&c)[4]) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float half_lo(uint32_t x) { return __low2float(*reinterpret_cast<const __half2 *>(&x)); }
__device__ __forceinline__ float half_hi(uint32_t x) { return __high2float(*reinterpret_cast<const __half2 *>(&x)); }

// The nibbles of a word's bytes 0 and 2 as two fp16 pairs, as they stand: whole numbers below 2048 in the bits of an fp16
// are that many times 2^-24 (its subnormal numbers and the first binade above), exactly, and the matrix unit takes them as
// any others.  The low nibbles are u 2^-24, the high ones u 2^-20.
__device__ __forceinline__ void code_pairs(uint32_t w, uint32_t &low, uint32_t &high) {
  low = w & 0x000F000Fu;
  high = w & 0x00F000F0u;
}
constexpr float LOW = 0x1p-24f, HIGH = 0x1p-20f;
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}

// 1 / x, and 0 of 0: a sum of weights, which is 0 where nothing is seen, else no smaller than its reference's weight
__device__ __forceinline__ float inverse(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return x == 0.f ? 0.f : r;
}
// Two outputs.
template <bool BF16>
__device__ __forceinline__ uint32_t pack_out(float lo, float hi) {
  uint32_t r;
  if (!BF16) return pack_half2(lo, hi);
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// a / b, in 32 bits where they fit: one chain of instructions instead of three.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (a | b) >> 32 ? a / b : (int64_t)((unsigned)a / (unsigned)b);
}

// A place in the list of tiles.
struct Cursor {
  int seq, head, block, tile;  // block: of COLS query rows; tile: within the segment (sequence, KV head, block)
  int blocks, n_tiles, first_tile;
  int user, length, first, count;
};

// (user, length, first token, tokens) of a sequence; its tiles start at key first_tile * 64
__device__ __forceinline__ int first_tile_of(int length, int count, int window) {
  return window > 0 ? max(0, length - count + 1 - window) / TILE : 0;
}

template <int COLS>
__device__ __forceinline__ void enter_sequence(Cursor &c, const int4 *info, const int *prefix, const AttendParams &p) {
  const int4 v = info[c.seq];
  c.user = v.x, c.length = v.y, c.first = v.z, c.count = v.w;
  c.blocks = (c.count * p.group + COLS - 1) / COLS;
  int units = prefix[c.seq + 1] - prefix[c.seq];
  if (c.blocks > 1) units /= c.blocks;
  c.n_tiles = units - 1;
  c.first_tile = first_tile_of(v.y, v.w, p.window);
}

// The tile of unit `flat` of the list, -1 for what comes before a segment's first (a segment of n tiles is n + 1 units).
template <int COLS>
__device__ __forceinline__ void locate_tile(Cursor &c, int64_t flat, const int4 *info, const int *prefix,
                                            const AttendParams &p) {
  int lo = 0, hi = p.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if ((int64_t)prefix[mid + 1] * p.pool.n_kv_heads > flat)
      hi = mid;
    else
      lo = mid + 1;
  }
  c.seq = lo;
  enter_sequence<COLS>(c, info, prefix, p);
  const int rest = (int)(flat - (int64_t)prefix[lo] * p.pool.n_kv_heads);  // (below heads * blocks * 2^20)
  const int segment = rest / (c.n_tiles + 1);
  c.tile = rest - segment * (c.n_tiles + 1) - 1;
  c.head = segment / c.blocks;
  c.block = segment - c.head * c.blocks;
}

template <int COLS>
__device__ __forceinline__ void next_tile(Cursor &c, const int4 *info, const int *prefix, const AttendParams &p) {
  if (++c.tile < c.n_tiles) return;
  c.tile = 0;
  if (++c.block < c.blocks) return;
  c.block = 0;
  if (++c.head < p.pool.n_kv_heads) return;
  c.head = 0;
  do {
    if (++c.seq >= p.n_seqs) return;
    enter_sequence<COLS>(c, info, prefix, p);
  } while (c.n_tiles <= 0);
}

// The token of a query row: row / group, for rows below 64 (group at most 128: the product's error stays below its place)
__device__ __forceinline__ int token_of(int row, const AttendParams &p) { return (unsigned)row * p.group_inv >> 16; }
// Query row `col` of the segment's block: the token's and the head's place.
template <int COLS>
__device__ __forceinline__ void row_of(const Cursor &c, int col, const AttendParams &p, int64_t &token, int &head) {
  const int row = c.block * COLS + col, t = token_of(row, p);
  token = c.first + t;
  head = c.head * p.group + row - t * p.group;
}

// One output row's channels from lane `lane`'s HD / 32 values.
template <int HD, int COLS, bool BF16>
__device__ __forceinline__ void store_row(const AttendParams &p, const Cursor &c, int col, int lane, const float (&v)[HD / 32],
                                          float top, float sum) {
  int64_t t;
  int head;
  row_of<COLS>(c, col, p, t, head);
  const float inv = inverse(sum);
  uint16_t *out = reinterpret_cast<uint16_t *>(p.out.row(t, head)) + lane * (HD / 32);
  uint32_t h[HD / 64];
#pragma unroll
  for (int i = 0; i < HD / 64; ++i) h[i] = pack_out<BF16>(v[2 * i] * inv, v[2 * i + 1] * inv);
  if (p.out_wide) {
    if constexpr (HD == 128)
      *reinterpret_cast<uint2 *>(out) = make_uint2(h[0], h[HD / 64 - 1]);
    else
      *reinterpret_cast<uint32_t *>(out) = h[0];
  } else {
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) out[i] = (uint16_t)(h[i / 2] >> 16 * (i & 1));
  }
  if (p.lse && lane == 0) p.lse[t * p.n_heads + head] = sum == 0.f ? -INFINITY : 0.69314718056f * top + logf(sum);
}

// NC columns from `col` on of several partial results, `n` of them at at(i), in order: merged by one warp.  Lanes take the
// parts' places, maxima and sums, 32 at a time; every lane takes its channels of all parts, four at a time, the first of them
// under way with the maxima.  (Eight at a time take the tiles' registers: 32 ragged users 45 us for 41.)
template <int HD, int COLS, int NC, class At>
__device__ __forceinline__ void merge_columns(int n, int col, int lane, const At &at, float (&v)[NC][HD / 32], float (&top)[NC],
                                              float (&sum)[NC]) {
  constexpr int C = HD / 32, COL = Few<HD, COLS / 8>::COL, AHEAD = 4;
  static_assert(32 % AHEAD == 0, "a round stays within the 32 parts whose weights the lanes hold");
  using Vec = typename std::conditional<C == 4, float4, float2>::type;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    top[c] = -INFINITY, sum[c] = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j) v[c][j] = 0.f;
  }
  Vec x[AHEAD][NC];
  const float *mine = at(min(lane, n - 1));
  const auto load = [&](int i) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (i + k >= n) break;
      const float *part = reinterpret_cast<const float *>(
                              __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), (i + k) & 31)) +
                          col * COL + lane * C;
#pragma unroll
      for (int c = 0; c < NC; ++c) x[k][c] = *reinterpret_cast<const Vec *>(part + c * COL);
    }
  };
  load(0);
  float m[NC], l[NC];  // of part `lane`
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m[c] = -INFINITY, l[c] = 0.f;
    if (lane < n) m[c] = mine[COLS * COL + col + c], l[c] = mine[COLS * COL + COLS + col + c];
    top[c] = m[c];
  }
  for (int i = lane + 32; i < n; i += 32)
#pragma unroll
    for (int c = 0; c < NC; ++c) top[c] = fmaxf(top[c], at(i)[COLS * COL + col + c]);
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], off));
#pragma unroll 1
  for (int i = 0; i < n; i += AHEAD) {
    if ((i & 31) == 0) {  // the next 32 parts' weights
      if (i > 0) {
        mine = at(min(i + lane, n - 1));
#pragma unroll
        for (int c = 0; c < NC; ++c) m[c] = mine[COLS * COL + col + c], l[c] = mine[COLS * COL + COLS + col + c];
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        m[c] = i + lane < n ? ex2(m[c] - (top[c] == -INFINITY ? 0.f : top[c])) : 0.f;
        if (i + lane < n) sum[c] = fmaf(l[c], m[c], sum[c]);
      }
    }
    if (i > 0) load(i);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (i + k >= n) break;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const float wi = __shfl_sync(0xffffffffu, m[c], (i + k) & 31);
        const float *y = reinterpret_cast<const float *>(&x[k][c]);
#pragma unroll
        for (int j = 0; j < C; ++j) v[c][j] = fmaf(y[j], wi, v[c][j]);
      }
    }
  }
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], off);
}

template <int HD, int NT, bool BF16>
__global__ void __launch_bounds__(Few<HD, NT>::THREADS, 1) kv4_attend_few_kernel(const AttendParams p) {
  using F = Few<HD, NT>;
  constexpr int G = F::GROUPS, COLS = F::COLS, W = F::WARPS;
  extern __shared__ __align__(128) uint8_t smem[];
  int4 *info = reinterpret_cast<int4 *>(smem + F::RING_BYTES);
  int *prefix = reinterpret_cast<int *>(info + FEW_SEQS);
  uint64_t *bars = reinterpret_cast<uint64_t *>(prefix + FEW_SEQS + 4);
  int *part_seg = reinterpret_cast<int *>(bars + W * F::SLOTS);  // [2 W]: segment of each partial result (packed), or -1
  int *part_place = part_seg + 2 * W, *group_seg = part_place + 2 * W;
  int *group_at = group_seg + 2 * W, *n_groups = group_at + 2 * W + 1;
  volatile int *cut = n_groups + 1, *span = cut + 2;  // of the segments that this block merges: blocks
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
  const int heads = p.pool.n_kv_heads, lp = p.pool.log2_tokens;
  pdl_launch_dependents();
  if (lane < F::SLOTS) mbar_init(smem_addr(bars + warp * F::SLOTS + lane), 1);  // (each warp its own)
  if (lane < 2) part_seg[2 * warp + lane] = -1;
  fence_mbar_init();
  pdl_wait();

  // ---- the list of tiles: each sequence's, summed (a sequence without rows has one, to write its zeros).  Each segment has
  // one unit more, since its rows and results take about as long as a tile (uncounted, 32 ragged users: 42.8 us for 40.9, drafts
  // 20.9 for 18.3).  Up to 32
  // sequences every warp makes the whole list, alike, and waits for no other
  const auto tiles_of = [&](int s) {
    const int user = p.users ? p.users[s] : p.seq0 + s;
    const int first = p.q_start ? p.q_start[s] : p.seq0 + s;
    int count = p.q_start ? p.q_start[s + 1] - first : 1, length = 0, bad = 0;
    if (first < 0 || count < 0 || count > p.max_q || first > p.n_tokens - count) bad |= KFL_BAD_POSITION, count = 0;
    if (user < 0 || user >= p.map.n_users)
      bad |= KFL_BAD_USER;
    else
      length = min(max(0, p.map.lengths[user]), p.map.max_pages << lp);
    if (bad && blockIdx.x == 0) report(p.status, bad);
    info[s] = make_int4(user, length, first, count);
    return (count * p.group + COLS - 1) / COLS *
           (max(1, (length + TILE - 1) / TILE - first_tile_of(length, count, p.window)) + 1);
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
  int longest = 0;  // units of a sequence, all its blocks of rows
  if (p.n_seqs <= 32) {
    const int units = lane < p.n_seqs ? tiles_of(lane) : 0, sum = warp_sum(units);
    if (lane < p.n_seqs) prefix[lane + 1] = sum;
    longest = __reduce_max_sync(0xffffffffu, units);
    __syncwarp();
  } else {
    for (int s = tid; s < p.n_seqs; s += F::THREADS) prefix[s + 1] = tiles_of(s);
    __syncthreads();
    if (warp == 0) {
      int before = 0;
      for (int s0 = 0; s0 < p.n_seqs; s0 += 32) {
        const int units = s0 + lane < p.n_seqs ? prefix[s0 + lane + 1] : 0, sum = warp_sum(units);
        longest = max(longest, units);
        if (s0 + lane < p.n_seqs) prefix[s0 + lane + 1] = before + sum;
        before += __shfl_sync(0xffffffffu, sum, 31);
      }
      longest = __reduce_max_sync(0xffffffffu, longest);
      if (lane == 0) prefix[FEW_SEQS + 1] = longest;
    }
    __syncthreads();
    longest = prefix[FEW_SEQS + 1];
  }
  const int64_t total = (int64_t)prefix[p.n_seqs] * heads;
  // at least a tile for every warp of a block: fewer blocks, fewer merges
  int64_t quota = max(quotient(total + gridDim.x - 1, gridDim.x), (int64_t)W);
  // A segment over more blocks than the ring holds parts of is merged from global memory, at some 330 clocks a part: it gets
  // larger pieces where those cost less, 460 clocks a tile (one KV head of 131072 keys: 27.0 us for 40.9)
  constexpr int MOST_PARTS = F::RING_BYTES / (F::PARTIAL * 4) - 4;
  if (longest > MOST_PARTS * p.most_blocks * quota) {
    const int segment = longest / p.most_blocks;
    const int64_t larger = segment / MOST_PARTS + 1;
    if (7 * (larger - quota) < 5 * (quotient(segment, quota) - 18)) quota = larger;
  }
  const int64_t c0 = min(blockIdx.x * quota, total), c1 = min(c0 + quota, total);
  if (c0 >= c1) return;
  const auto share = [&](int w) { return c0 + (c1 - c0 <= 1 << 27 ? (unsigned)(c1 - c0) * w / W : (c1 - c0) * w / W); };
  int64_t w0 = share(warp);
  const int64_t w1 = share(warp + 1);

  const uint32_t ring = smem_addr(smem) + warp * F::SLOTS * F::TILE_BYTES;
  const uint32_t bar0 = smem_addr(bars + warp * F::SLOTS);
  constexpr int CODES = TILE * HD / 2, PARAMS = TILE * HD / 16;  // of a tile's K or V, as in a block of 64 tokens
  const int lb = min(lp, LOG_TILE);                         // log2 of a page's tokens in a tile
  const int block_bytes = p.pool.block_bytes();
  const size_t page_bytes = p.pool.page_bytes();
  const uint8_t *layer_pages = p.pool.pages + (size_t)p.layer * heads * block_bytes;
  const uint64_t policy = policy_evict_normal();

  // ---- copies: a page of a tile's size is one as it stands; of others a page's part of the tile comes in four (codes and
  // parameters of K and V), a lane each
  Cursor fetch;
  int fetch_page = -2;  // (behind the sequence's end)
  unsigned fetch_slot = 0;
  const int lane_key = lane >> 2 << lb;              // of this lane's copy, in the tile
  const bool copies = lane < (lp == LOG_TILE ? 1 : 4 * TILE >> lb);
  const int32_t *fetch_row = nullptr;
  if (w0 < w1) {
    locate_tile<COLS>(fetch, w0, info, prefix, p);
    if (fetch.tile < 0) fetch.tile = 0, ++w0;
    fetch_row = p.map.table + (int64_t)fetch.user * p.map.max_pages;
  }
  int64_t fetch_flat = w0;  // (w1: all are brought or under way)
  const auto load_page = [&]() {  // the page of this lane's copy for the tile at `fetch`
    const int key = (fetch.first_tile + fetch.tile) * TILE + lane_key;
    fetch_page = copies && key < fetch.length ? fetch_row[key >> lp] : -2;
  };
  constexpr unsigned ALL = (1u << TILE / 16) - 1;
  unsigned valid[F::SLOTS] = {};  // which 16 keys of a slot's tile are there, a bit each
  bool dead = false;              // a wait gave up: no more copies, no results
  const auto issue = [&]() {
    const uint32_t bar = bar0 + fetch_slot * 8, dst = ring + fetch_slot * F::TILE_BYTES;
    unsigned have = 0;
    if (lp == LOG_TILE) {
      // (an elected lane of a page number that all have: one instruction and not a loop over the lanes)
      const int page = __shfl_sync(0xffffffffu, fetch_page, 0);
      const bool there = page >= 0 && page < p.pool.n_pages;
      if (there) have = ALL;
      if (elect_one()) {
        if (page != -2 && !there) report(p.status, KFL_BAD_PAGE);
        mbar_arrive_expect_tx(bar, there ? F::TILE_BYTES : 0);
        const uint8_t *src = layer_pages + (unsigned)page * page_bytes + (unsigned)(fetch.head * block_bytes);
        if (there) bulk_g2s(dst, src, F::TILE_BYTES, bar, policy);
      }
      __syncwarp();
    } else {
      const bool there = fetch_page >= 0 && fetch_page < p.pool.n_pages;
      if (fetch_page != -2 && !there) report(p.status, KFL_BAD_PAGE);
      const unsigned lanes = __ballot_sync(0xffffffffu, there);
#pragma unroll
      for (int i = 0; i < TILE / 16; ++i) have |= (lanes >> ((16 * i >> lb) * 4) & 1) << i;
      if (lane == 0) mbar_arrive_expect_tx(bar, __popc(have) * (F::TILE_BYTES / (TILE / 16)));
      __syncwarp();
      if (there) {
        // part 0, 1: codes of K, V; 2, 3: parameters.  A larger page holds several tiles
        const uint8_t *src = layer_pages + (unsigned)fetch_page * page_bytes + (unsigned)(fetch.head * block_bytes);
        const int part = lane & 3, block = lane >> 2, size = part < 2 ? CODES : PARAMS, bytes = size >> (LOG_TILE - lb);
        const int to = (part < 2 ? 0 : 2 * CODES) + (part & 1) * size;  // as in a page of a tile's size
        const int more = lp - LOG_TILE, nth = more > 0 ? (fetch.first_tile + fetch.tile) & ((1 << more) - 1) : 0;
        bulk_g2s(dst + to + block * bytes, src + (more > 0 ? (to << more) + nth * size : to >> -more), bytes, bar, policy);
      }
    }
#pragma unroll
    for (int i = 0; i < F::SLOTS; ++i)
      if (i == (int)fetch_slot) valid[i] = have;
    fetch_slot = fetch_slot + 1 == F::SLOTS ? 0 : fetch_slot + 1;
    const int seq = fetch.seq;
    fetch_flat += fetch.tile + 1 == fetch.n_tiles ? 2 : 1;
    if (fetch_flat < w1) {
      next_tile<COLS>(fetch, info, prefix, p);
      if (fetch.seq != seq) fetch_row = p.map.table + (int64_t)fetch.user * p.map.max_pages;
      load_page();
    }
  };
  Cursor at = fetch;
  if (fetch_flat < w1) load_page();

  // ---- this warp's tiles
  uint32_t q[NT][G][2][2][2];     // B fragments: [group][word of a lane][half of its pairs][register]
  float seed[NT][G][4], qs[NT][G][2], cf[NT][2];
  float o[NT][G][4][4], ones[NT][G][4], top[NT][2], sum[NT][2], centre[NT][G][2];
  float v_unit = 0.f;             // the value scales' reference, a power of two
  unsigned slot = 0, phase = 0;
  int rows = 0;
  float *block_ws = p.partials + (size_t)blockIdx.x * (W + 2) * F::PARTIAL;
  const float log2_scale = fabsf(p.scale) * 1.44269504089f;
  for (int64_t flat = w0; flat < w1;) {
    if (flat == w0 || at.tile == 0) {
      // ---- a new (sequence, head): its query rows as fp16 (a power of two per row brings the largest to [2^14, 2^15))
      // 16 channels of each group for column gid; under way before the first tiles' copies, whose page numbers come first
      uint32_t raw[NT][G][8];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int col = n * 8 + gid;
        const bool there = col < at.count * p.group - at.block * COLS;
        int64_t token;
        int head;
        row_of<COLS>(at, col, p, token, head);
        const uint16_t *e = reinterpret_cast<const uint16_t *>(there ? p.q.row(token, head) : nullptr) +
                            tig * 16;
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
      if (flat == w0) issue();
      rows = at.count * p.group - at.block * COLS;
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
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            qs[n][g][c] = LOW * fmaf(16.f, odd[c], even[c]);
            seed[n][g][c] = seed[n][g][c + 2] = -8.f * qs[n][g][c];
            centre[n][g][c] = 0.f;
          }
        }
        // (columns of the accumulators: 2 tig, 2 tig + 1)
        // (not 0: -inf times it stays)
        const float factor = p.scale == 0.f ? 1.f : fmaxf(unit * log2_scale * (1.f / LOW), 1e-37f);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          cf[n][c] = __shfl_sync(0xffffffffu, factor, (2 * tig + c) * 4);
          top[n][c] = -INFINITY, sum[n][c] = 0.f;
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            ones[n][g][i] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[n][g][i][j] = 0.f;
          }
        }
      }
      v_unit = 0.f;
      if (flat == w0)
#pragma unroll
        for (int i = 1; i < F::SLOTS; ++i)
          if (fetch_flat < w1) issue();
    }

    // ---- one tile
    if (!dead && !wait_2s(bar0 + slot * 8, phase)) {
      dead = true, fetch_flat = w1;
      if (lane == 0) report(p.status, KFL_TIMED_OUT);
      for (int i = 0; i < F::SLOTS; ++i) wait_2s(bar0 + i * 8, i < (int)slot ? phase ^ 1 : phase);
    }
    dead = __any_sync(0xffffffffu, dead);
    unsigned have = 0;
#pragma unroll
    for (int i = 0; i < F::SLOTS; ++i)
      if (i == (int)slot) have = valid[i];
    // in steps of 16 SUB keys: the tile at once is more code than the instruction cache next to the scheduler holds
#pragma unroll 1
    for (int s0 = 0; s0 < TILE / 16 && !dead; s0 += SUB, have >>= SUB) {
      const uint32_t base = ring + slot * F::TILE_BYTES + 16 * s0 * (HD / 2);
      const uint32_t base_p = ring + slot * F::TILE_BYTES + 2 * CODES + 16 * s0 * (G * 4);
      const int key0 = (at.first_tile + at.tile) * TILE + 16 * s0;
      // some rows do not see all of the tile: its last keys, a window's first ones, a missing page
      const int all_end = at.length - at.count + 1;
      const bool masked = key0 + 16 * SUB > all_end || (have & ((1 << SUB) - 1)) != (1 << SUB) - 1 ||
                          (p.window > 0 && key0 < at.length - p.window);
      float x[NT][SUB][4];
      uint32_t vpar[SUB][2][G];  // (scale, centre) of the lane's two keys of each subtile, as they are stored
      const int key_lane = (gid >> 1) + 4 * (gid & 1);  // matrix row gid is this key of a subtile, row gid + 8 key_lane + 8
#pragma unroll
      for (int st = 0; st < SUB; ++st) {
        const uint32_t kb = base + 16 * st * (HD / 2);
        const uint32_t kp = base_p + 16 * st * (G * 4), vp = kp + PARAMS;
        uint2 kw[2][G];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int g = 0; g < G; ++g) kw[h][g] = lds64(kb + (key_lane + 8 * h) * (HD / 2) + g * 32 + tig * 8);
        float ks[2][G], kc[2][G];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t off = (key_lane + 8 * h) * (G * 4);
          uint32_t pk[G], pv[G];
          if constexpr (G == 2) {
            const uint2 a = lds64(kp + off), c = lds64(vp + off);
            pk[0] = a.x, pk[G - 1] = a.y, pv[0] = c.x, pv[G - 1] = c.y;
          } else {
            pk[0] = lds32(kp + off), pv[0] = lds32(vp + off);
          }
#pragma unroll
          for (int g = 0; g < G; ++g) {
            ks[h][g] = half_lo(pk[g]), kc[h][g] = half_hi(pk[g]);
            vpar[st][h][g] = pv[g];
          }
        }
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
              if (j == 0)
                mma16816(acc[n], a0, a1, a2, a3, q[n][g][j][0][0], q[n][g][j][0][1], seed[n][g]);
              else
                mma16816(acc[n], a0, a1, a2, a3, q[n][g][j][0][0], q[n][g][j][0][1]);
              mma16816(acc[n], a4, a5, a6, a7, q[n][g][j][1][0], q[n][g][j][1][1]);
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float t = kc[i >> 1][g] * qs[n][g][i & 1];
              x[n][st][i] = g == 0 ? fmaf(ks[i >> 1][g], acc[n][i], t)
                                  : fmaf(ks[i >> 1][g], acc[n][i], fmaf(kc[i >> 1][g], qs[n][g][i & 1], x[n][st][i]));
            }
        }
      }
      if (masked) {
        unsigned hidden[NT] = {};  // a bit per score of this lane
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int k = 16 * st + key_lane + 8 * (i >> 1);
              const int end = all_end + min(token_of(at.block * COLS + n * 8 + 2 * tig + (i & 1), p), at.count - 1);
              const bool sees = key0 + k < end && (p.window == 0 || key0 + k >= end - p.window) && (have >> st & 1);
              if (!sees) x[n][st][i] = -INFINITY, hidden[n] |= 1u << (4 * st + i);
            }
        // Parameters that no row sees may be anything.  A NaN that some rows see and others do not: theirs at once
        // (through the group's centres), and gone for the products, where it would meet the others' zeros
#pragma unroll
        for (int st = 0; st < SUB; ++st)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int g = 0; g < G; ++g) {
              const int k = 16 * st + key_lane + 8 * h;
              if (key0 + k >= at.length || !(have >> st & 1)) vpar[st][h][g] = 0;
              const uint32_t v = vpar[st][h][g];
              if ((v & 0x7c00u) == 0x7c00u || (v & 0x7c000000u) == 0x7c000000u) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                  for (int c = 0; c < 2; ++c)
                    if (!(hidden[n] >> (4 * st + 2 * h + c) & 1)) centre[n][g][c] = __uint_as_float(0x7fc00000u);
                vpar[st][h][g] = 0;
              }
            }
      }
      // ---- weights against the reference that the columns have: it holds unless it is not there yet, a weight has outgrown
      // it, or the value scales have outgrown their common unit (the products of the two are fp16, below 2^15)
      __half2 v_most = __float2half2_rn(0.f);  // (hmax2 passes over NaN)
#pragma unroll
      for (int st = 0; st < SUB; ++st)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int g = 0; g < G; ++g) v_most = __hmax2(v_most, *reinterpret_cast<const __half2 *>(&vpar[st][h][g]));
      float v_max = __low2float(v_most);
      bool grows = v_max > v_unit;
      float pr[NT][SUB][4], part[NT][2];
      const auto weigh = [&]() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const float2 scale = {cf[n][0], cf[n][1]};
          const float2 from = {top[n][0] == -INFINITY ? 0.f : -top[n][0] * cf[n][0],
                               top[n][1] == -INFINITY ? 0.f : -top[n][1] * cf[n][1]};
          part[n][0] = part[n][1] = 0.f;
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
              const float2 e = fma2({x[n][st][i], x[n][st][i + 1]}, scale, from);
              pr[n][st][i] = ex2(e.x), pr[n][st][i + 1] = ex2(e.y);
              part[n][0] += pr[n][st][i], part[n][1] += pr[n][st][i + 1];
            }
        }
      };
      weigh();
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) grows = grows || part[n][c] > WEIGHT_MOST || top[n][c] == -INFINITY;
      if (__any_sync(0xffffffffu, grows)) {
      float now[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float m = fmaxf(x[n][0][c], x[n][0][c + 2]);
#pragma unroll
          for (int st = 1; st < SUB; ++st) m = fmaxf(m, fmaxf(x[n][st][c], x[n][st][c + 2]));
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
          now[n][c] = fmaxf(m, top[n][c]);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) v_max = fmaxf(v_max, __shfl_xor_sync(0xffffffffu, v_max, off));
        float shrink = 1.f;
        if (v_max > v_unit) {
          // the power of two above the largest (at least the least fp16, so that its inverse is finite)
          const float unit = __uint_as_float((__float_as_uint(v_max) & 0x7F800000u) + 0x00800000u);
          shrink = v_unit / unit;
          v_unit = unit;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float keep[2];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            keep[c] = now[n][c] == -INFINITY ? 1.f : ex2((top[n][c] - now[n][c]) * cf[n][c]);
            top[n][c] = now[n][c];
            sum[n][c] *= keep[c];
#pragma unroll
            for (int g = 0; g < G; ++g) centre[n][g][c] *= keep[c];
            keep[c] *= shrink;
          }
#pragma unroll
          for (int g = 0; g < G; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              ones[n][g][i] *= keep[i & 1];
#pragma unroll
              for (int j = 0; j < 4; ++j) o[n][g][i][j] *= keep[j & 1];
            }
          }
        }
        weigh();
      }
      const float weight_unit = v_unit > 0.f ? WEIGHT_UNIT / v_unit : 0.f;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) sum[n][c] += part[n][c];
#pragma unroll
      for (int st = 0; st < SUB; ++st) {
        const uint32_t vb = base + CODES + (16 * st + tig) * (HD / 2) + gid * 4;
        uint32_t pf[NT][G][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
              const float s = half_lo(vpar[st][i >> 1][g]) * weight_unit, d = half_hi(vpar[st][i >> 1][g]);
              centre[n][g][0] = fmaf(pr[n][st][i], d, centre[n][g][0]);
              centre[n][g][1] = fmaf(pr[n][st][i + 1], d, centre[n][g][1]);
              w[i] = pr[n][st][i] * s, w[i + 1] = pr[n][st][i + 1] * s;
            }
            pf[n][g][0] = transpose8x8(pack_half2(w[0], w[1]));
            pf[n][g][1] = transpose8x8(pack_half2(w[2], w[3]));
          }
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const uint32_t wa = lds32(vb + g * 32), wb = lds32(vb + g * 32 + 4 * (HD / 2));
          const uint32_t wc = lds32(vb + g * 32 + 8 * (HD / 2)), wd = lds32(vb + g * 32 + 12 * (HD / 2));
          // [byte 0 or 1 of the tokens' words' lower, upper half][which two tokens]: the pairs of two tiles of 16 channels
          uint32_t x0[2][2], x1[2][2], y0[2][2], y1[2][2];  // low and high nibbles of: lower half, upper half
          code_pairs(__byte_perm(wa, wb, 0x5410), x0[0][0], x1[0][0]);
          code_pairs(__byte_perm(wa, wb, 0x5511), x0[1][0], x1[1][0]);
          code_pairs(__byte_perm(wa, wb, 0x7632), y0[0][0], y1[0][0]);
          code_pairs(__byte_perm(wa, wb, 0x7733), y0[1][0], y1[1][0]);
          code_pairs(__byte_perm(wc, wd, 0x5410), x0[0][1], x1[0][1]);
          code_pairs(__byte_perm(wc, wd, 0x5511), x0[1][1], x1[1][1]);
          code_pairs(__byte_perm(wc, wd, 0x7632), y0[0][1], y1[0][1]);
          code_pairs(__byte_perm(wc, wd, 0x7733), y0[1][1], y1[1][1]);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint32_t b0 = pf[n][g][0], b1 = pf[n][g][1];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              mma16816(o[n][g][2 * j], x0[j][0], y0[j][0], x0[j][1], y0[j][1], b0, b1);
              mma16816(o[n][g][2 * j + 1], x1[j][0], y1[j][0], x1[j][1], y1[j][1], b0, b1);
            }
            mma16816(ones[n][g], 0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u, b0, b1);
          }
        }
      }
    }
    __syncwarp();  // (every lane has read the slot)
    if (fetch_flat < w1) issue();
    if (++slot == F::SLOTS) slot = 0, phase ^= 1;

    // ---- the end of a (sequence, head), or of this warp's piece of it
    const bool ends = at.tile + 1 == at.n_tiles;
    const int64_t next = flat + (ends ? 2 : 1);
    if (ends || next >= w1) {
      const int64_t seg_first = flat - at.tile;
      const bool alone = ends && seg_first >= w0;
      const float unit = v_unit * (1.f / WEIGHT_UNIT);
      // a result that others continue goes to global memory while the ring is in use, else into the ring
      const bool last = next >= w1;
      float *part = last ? reinterpret_cast<float *>(smem + (size_t)warp * F::SLOTS * F::TILE_BYTES)
                         : block_ws + (size_t)warp * F::PARTIAL;
      if (!alone && lane == 0) part_seg[2 * warp + last] = (at.seq << 10) | (at.head << 2) | at.block;
      __syncwarp();
      // sums over the lanes that share a column
#pragma unroll
      for (int off = 4; off < 32; off <<= 1)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            sum[n][c] += __shfl_xor_sync(0xffffffffu, sum[n][c], off);
#pragma unroll
            for (int g = 0; g < G; ++g) centre[n][g][c] += __shfl_xor_sync(0xffffffffu, centre[n][g][c], off);
          }
      // channels 64 g + 8 gid + 0..7 of column 2 tig + c: o[..][0..3][c], then o[..][0..3][c + 2]
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              o[n][g][i][j] = fmaf(fmaf(o[n][g][i][j], i & 1 ? 1.f / HIGH : 1.f / LOW, -8.f * ones[n][g][j & 1]), unit,
                                   centre[n][g][j & 1]);
      if (!alone) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int col = n * 8 + 2 * tig + c;
#pragma unroll
            for (int g = 0; g < G; ++g) {
              float4 *to = reinterpret_cast<float4 *>(part + col * F::COL + 64 * g + 8 * gid);
              to[0] = make_float4(o[n][g][0][c], o[n][g][1][c], o[n][g][2][c], o[n][g][3][c]);
              to[1] = make_float4(o[n][g][0][c + 2], o[n][g][1][c + 2], o[n][g][2][c + 2], o[n][g][3][c + 2]);
            }
            if (gid == 0) {
              part[COLS * F::COL + col] = top[n][c] == -INFINITY ? -INFINITY : top[n][c] * cf[n][c];
              part[COLS * F::COL + COLS + col] = sum[n][c];
            }
          }
      } else if (!dead) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int col = n * 8 + 2 * tig + c;
            if (col >= rows) continue;
            int64_t token;
            int head;
            row_of<COLS>(at, col, p, token, head);
            const float inv = inverse(sum[n][c]);
#pragma unroll
            for (int g = 0; g < G; ++g) {
              uint32_t h[4];
#pragma unroll
              for (int i = 0; i < 4; ++i)
                h[i] = pack_out<BF16>(o[n][g][2 * (i & 1)][c + (i & 2)] * inv, o[n][g][2 * (i & 1) + 1][c + (i & 2)] * inv);
              uint16_t *out = reinterpret_cast<uint16_t *>(p.out.row(token, head)) + 64 * g + 8 * gid;
              if (p.out_wide) {
                *reinterpret_cast<uint4 *>(out) = make_uint4(h[0], h[1], h[2], h[3]);
              } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = (uint16_t)(h[i / 2] >> 16 * (i & 1));
              }
            }
            if (gid == 0 && p.lse)
              p.lse[token * p.n_heads + head] =
                  sum[n][c] == 0.f ? -INFINITY : 0.69314718056f * (top[n][c] * cf[n][c]) + logf(sum[n][c]);
          }
      }
    }
    if (next < w1) next_tile<COLS>(at, info, prefix, p);
    flat = next;
  }

  // ---- partial results of this block, in list order ([warp][0: its first segment's, 1: its last's], without the
  // places that hold none): those of a segment are neighbours, a group
  __syncthreads();
  {  // (every warp makes the same list, and waits for no other)
    const int id = lane < 2 * W ? part_seg[lane] : -1;
    const unsigned there = __ballot_sync(0xffffffffu, id >= 0);
    const unsigned before = there & ((1u << lane) - 1);
    const int last_id = __shfl_sync(0xffffffffu, id, before ? 31 - __clz(before) : 0);
    const bool opens = id >= 0 && (before == 0 || last_id != id);
    const unsigned groups = __ballot_sync(0xffffffffu, opens);
    if (id >= 0) part_place[__popc(before)] = lane;
    if (opens) {
      const int k = __popc(groups & ((1u << lane) - 1));
      group_seg[k] = id, group_at[k] = __popc(before);
    }
    if (lane == 0) n_groups[0] = __popc(groups), group_at[__popc(groups)] = __popc(there);
    __syncwarp();
  }
  // a segment's places in the list, and how it stands to this block's: whole, or begun (0) or continued (1) elsewhere
  const auto segment = [&](int id, Cursor &c, int64_t &sa, int64_t &sb) {
    c.seq = id >> 10, c.head = id >> 2 & 255, c.block = id & 3;
    enter_sequence<COLS>(c, info, prefix, p);
    sa = (int64_t)prefix[c.seq] * heads + (c.head * c.blocks + c.block) * (c.n_tiles + 1) + 1, sb = sa + c.n_tiles;
  };
  Cursor seg;
  int64_t sa, sb;
  // part i of a segment that is cut, from block `first` on: the block where it begins has it as its last part, the others as
  // their first
  const auto part_of = [&](int first, int i) {
    return static_cast<const float *>(p.partials + ((size_t)(first + i) * (W + 2) + W + (i == 0)) * F::PARTIAL);
  };
  bool staged = false;
  const auto merge = [&](auto columns, int across, int groups) {
    constexpr int NC = decltype(columns)::value;
    for (int u = warp; u < groups * (COLS / NC); u += W) {
      const int k = u / (COLS / NC), col = u % (COLS / NC) * NC, id = across ? cut[k] : group_seg[k];
      if (id < 0) continue;
      segment(id, seg, sa, sb);
      const int rows_here = seg.count * p.group - seg.block * COLS;
      if (col >= rows_here) continue;
      const int first = across ? span[2 * k] : group_at[k], n = across ? span[2 * k + 1] : group_at[k + 1] - first;
      const auto nth = [&](int i) {
        if (across)
          return staged ? reinterpret_cast<const float *>(smem) + (k * span[1] + i) * F::PARTIAL : part_of(first, i);
        const int at = part_place[first + i];
        return at & 1 ? reinterpret_cast<const float *>(smem + (size_t)(at >> 1) * F::SLOTS * F::TILE_BYTES)
                      : static_cast<const float *>(block_ws + (at >> 1) * F::PARTIAL);
      };
      alignas(16) float v[NC][HD / 32], tops[NC], sums[NC];
      merge_columns<HD, COLS, NC>(n, col, lane, nth, v, tops, sums);
      const bool whole = across || (sa >= c0 && sb <= c1);
      float *to = block_ws + (W + (sa < c0 ? 0 : 1)) * F::PARTIAL;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (whole) {
          if (col + c < rows_here) store_row<HD, COLS, BF16>(p, seg, col + c, lane, v[c], tops[c], sums[c]);
        } else {
          using Vec = typename std::conditional<HD == 128, float4, float2>::type;
          *reinterpret_cast<Vec *>(to + (col + c) * F::COL + lane * (HD / 32)) = *reinterpret_cast<const Vec *>(v[c]);
          if (lane == 0) to[COLS * F::COL + col + c] = tops[c], to[COLS * F::COL + COLS + col + c] = sums[c];
        }
      }
    }
  };
  // First the block's own partial results, then those that blocks have left to this one as the last to arrive: the same
  // code, which costs more the first time than what it does.  A warp takes two columns at a time, or four where two would
  // need another round (32 ragged users: 1.4 us less than with two; 136 keys: 0.4 us less than with four)
#pragma unroll 1
  for (int across = 0; across < 2; ++across) {
    const int groups = across ? 2 : n_groups[0];
    if (NT == 1 && groups * (COLS / 2) <= W)
      merge(std::integral_constant<int, NT == 1 ? 2 : 4>(), across, groups);
    else
      merge(std::integral_constant<int, 4>(), across, groups);
    if (across) break;
    // ---- segments that other blocks have parts of: the first and the last group at most.  (The last warps, which have
    // fewer columns to merge)
    const int k = W - 1 - warp;
    int mine = -1, from = 0, to = 0;
    if (lane == 0 && k < 2 && n_groups[0] > k) {
      mine = group_seg[k == 0 ? 0 : n_groups[0] - 1];
      segment(mine, seg, sa, sb);
      if (sa < c0 || sb > c1)
        from = (int)quotient(sa, quota), to = (int)quotient(sb - 1, quota);
      else
        mine = -1;
    }
    __syncthreads();
    if (lane == 0 && k < 2) {
      if (mine >= 0) {
        unsigned *ticket = p.tickets + (seg.seq * heads + seg.head) * p.most_blocks + seg.block;
        if (atom_add_acq_rel(ticket, 1u) == (unsigned)(to - from))
          atomicExch(ticket, 0u);  // as the next call has to find it
        else
          mine = -1;
      }
      cut[k] = mine, span[2 * k] = from, span[2 * k + 1] = mine < 0 ? 0 : to - from + 1;
    }
    __syncthreads();
    const int parts = span[1] + span[3];
    if (parts == 0) return;
    // all of them into the ring, where there is room: one round trip instead of one for every four
    staged = parts <= F::RING_BYTES / (F::PARTIAL * 4);
    if (staged) {
      for (int i = warp; i < parts; i += W) {
        const bool second = i >= span[1];
        const float *src = part_of(span[second ? 2 : 0], second ? i - span[1] : i);
        float *dst = reinterpret_cast<float *>(smem) + i * F::PARTIAL;
        for (int j = 4 * lane; j < F::PARTIAL; j += 128) cp_async16(dst + j, src + j);
      }
      cp_async_commit();
      cp_async_wait<0>();
      __syncthreads();
    }
  }
}

template <int HD, int NT, bool BF16>
cudaError_t launch(const AttendParams &p, int n_sm, cudaStream_t s) {
  using F = Few<HD, NT>;
  static SmemOptIn opt_in;
  const void *kernel = reinterpret_cast<const void *>(&kv4_attend_few_kernel<HD, NT, BF16>);
  const cudaError_t e = opt_in(kernel, F::SMEM);
  if (e != cudaSuccess) return e;
  // as many blocks as the longest contexts could fill
  const int64_t most = (int64_t)p.n_seqs * p.pool.n_kv_heads * p.most_blocks *
                       (((int64_t)p.map.max_pages << p.pool.log2_tokens) / TILE + 2);
  const unsigned grid = (unsigned)std::min<int64_t>(std::min(n_sm, FEW_BLOCKS), (most + F::WARPS - 1) / F::WARPS);
  return launch_chained(kv4_attend_few_kernel<HD, NT, BF16>, grid, F::THREADS, F::SMEM, s, p);
}

}  // namespace

size_t attend_few_partials(int head_dim, int cols) {
  const size_t floats = head_dim == 128 ? (cols <= 8 ? (size_t)Few<128, 1>::PARTIAL * (Few<128, 1>::WARPS + 2)
                                                     : (size_t)Few<128, 2>::PARTIAL * (Few<128, 2>::WARPS + 2))
                                        : (cols <= 8 ? (size_t)Few<64, 1>::PARTIAL * (Few<64, 1>::WARPS + 2)
                                                     : (size_t)Few<64, 2>::PARTIAL * (Few<64, 2>::WARPS + 2));
  return FEW_BLOCKS * floats * sizeof(float);
}

template <bool BF16>
static cudaError_t launch_type(const AttendParams &p, int cols, int n_sm, cudaStream_t s) {
  if (p.pool.head_dim == 128) return cols <= 8 ? launch<128, 1, BF16>(p, n_sm, s) : launch<128, 2, BF16>(p, n_sm, s);
  return cols <= 8 ? launch<64, 1, BF16>(p, n_sm, s) : launch<64, 2, BF16>(p, n_sm, s);
}
cudaError_t launch_attend_few(const AttendParams &p, int cols, int n_sm, cudaStream_t s) {
  return p.bf16 ? launch_type<true>(p, cols, n_sm, s) : launch_type<false>(p, cols, n_sm, s);
}

}  // namespace kfl
