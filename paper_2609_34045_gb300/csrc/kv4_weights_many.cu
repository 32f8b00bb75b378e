// The attention weight that many query rows of a KV head (a prompt's) give its cached rows, on tcgen05
// (include/kafila_kv4_evict.h).
//
// Mathematics.  A key t and a query row j, in groups g of 64 channels:
//   a_tjg = sum_c (u_tc - 8) q_jc,   mass_t += sum_j 2^( sum_g s_tg a_tjg + sum_g c_tg sum_c q_jc - log2(e) lse_j )
// (s, c: the key's scale and centre times scale log2(e)).  The a are matrix products of the codes, which are exact as fp16 or
// bf16, with the queries as they stand, in their own type: nothing is rounded before the fp32 sums.  Scales and centres
// act on the sums, four fused operations a score with two groups.
//
// What bounds it.  An exponential a score: 16 a clock and SM, 1024 clocks for a unit of 256 keys by 64 rows, whose products take
// some 600 and whose other fp32 work about 700 of the issue slots.
//
// Roles.  Warps 0-15: two threads per key (32 rows of a unit each), keys on the tensor memory's lanes, so that a key's weights
// are summed in a register.  They also decode their keys, into tensor memory: the products' first operand.  16-19: queries, a
// thread per row, into swizzled shared memory, with the sums and log-sum-exps; 20: products.
//
// Work split.  The units (sequence, KV head, 256 keys, 64 rows) in sight form one list that the blocks share equally, rows
// fastest: a block decodes its keys once.  Keys whose rows are cut between blocks are summed by the last to arrive, in list
// order, so results do not depend on arrival.
#include <algorithm>

#include "kv4_tc.cuh"
#include "kv4_weights.cuh"

namespace kfl {
namespace {

constexpr int WM_KEYS = 256, WM_ROWS = 64;
constexpr int WM_SUMMERS = 16, WM_LOADERS = 4;  // warps
constexpr int WM_MMA_WARP = WM_SUMMERS + WM_LOADERS;
constexpr int WM_THREADS = (WM_MMA_WARP + 1) * 32;
constexpr int WM_STAGES = 4;  // of queries

template <int HD>
struct Many {
  static constexpr int GROUPS = HD / 64;
  static constexpr int STAGE = WM_ROWS * HD * 2;   // bytes of a unit's queries
  static constexpr int A_COLS = HD / 2;            // of a half's keys (128) in tensor memory
  static constexpr int D_COLS = GROUPS * WM_ROWS;  // of a half's sums
  static constexpr int BUFFERS = HD == 128 ? 3 : 4;
  static constexpr int D_AT = 2 * A_COLS;
  static_assert(D_AT + BUFFERS * D_COLS <= 512, "tensor memory");
  static constexpr int ROWS_AT = WM_STAGES * STAGE;              // float [stages][4][64]: sums of both groups, -lse, end
  static constexpr int SUM_AT = ROWS_AT + WM_STAGES * 4 * WM_ROWS * 4;  // float [256]: the second threads' sums
  static constexpr int INFO_AT = SUM_AT + WM_KEYS * 4;           // int4 [FEW_SEQS], then int prefix[FEW_SEQS + 4]
  static constexpr int BAR_AT = INFO_AT + FEW_SEQS * 16 + (FEW_SEQS + 4) * 4;
  static constexpr int N_BARS = 2 * WM_STAGES + 2 * 4 + 2 + 1;
  static constexpr int SMEM = BAR_AT + N_BARS * 8 + 32;
};
// Barriers.  Sums are done by half and by the unit's parity (a half's next-but-one job waits, through the buffers, for this one
// to be read), buffers and stages are free again by number.
enum { W_QFULL = 0, W_QFREE = WM_STAGES, W_DFULL = 2 * WM_STAGES, W_DFREE = W_DFULL + 4, W_A = W_DFREE + 4, W_DRAIN = W_A + 2 };

// A run of one key tile's units.
struct Keys {
  int seq, head, tile;
  int user, length, first, count;
  int first_tile, n_tiles;  // of the sequence
  int row_tile, n;          // the tile's first row tile and how many see it
  int from, to;             // this block's run of them
  int64_t flat;             // place of its first unit in the list
};
struct WmList {
  const int4 *info;
  const int *prefix;
  int n_seqs, heads, group, window;
};

// Which rows, in tiles of 64, see a key of the tile (at least one does, between a sequence's first tile and its last).
__device__ __forceinline__ void rows_of_tile(int length, int count, int tile, const WmList &l, int &row_tile, int &n) {
  const int base = length - count, k0 = tile * WM_KEYS, k1 = min(k0 + WM_KEYS, length);
  const int t0 = max(0, k0 - base), t1 = l.window > 0 ? min(count, k1 - base - 1 + l.window) : count;
  row_tile = t0 * l.group / WM_ROWS;
  n = (t1 * l.group + WM_ROWS - 1) / WM_ROWS - row_tile;
}
__device__ __forceinline__ void enter(Keys &k, const WmList &l) {
  const int4 v = l.info[k.seq];
  k.user = v.x, k.length = v.y, k.first = v.z, k.count = v.w;
  k.first_tile = l.window > 0 ? max(0, v.y - v.w + 1 - l.window) / WM_KEYS : 0;
  k.n_tiles = (v.y + WM_KEYS - 1) / WM_KEYS;
}
__device__ __forceinline__ void open(Keys &k, const WmList &l, int skip, int64_t limit) {
  rows_of_tile(k.length, k.count, k.tile, l, k.row_tile, k.n);
  k.from = skip, k.to = (int)min((int64_t)k.n, limit - k.flat);
}
// The run at place `at` of the list (at < limit).  The whole warp calls it: lanes count a tile's units each.
__device__ void find_keys(Keys &k, const WmList &l, int64_t at, int64_t limit) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = l.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if ((int64_t)l.prefix[mid + 1] * l.heads > at)
      hi = mid;
    else
      lo = mid + 1;
  }
  k.seq = lo;
  enter(k, l);
  const int64_t start = (int64_t)l.prefix[lo] * l.heads;
  const int per_head = l.prefix[lo + 1] - l.prefix[lo];
  k.head = (int)((at - start) / per_head);
  const int rest = (int)(at - start - (int64_t)k.head * per_head);
  int before = 0;
  for (int b0 = k.first_tile;; b0 += 32) {
    int row_tile, n = 0;
    if (b0 + lane < k.n_tiles) rows_of_tile(k.length, k.count, b0 + lane, l, row_tile, n);
    int sum = n;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, sum, off);
      if (lane >= off) sum += o;
    }
    const unsigned here = __ballot_sync(0xffffffffu, before + sum > rest);
    if (here != 0 || b0 + 32 >= k.n_tiles) {
      const int i = here ? __ffs(here) - 1 : 31;
      k.tile = b0 + i;
      before += __shfl_sync(0xffffffffu, sum - n, i);
      break;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  k.flat = start + (int64_t)k.head * per_head + before;
  open(k, l, (int)(at - k.flat), limit);
}
__device__ void next_keys(Keys &k, const WmList &l, int64_t limit) {  // (the list goes on to `limit`)
  k.flat += k.n;
  if (++k.tile == k.n_tiles) {
    if (++k.head == l.heads) {
      k.head = 0;
      do {
        ++k.seq;
      } while (l.prefix[k.seq + 1] == l.prefix[k.seq]);
      enter(k, l);
    }
    k.tile = k.first_tile;
  }
  open(k, l, 0, limit);
}

__device__ __forceinline__ float wm_ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Eight codes (a word's nibbles, in channel order) as four pairs of fp16 or bf16, less 8: the nibbles become the last bits of
// 1024 (128) + u, exactly.
template <bool BF16>
__device__ __forceinline__ void decode8(uint32_t w, uint32_t (&out)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t b = w >> 8 * i;
    const uint32_t u = (b & 0xFu) | ((b & 0xF0u) << 12);
    if (BF16)
      asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(out[i]) : "r"(u | 0x43004300u), "r"(0x3F803F80u), "r"(0xC308C308u));
    else
      out[i] = hfma2(u | 0x64006400u, 0x3C003C00u, 0xE408E408u);
  }
}

template <int HD, bool BF16>
__global__ void __launch_bounds__(WM_THREADS, 1) kv4_weights_many_kernel(const WeightParams p) {
  using F = Many<HD>;
  constexpr int G = F::GROUPS, NB = F::BUFFERS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  const uint32_t base = smem_addr(smem);
  int4 *info = reinterpret_cast<int4 *>(smem + F::INFO_AT);
  int *prefix = reinterpret_cast<int *>(info + FEW_SEQS);
  volatile uint32_t *words = reinterpret_cast<volatile uint32_t *>(smem + F::BAR_AT + F::N_BARS * 8);  // TMEM, abort, last
  const auto bar = [&](int b) { return base + F::BAR_AT + 8 * b; };
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int heads = p.pool.n_kv_heads, lp = p.pool.log2_tokens;
  const WmList list = {info, prefix, p.n_seqs, heads, p.group, p.window};
  if (tid == 0) {
    for (int i = 0; i < WM_STAGES; ++i) {
      mbar_init(bar(W_QFULL + i), 2);
      mbar_init(bar(W_QFREE + i), 1 + WM_SUMMERS);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(W_DFULL + i), 1);
      mbar_init(bar(W_DFREE + i), WM_SUMMERS / 2);
    }
    for (int i = 0; i < 2; ++i) mbar_init(bar(W_A + i), WM_SUMMERS / 2);
    mbar_init(bar(W_DRAIN), 1);
    words[1] = 0;
    prefix[0] = 0;
  }
  fence_mbar_init();
  if (warp == WM_MMA_WARP) tmem_alloc(base + F::BAR_AT + F::N_BARS * 8, 512);
  pdl_wait();

  // ---- the list: every sequence's units per head, summed
  for (int s = warp; s < p.n_seqs; s += WM_THREADS / 32) {
    bool again = false;
    if (p.all_users)
      for (int j = lane; j < p.seq0 + s; j += 32) again |= p.all_users[j] == p.users[s];
    const int4 v = weight_sequence(p, s, __any_sync(0xffffffffu, again), blockIdx.x == 0 && lane == 0);
    int64_t units = 0;
    if (v.w > 0)
      for (int b = (p.window > 0 ? max(0, v.y - v.w + 1 - p.window) / WM_KEYS : 0) + lane; b * WM_KEYS < v.y; b += 32) {
        int row_tile, n;
        rows_of_tile(v.y, v.w, b, list, row_tile, n);
        units += n;
      }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) units += __shfl_xor_sync(0xffffffffu, units, off);
    if (lane == 0) info[s] = v, prefix[s + 1] = (int)min(units, (int64_t)0x7fffffff);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = words[0];
  // (not before this block has its tensor memory: a block of the next kernel that took it first would wait for this grid's end,
  // and this block for that one's)
  pdl_launch_dependents();
  if (warp == 0) {
    int64_t before = 0;
    for (int s0 = 0; s0 < p.n_seqs; s0 += 32) {
      int64_t v = s0 + lane < p.n_seqs ? prefix[s0 + lane + 1] : 0;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, v, off);
        if (lane >= off) v += o;
      }
      if (s0 + lane < p.n_seqs) prefix[s0 + lane + 1] = (int)(before + v);
      before += __shfl_sync(0xffffffffu, v, 31);
    }
    // (a list of that many units would run for seconds: refused)
    if (before >= 0x7fffffff) {
      __syncwarp();
      if (lane == 0) prefix[p.n_seqs] = 0;
      if (blockIdx.x == 0 && lane == 0) report(p.status, KFL_BAD_POSITION);
    }
  }
  __syncthreads();
  const int64_t total = (int64_t)prefix[p.n_seqs] * heads;
  const int64_t quota = max((total + gridDim.x - 1) / gridDim.x, (int64_t)1);
  const int64_t c0 = min(blockIdx.x * quota, total), c1 = min(c0 + quota, total);

  // a wait that gives up lets no later one last
  const auto wait = [&](int b, uint32_t parity) {
    if (mbar_try_wait(bar(b), parity)) return true;
    if (words[1]) return false;
    if (wait_2s(bar(b), parity)) return true;
    words[1] = 1;
    report(p.status, KFL_TIMED_OUT);
    return false;
  };

  if (c0 < c1 && warp < WM_SUMMERS) {
    // ---- keys: two threads each, with 32 of a unit's rows
    const int half = warp >> 2 & 1, part = warp >> 3, key = half * 128 + (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // TMEM lane 32 (warp mod 4), in bits 16 up
    float *second = reinterpret_cast<float *>(smem + F::SUM_AT);
    const float factor = p.scale * 1.44269504089f;
    unsigned unit = 0, tiles = 0;
    Keys k;
    find_keys(k, list, c0, c1);
    for (;;) {
      // ---- its codes, into tensor memory (all products with the ones before have been waited for), half of them each
      const int slot = k.tile * WM_KEYS + key;
      bool there = false;
      float2 s[G], c[G];
      bool odd = false;  // a scale or centre that is no number
      {
        uint32_t par[G] = {};
        uint4 raw[HD / 64] = {};
        if (slot < k.length) {
          const int page = p.map.table[(int64_t)k.user * p.map.max_pages + (slot >> lp)];
          there = page >= 0 && page < p.pool.n_pages;
          if (there) {
            const uint8_t *b = p.pool.block(page, p.layer, k.head);
            const int at = slot & (p.pool.page_tokens() - 1);
            const uint4 *codes = reinterpret_cast<const uint4 *>(b + at * (HD / 2)) + part * (HD / 64);
            const uint32_t *params = reinterpret_cast<const uint32_t *>(b + 2 * p.pool.code_bytes() + at * (G * 4));
#pragma unroll
            for (int i = 0; i < HD / 64; ++i) raw[i] = codes[i];
#pragma unroll
            for (int g = 0; g < G; ++g) par[g] = params[g];
          } else if (part == 0) {
            report(p.status, KFL_BAD_PAGE);
          }
        }
        uint32_t w[HD / 4];
#pragma unroll
        for (int i = 0; i < HD / 64; ++i) {
          decode8<BF16>(raw[i].x, reinterpret_cast<uint32_t(&)[4]>(w[16 * i]));
          decode8<BF16>(raw[i].y, reinterpret_cast<uint32_t(&)[4]>(w[16 * i + 4]));
          decode8<BF16>(raw[i].z, reinterpret_cast<uint32_t(&)[4]>(w[16 * i + 8]));
          decode8<BF16>(raw[i].w, reinterpret_cast<uint32_t(&)[4]>(w[16 * i + 12]));
        }
#pragma unroll
        for (int i = 0; i < HD / 64; ++i)
          tmem_st16(tmem + lanes + half * F::A_COLS + part * (HD / 4) + 16 * i, reinterpret_cast<uint32_t(&)[16]>(w[16 * i]));
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(W_A + half));
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const float a = f16_to_f32((uint16_t)par[g]) * factor, b = f16_to_f32((uint16_t)(par[g] >> 16)) * factor;
          s[g] = {a, a}, c[g] = {b, b};
          odd = odd || (par[g] & 0x7c00u) == 0x7c00u || (par[g] & 0x7c000000u) == 0x7c000000u;
        }
      }
      const bool any_odd = __any_sync(0xffffffffu, odd);
      const int key0 = slot - lane, before = k.length - k.count;
      float2 sum = {0.f, 0.f};
      for (int t = k.from; t < k.to; ++t, ++unit) {
        const unsigned stage = unit % WM_STAGES, job = 2 * unit + half, buf = job % NB;
        const int row0 = (k.row_tile + t) * WM_ROWS;
        const int least = before + row0 / p.group + 1, most = before + min(k.count - 1, (row0 + WM_ROWS - 1) / p.group) + 1;
        const bool masked = any_odd || key0 + 32 > least || (p.window > 0 && key0 < most - p.window);
        wait(W_QFULL + stage, unit / WM_STAGES & 1);
        wait(W_DFULL + 2 * half + (unit & 1), unit >> 1 & 1);
        __syncwarp();
        tc_fence_after();
        const float *rows = reinterpret_cast<const float *>(smem + F::ROWS_AT) + stage * 4 * WM_ROWS + part * 32;
        const uint32_t d = tmem + lanes + F::D_AT + buf * F::D_COLS + part * 32;
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += 16) {
          uint32_t a[G][16];
#pragma unroll
          for (int g = 0; g < G; ++g) tmem_ld16(d + g * WM_ROWS + r0, a[g]);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            float4 q[G];
#pragma unroll
            for (int g = 0; g < G; ++g) q[g] = *reinterpret_cast<const float4 *>(rows + g * WM_ROWS + r0 + i);
            const float4 nl = *reinterpret_cast<const float4 *>(rows + 2 * WM_ROWS + r0 + i);
            float2 x0 = {nl.x, nl.y}, x1 = {nl.z, nl.w};
#pragma unroll
            for (int g = 0; g < G; ++g) {
              x0 = fma2(c[g], {q[g].x, q[g].y}, x0), x1 = fma2(c[g], {q[g].z, q[g].w}, x1);
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
              x0 = fma2(s[g], {__uint_as_float(a[g][i]), __uint_as_float(a[g][i + 1])}, x0);
              x1 = fma2(s[g], {__uint_as_float(a[g][i + 2]), __uint_as_float(a[g][i + 3])}, x1);
            }
            float2 w0 = {wm_ex2(x0.x), wm_ex2(x0.y)}, w1 = {wm_ex2(x1.x), wm_ex2(x1.y)};
            if (masked) {
              const int4 e = *reinterpret_cast<const int4 *>(rows + 3 * WM_ROWS + r0 + i);
              const auto sees = [&](int end) { return slot < end && (p.window == 0 || slot >= end - p.window); };
              w0 = {sees(e.x) ? w0.x : 0.f, sees(e.y) ? w0.y : 0.f};
              w1 = {sees(e.z) ? w1.x : 0.f, sees(e.w) ? w1.y : 0.f};
            }
            sum = add2(sum, add2(w0, w1));
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(W_DFREE + buf));
          mbar_arrive(bar(W_QFREE + stage));
        }
      }
      // ---- the tile's end: both threads' sums, added to the mass or handed on
      const int pair = half * 4 + (warp & 3);
      if (part == 1) second[key] = sum.x + sum.y;
      named_bar_sync(1 + pair, 64);
      if (part == 0) {
        const float all = sum.x + sum.y + second[key];
        if (k.from == 0 && k.to == k.n) {
          if (there) {
            float *m = p.mass.row(p.layer, k.user, k.head) + slot;
            *m += all;
          }
        } else {
          p.partials[((size_t)blockIdx.x * 2 + (k.from > 0 ? 0 : 1)) * WM_KEYS + key] = all;
        }
      }
      named_bar_sync(1 + pair, 64);  // (before the second sums are written again)
      ++tiles;
      if (k.flat + k.to >= c1) break;
      next_keys(k, list, c1);
    }
  } else if (c0 < c1 && warp < WM_MMA_WARP) {
    // ---- queries: two warps for every other unit, a thread per row
    const int mine = (warp - WM_SUMMERS) >> 1, r = (warp & 1) * 32 + lane;
    unsigned unit = 0;
    Keys k;
    find_keys(k, list, c0, c1);
    for (;;) {
      for (int t = k.from; t < k.to; ++t, ++unit) {
        if ((int)(unit & 1) != mine) continue;
        const int row = (k.row_tile + t) * WM_ROWS + r, token = row / p.group, head = k.head * p.group + row - token * p.group;
        const bool there = row < k.count * p.group;
        uint4 v[HD / 8] = {};
        float lse = -INFINITY;
        if (there) {
          lse = p.lse[((int64_t)k.first + token) * p.n_heads + head];
          const uint16_t *src = reinterpret_cast<const uint16_t *>(p.q.row((int64_t)k.first + token, head));
          if (p.q_wide) {
#pragma unroll
            for (int i = 0; i < HD / 8; ++i) v[i] = reinterpret_cast<const uint4 *>(src)[i];
          } else {
#pragma unroll
            for (int i = 0; i < HD / 8; ++i) {
              uint32_t *w = reinterpret_cast<uint32_t *>(&v[i]);
#pragma unroll
              for (int j = 0; j < 4; ++j) w[j] = src[8 * i + 2 * j] | ((uint32_t)src[8 * i + 2 * j + 1] << 16);
            }
          }
        }
        // (a row that saw nothing adds nothing, whatever it holds)
        const bool counts = lse != -INFINITY;
        float sums[2] = {};
#pragma unroll
        for (int i = 0; i < HD / 8; ++i) {
          if (!counts) v[i] = make_uint4(0, 0, 0, 0);
          const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
          float e[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            e[j] = BF16 ? bf16_lo(w[j]) + bf16_hi(w[j]) : f16_to_f32((uint16_t)w[j]) + f16_to_f32((uint16_t)(w[j] >> 16));
          sums[i / 8] += e[0] + e[1] + (e[2] + e[3]);
        }
        const unsigned stage = unit % WM_STAGES;
        wait(W_QFREE + stage, unit / WM_STAGES & 1 ^ 1);
        __syncwarp();
        const uint32_t to = base + stage * F::STAGE + r * 128;
#pragma unroll
        for (int i = 0; i < HD / 8; ++i)
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (i / 8) * (WM_ROWS * 128) + (((i & 7) ^ (r & 7)) << 4)),
                       "r"(v[i].x), "r"(v[i].y), "r"(v[i].z), "r"(v[i].w)
                       : "memory");
        float *rows = reinterpret_cast<float *>(smem + F::ROWS_AT) + stage * 4 * WM_ROWS + r;
        rows[0] = sums[0], rows[WM_ROWS] = sums[1];
        rows[2 * WM_ROWS] = counts ? lse * -1.44269504089f : -INFINITY;
        reinterpret_cast<int *>(rows)[3 * WM_ROWS] = counts ? k.length - k.count + token + 1 : -1;
        fence_async_proxy();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(W_QFULL + stage));
      }
      if (k.flat + k.to >= c1) break;
      next_keys(k, list, c1);
    }
  } else if (c0 < c1) {
    // ---- products, issued by an elected lane (descriptors through shuffles: known to be the same in every lane)
    constexpr uint32_t idesc = idesc_kind_f16(128, WM_ROWS, BF16);
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), at = __shfl_sync(0xffffffffu, base, 0);
    unsigned unit = 0, tiles = 0;
    bool ok = true;
    Keys k;
    find_keys(k, list, c0, c1);
    for (;; ++tiles) {
      const int n = __shfl_sync(0xffffffffu, k.to - k.from, 0);
      for (int t = 0; t < n; ++t, ++unit) {
        const unsigned stage = __shfl_sync(0xffffffffu, unit % WM_STAGES, 0);
        ok = wait(W_QFULL + stage, unit / WM_STAGES & 1);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const unsigned job = 2 * unit + half, buf = __shfl_sync(0xffffffffu, job % NB, 0);
          if (t == 0) ok = ok && wait(W_A + half, tiles & 1);
          ok = ok && wait(W_DFREE + buf, job / NB & 1 ^ 1);
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
          tc_fence_after();
          const uint64_t q = sdesc_k_sw128(at + stage * F::STAGE);
          const uint32_t d = tm + F::D_AT + buf * F::D_COLS, a = tm + half * F::A_COLS;
          if (elect_one()) {
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
              for (int i = 0; i < 4; ++i)  // (descriptors count 16 bytes)
                mma_ts(d + g * WM_ROWS, a + g * 32 + i * 8, q + g * (WM_ROWS * 128 >> 4) + i * 2, idesc, i > 0);
            mma_commit(bar(W_DFULL + 2 * half + (unit & 1)));
            if (half == 1) mma_commit(bar(W_QFREE + stage));
          }
          __syncwarp();
        }
        if (!ok) break;
      }
      if (!ok || k.flat + k.to >= c1) break;
      next_keys(k, list, c1);
    }
    // every product has to be done before the tensor memory goes
    if (elect_one()) mma_commit(bar(W_DRAIN));
    __syncwarp();
    wait_2s(bar(W_DRAIN), 0);
  }
  tc_fence_before();
  __threadfence();
  __syncthreads();
  tc_fence_after();
  if (warp == WM_MMA_WARP) tmem_dealloc(tmem, 512);
  if (c0 >= c1 || words[1]) return;

  // ---- key tiles that other blocks have parts of: this one's first, its last
  for (int i = 0; i < 2; ++i) {
    Keys k;
    find_keys(k, list, i == 0 ? c0 : c1 - 1, c1);
    const int64_t sa = k.flat, sb = sa + k.n;
    if (!(i == 0 ? sa < c0 : sb > c1 && sa >= c0)) continue;
    const int from = (int)(sa / quota), to = (int)((sb - 1) / quota);
    __syncthreads();
    if (tid == 0) {
      unsigned *ticket = p.tickets + from;  // (a tile that is cut begins in one block, as its last one)
      words[2] = atom_add_acq_rel(ticket, 1u) == (unsigned)(to - from);
      if (words[2]) atomicExch(ticket, 0u);
    }
    __syncthreads();
    if (!words[2]) continue;
    const int slot = k.tile * WM_KEYS + tid;
    if (tid < WM_KEYS && slot < k.length) {
      // (the block where the tile begins has it as its last part, the others as their first)
      float all = p.partials[((size_t)from * 2 + 1) * WM_KEYS + tid];
#pragma unroll 8
      for (int j = from + 1; j <= to; ++j) all += p.partials[(size_t)j * 2 * WM_KEYS + tid];
      const int page = p.map.table[(int64_t)k.user * p.map.max_pages + (slot >> lp)];
      if (page >= 0 && page < p.pool.n_pages) p.mass.row(p.layer, k.user, k.head)[slot] += all;
    }
  }
}

template <int HD, bool BF16>
cudaError_t launch(const WeightParams &p, int n_sm, cudaStream_t s) {
  static SmemOptIn opt_in;
  const void *kernel = reinterpret_cast<const void *>(&kv4_weights_many_kernel<HD, BF16>);
  const int smem = Many<HD>::SMEM + 1024;
  const cudaError_t e = opt_in(kernel, smem);
  if (e != cudaSuccess) return e;
  return launch_chained(kv4_weights_many_kernel<HD, BF16>, std::min(n_sm, FEW_BLOCKS), WM_THREADS, smem, s, p);
}

}  // namespace

cudaError_t launch_weights_many(const WeightParams &p, int n_sm, cudaStream_t s) {
  if (p.pool.head_dim == 128) return p.bf16 ? launch<128, true>(p, n_sm, s) : launch<128, false>(p, n_sm, s);
  return p.bf16 ? launch<64, true>(p, n_sm, s) : launch<64, false>(p, n_sm, s);
}

}  // namespace kfl
