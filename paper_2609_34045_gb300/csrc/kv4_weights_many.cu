// The attention weight that many query rows of a KV head (a prompt's) give its cached rows, on tcgen05
// (include/kafila_kv4_evict.h).
//
// Mathematics.  A key t and a query row j, in groups g of 64 channels:
//   a_tjg = sum_c (u_tc - 8) q_jc,   mass_t += sum_j 2^( sum_g s_tg a_tjg + sum_g c_tg Q_jg - log2(e) lse_j ),  Q_jg = sum_c q_jc
// (s, c: the key's scale and centre times scale log2(e)).  The a are matrix products of the codes, which are exact as fp16 or
// bf16, with the queries as they stand, in their own type: nothing is rounded before the fp32 sums.  Scales act on the sums.
// bf16 takes all but the scales along in the products: s_0 (a_0 + (c_0 / s_0) Q_0 - (1 / s_0) log2(e) lse) + s_1 (a_1 + (c_1 /
// s_1) Q_1), each factor as a sum of three bf16 numbers, of whose products the six larger ones are channels more (2^-24 is left
// out): ten instructions for four scores in place of 17, and no load.  (fp16 has not got the exponents for it; a
// key with scale 0, or so small a one that 1 / s_0 is 2^27 and more, takes the long way.)
//
// What bounds it.  2 head_dim flops and an exponential a (query head, visible key).  2048 tokens over 8192 keys, 64/8 heads of 128:
// 305 us in bf16, 0.79 PFLOP/s of the 1.98 that a plain bf16 product reaches, 355 in fp16.  A unit of 256 keys by 128 rows takes
// some 3250 clocks: its products 1400 of the tensor pipe (fed from shared memory at nearly all of its rate), its exponentials 1024, its
// other fp32 operations about 1000 of a scheduler's slots; a half's products and the reading of their sums follow one another, as
// two halves of two groups fill the tensor memory.  Few rows: a tile's keys come, are decoded and multiplied one after
// the other, 5 us a tile of 256 keys however few the rows.
// (Measured slower: 64 rows a product, two sets of sums a half, 382 us for 349 of the form then; four threads a key with all their
// sums loaded at once, 374, a warp for each half's products, 368, and the next tile's keys under way in registers, 314, each for
// 302 of the form then; a barrier for each copy that one warp waits for in every phase made 305 of that.)
//
// Roles.  Warps 0-15: two threads per key (64 rows of a unit each), keys on the tensor memory's lanes, so that a key's weights
// are summed in a register.  They also decode their keys into swizzled shared memory.  16: tensor copies of the queries, which
// need no conversion; 17, 18: every other unit's sums of the queries (as products with ones) and log-sum-exps; 19: products.
// While one half's (128 keys) sums are read, the other half's products run.
//
// Work split.  The units (sequence, KV head, 256 keys, as many tokens as fill 128 rows) in sight form one list that the blocks
// share equally, rows fastest: a block decodes its keys once.  Keys whose rows are cut between blocks are summed by the last to
// arrive, in list order, so results do not depend on arrival.
#include <algorithm>
#include <type_traits>

#include "kv4_tc.cuh"
#include "kv4_weights.cuh"

namespace kfl {
namespace {

constexpr int WM_KEYS = 256, WM_ROWS = 128;
constexpr int WM_SUMMERS = 16;  // warps
constexpr int WM_COPY_WARP = 16, WM_STAT_WARP = 17, WM_MMA_WARP = 19;
constexpr int WM_THREADS = (WM_MMA_WARP + 1) * 32;
constexpr int WM_STAGES = 3;   // of queries, free again when summed and multiplied
constexpr int WM_RECORDS = 4;  // of what is known of the queries' rows, which the sums' readers need for longer
constexpr int WM_FULL = 2 * WM_STAGES;  // barriers of the copies: an even number, so that each is waited for by one of the two
                                        // warps that sum, in every phase

template <int HD>
struct Many {
  static constexpr int GROUPS = HD / 64;
  static constexpr int STAGE = WM_ROWS * HD * 2;   // bytes of a unit's queries
  static constexpr int HALF = 128 * HD * 2;        // of 128 keys
  static constexpr int D_COLS = GROUPS * WM_ROWS;  // of a half's sums in tensor memory
  static constexpr int BUFFERS = 256 / D_COLS;     // of each half
  static constexpr int FOLD = 128 * 32;            // of sixteen more channels of 128 keys or rows: [2][row] of 8
  static constexpr int K_AT = WM_STAGES * STAGE;
  static constexpr int KF_AT = K_AT + 2 * HALF;                        // [half][group]
  static constexpr int QF_AT = KF_AT + 2 * GROUPS * FOLD;              // [stages][group]
  static constexpr int ROWS_AT = QF_AT + WM_STAGES * GROUPS * FOLD;    // float [records][4][128]: sums of both groups, -lse, end
  static constexpr int SUM_AT = ROWS_AT + WM_RECORDS * 4 * WM_ROWS * 4;  // float [256]: the second threads' sums
  static constexpr int ODD_AT = SUM_AT + WM_KEYS * 4;                  // int [records]: a row that is not like the others
  static constexpr int INFO_AT = ODD_AT + 16;                          // int4 [FEW_SEQS], then int prefix[FEW_SEQS + 4]
  static constexpr int BAR_AT = INFO_AT + FEW_SEQS * 16 + (FEW_SEQS + 4) * 4;
  static constexpr int N_BARS = WM_FULL + WM_STAGES + 2 * WM_RECORDS + 8 + 3;
  static constexpr int SMEM = BAR_AT + N_BARS * 8 + 32;
  static_assert(SMEM + 1024 <= 232448, "shared memory of a block");
};
// Barriers: queries are there, may be overwritten; their rows' records are there, may be overwritten; a half's sums are there,
// have been read; a half's keys are there.
enum {
  W_QFULL = 0,
  W_QFREE = W_QFULL + WM_FULL,
  W_STATS = W_QFREE + WM_STAGES,
  W_RFREE = W_STATS + WM_RECORDS,
  W_DFULL = W_RFREE + WM_RECORDS,
  W_DFREE = W_DFULL + 4,
  W_A = W_DFREE + 4,
  W_DRAIN = W_A + 2
};

// Shared-memory descriptor of a K-major operand of sixteen channels without a swizzle: 8 rows of 16 bytes are 128 bytes, the next 8
// rows follow, their other 8 channels lie `next` bytes on.
__device__ __forceinline__ uint64_t sdesc_k_plain(uint32_t addr, uint32_t next) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(next >> 4) << 16;
  d |= (uint64_t)(128 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  return d;
}
// A number as three bf16 terms, each the rounding of what the ones before left.
__device__ __forceinline__ void three_terms(float x, uint32_t (&t)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    t[i] = __bfloat16_as_ushort(__float2bfloat16_rn(x));
    x -= __uint_as_float(t[i] << 16);
  }
}

// A run of one key tile's units.
struct Keys {
  int seq, head, tile;
  int user, length, first, count;
  int first_tile, n_tiles;  // of the sequence
  int row_tile, n;          // the tile's first tile of tokens and how many see it
  int from, to;             // this block's run of them
  int64_t flat;             // place of its first unit in the list
};
struct WmList {
  const int4 *info;
  const int *prefix;
  int n_seqs, heads, window;
  int tokens;  // of a unit: as many as fill its rows
};

// Which tokens, in tiles, see a key of the tile (at least one does, between a sequence's first tile and its last).
__device__ __forceinline__ void rows_of_tile(int length, int count, int tile, const WmList &l, int &row_tile, int &n) {
  const int base = length - count, k0 = tile * WM_KEYS, k1 = min(k0 + WM_KEYS, length);
  const int t0 = max(0, k0 - base), t1 = l.window > 0 ? min(count, k1 - base - 1 + l.window) : count;
  row_tile = t0 / l.tokens;
  n = (t1 + l.tokens - 1) / l.tokens - row_tile;
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

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// Sums over 16 channels, as a product with ones: of rows gid (d[0], d[1]) and gid + 8 (d[2], d[3]).
template <bool BF16>
__device__ __forceinline__ void mma_ones(float (&d)[4], const uint32_t (&a)[4]) {
  if (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %8}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(0x3F803F80u));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %8}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(0x3C003C00u));
}

template <int HD, bool BF16>
__global__ void __launch_bounds__(WM_THREADS, 1)
    kv4_weights_many_kernel(const WeightParams p, const __grid_constant__ CUtensorMap q_map, int use_map, int tokens) {
  using F = Many<HD>;
  constexpr int G = F::GROUPS, NB = F::BUFFERS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  const uint32_t base = smem_addr(smem);
  volatile int *unlike = reinterpret_cast<volatile int *>(smem + F::ODD_AT);
  int4 *info = reinterpret_cast<int4 *>(smem + F::INFO_AT);
  int *prefix = reinterpret_cast<int *>(info + FEW_SEQS);
  volatile uint32_t *words = reinterpret_cast<volatile uint32_t *>(smem + F::BAR_AT + F::N_BARS * 8);  // TMEM, abort, last
  const auto bar = [&](int b) { return base + F::BAR_AT + 8 * b; };
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int heads = p.pool.n_kv_heads, lp = p.pool.log2_tokens, group = p.group;
  const WmList list = {info, prefix, p.n_seqs, heads, p.window, tokens};
  if (tid == 0) {
    for (int i = 0; i < WM_FULL; ++i) mbar_init(bar(W_QFULL + i), 1);
    for (int i = 0; i < WM_STAGES; ++i) mbar_init(bar(W_QFREE + i), 2);
    for (int i = 0; i < WM_RECORDS; ++i) {
      mbar_init(bar(W_STATS + i), 1);
      mbar_init(bar(W_RFREE + i), WM_SUMMERS);
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
  // (rows behind a unit's tokens stay zero, and the second half of the sixteen channels)
  for (int i = tid; i < F::ROWS_AT / 16; i += WM_THREADS) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
  fence_async_proxy();
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
  const int unit_rows = tokens * group;

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
    // ---- keys: two threads each, with 64 of a unit's rows
    const int half = warp >> 2 & 1, part = warp >> 3, row = (warp & 3) * 32 + lane, key = half * 128 + row;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // TMEM lane 32 (warp mod 4), in bits 16 up
    float *second = reinterpret_cast<float *>(smem + F::SUM_AT);
    const float factor = p.scale * 1.44269504089f;
    unsigned unit = 0;
    Keys k;
    find_keys(k, list, c0, c1);
    for (;;) {
      // ---- its codes, half of them each (all products with the ones before have been waited for)
      const int slot = k.tile * WM_KEYS + key;
      bool there = false;
      float2 s[G], c[G];
      bool odd = false;  // a scale or centre that is no number, or (bf16) not to be divided by
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
        const uint32_t tile = base + F::K_AT + half * F::HALF + row * 128;
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) {  // a word's eight codes are 16 bytes of the row
          const uint32_t w = i % 4 == 0 ? raw[i / 4].x : i % 4 == 1 ? raw[i / 4].y : i % 4 == 2 ? raw[i / 4].z : raw[i / 4].w;
          const int chunk = part * (HD / 16) + i;
          uint32_t v[4];
          decode8<BF16>(w, v);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(tile + (chunk / 8) * (128 * 128) + (((chunk & 7) ^ (row & 7)) << 4)),
                       "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
                       : "memory");
        }
        float ratio[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const float a = f16_to_f32((uint16_t)par[g]), b = f16_to_f32((uint16_t)(par[g] >> 16));
          s[g] = {a * factor, a * factor}, c[g] = {b * factor, b * factor};
          ratio[g] = b / a;
          odd = odd || (par[g] & 0x7c00u) == 0x7c00u || (par[g] & 0x7c000000u) == 0x7c000000u || (BF16 && a == 0.f);
        }
        if constexpr (BF16) {
          const float inv = 1.f / s[0].x;
          // (a row without weight goes along as -2^100: its products with the terms of 1 / s_0 stay finite below 2^27, which holds
          // for every scale of a key, 2^-24 and up, under the usual softmax scales)
          odd = odd || !(fabsf(inv) < 0x1p27f);
          // (the first thread's are the channels of the first group, the second's of the second)
          if (part < G) {
            const int g = G == 2 ? part : 0;
            uint32_t r[3], n[3];
            three_terms(odd ? 0.f : ratio[g], r);
            three_terms(odd || g > 0 ? 0.f : inv, n);
            const uint32_t at = base + F::KF_AT + (half * G + g) * F::FOLD + row * 16;
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(r[0] | r[0] << 16), "r"(r[1] | r[0] << 16),
                         "r"(r[1] | r[2] << 16), "r"(n[0] | n[0] << 16)
                         : "memory");
            asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at + F::FOLD / 2), "r"(n[1] | n[0] << 16), "r"(n[1] | n[2] << 16)
                         : "memory");
          }
        }
        fence_async_proxy();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(W_A + half));
      }
      const bool any_odd = __any_sync(0xffffffffu, odd);
      const int key0 = slot - lane, before = k.length - k.count;
      float2 sum = {0.f, 0.f};
      for (int t = k.from; t < k.to; ++t, ++unit) {
        const unsigned record = unit % WM_RECORDS, buf = half * NB + unit % NB;
        const int token0 = (k.row_tile + t) * tokens;
        const int least = before + token0 + 1, most = before + min(k.count, token0 + tokens);
        wait(W_STATS + record, unit / WM_RECORDS & 1);
        wait(W_DFULL + buf, unit / NB & 1);
        __syncwarp();
        tc_fence_after();
        const bool masked = any_odd || key0 + 32 > least || (p.window > 0 && key0 < most - p.window) || unlike[record];
        const float *rows = reinterpret_cast<const float *>(smem + F::ROWS_AT) + record * 4 * WM_ROWS + part * 64;
        const uint32_t d = tmem + lanes + buf * F::D_COLS + part * 64;
        // Half the rows' sums at a time: the buffer is free for the next products while the second half is weighed.  (Two
        // forms: a branch between the rows would keep their operations apart)
        const auto weigh = [&](auto some) {
#pragma unroll
          for (int r0 = 0; r0 < 64; r0 += 32) {
            uint32_t a[G][32];
#pragma unroll
            for (int g = 0; g < G; ++g) {
              tmem_ld16(d + g * WM_ROWS + r0, reinterpret_cast<uint32_t(&)[16]>(a[g][0]));
              tmem_ld16(d + g * WM_ROWS + r0 + 16, reinterpret_cast<uint32_t(&)[16]>(a[g][16]));
            }
            tmem_wait_ld();
            if (r0 > 0) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar(W_DFREE + buf));
            }
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              float2 x0 = {0.f, 0.f}, x1 = {0.f, 0.f};
              if (!BF16 || (decltype(some)::value && odd)) {
                const float4 nl = *reinterpret_cast<const float4 *>(rows + 2 * WM_ROWS + r0 + i);
                x0 = {nl.x, nl.y}, x1 = {nl.z, nl.w};
#pragma unroll
                for (int g = 0; g < G; ++g) {
                  const float4 q = *reinterpret_cast<const float4 *>(rows + g * WM_ROWS + r0 + i);
                  x0 = fma2(c[g], {q.x, q.y}, x0), x1 = fma2(c[g], {q.z, q.w}, x1);
                }
              }
#pragma unroll
              for (int g = 0; g < G; ++g) {
                x0 = fma2(s[g], {__uint_as_float(a[g][i]), __uint_as_float(a[g][i + 1])}, x0);
                x1 = fma2(s[g], {__uint_as_float(a[g][i + 2]), __uint_as_float(a[g][i + 3])}, x1);
              }
              float2 w0 = {wm_ex2(x0.x), wm_ex2(x0.y)}, w1 = {wm_ex2(x1.x), wm_ex2(x1.y)};
              if constexpr (decltype(some)::value) {
                const int4 e = *reinterpret_cast<const int4 *>(rows + 3 * WM_ROWS + r0 + i);
                const auto sees = [&](int end) { return slot < end && (p.window == 0 || slot >= end - p.window); };
                w0 = {sees(e.x) ? w0.x : 0.f, sees(e.y) ? w0.y : 0.f};
                w1 = {sees(e.z) ? w1.x : 0.f, sees(e.w) ? w1.y : 0.f};
              }
              sum = add2(sum, add2(w0, w1));
            }
          }
        };
        if (masked)
          weigh(std::true_type());
        else
          weigh(std::false_type());
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(W_RFREE + record));
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
      if (k.flat + k.to >= c1) break;
      next_keys(k, list, c1);
    }
  } else if (c0 < c1 && warp == WM_COPY_WARP) {
    // ---- queries: a box of the group's heads by the unit's tokens, 64 channels at a time; rows off 16 bytes by hand
    unsigned unit = 0;
    bool ok = true;
    Keys k;
    find_keys(k, list, c0, c1);
    for (;;) {
      for (int t = k.from; t < k.to; ++t, ++unit) {
        const unsigned stage = unit % WM_STAGES, full = unit % WM_FULL;
        const int token0 = (k.row_tile + t) * tokens;
        if (!(ok = __all_sync(0xffffffffu, wait(W_QFREE + stage, unit / WM_STAGES & 1 ^ 1)))) break;
        const uint32_t to = base + stage * F::STAGE;
        if (use_map) {
          if (elect_one()) {
            mbar_arrive_expect_tx(bar(W_QFULL + full), unit_rows * HD * 2);
#pragma unroll
            for (int g = 0; g < G; ++g)
              tma_load_3d(to + g * (WM_ROWS * 128), &q_map, 64 * g, k.head * group, k.first + token0, bar(W_QFULL + full));
          }
          __syncwarp();
        } else {
          for (int r = 0; r < unit_rows; ++r) {
            const int token = token0 + r / group;
            uint32_t w[HD / 64] = {};
            if (token < k.count) {
              const uint16_t *e = reinterpret_cast<const uint16_t *>(p.q.row((int64_t)k.first + token, k.head * group + r % group));
#pragma unroll
              for (int j = 0; j < HD / 64; ++j) w[j] = e[64 * j + 2 * lane] | ((uint32_t)e[64 * j + 2 * lane + 1] << 16);
            }
#pragma unroll
            for (int j = 0; j < HD / 64; ++j)
              asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + j * (WM_ROWS * 128) + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4),
                           "r"(w[j])
                           : "memory");
          }
          fence_async_proxy();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(W_QFULL + full));
        }
      }
      if (!ok || k.flat + k.to >= c1) break;
      next_keys(k, list, c1);
    }
    // (no copy outlives the block, whoever has given up)
    for (unsigned u = unit > WM_STAGES ? unit - WM_STAGES : 0; u < unit; ++u) wait_2s(bar(W_QFULL + u % WM_FULL), u / WM_FULL & 1);
  } else if (c0 < c1 && warp < WM_MMA_WARP) {
    // ---- every other unit's rows: their sums over each group's channels, log-sum-exps, and the keys that they see.  A lane
    // has the rows lane, lane + 32, ...: their tokens and heads are the same in every unit
    const unsigned mine = warp - WM_STAT_WARP;
    int row_token[4], row_head[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 32 * i + lane;
      row_token[i] = r / group, row_head[i] = r % group;
    }
    unsigned unit = 0;
    Keys k;
    find_keys(k, list, c0, c1);
    for (;;) {
      for (int t = k.from; t < k.to; ++t, ++unit) {
        const unsigned stage = unit % WM_STAGES, record = unit % WM_RECORDS;
        if ((unit & 1) != mine) continue;
        const int token0 = (k.row_tile + t) * tokens;
        float lse[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int token = token0 + row_token[i];
          lse[i] = -INFINITY;
          if (32 * i + lane < unit_rows && token < k.count)
            lse[i] = p.lse[((int64_t)k.first + token) * p.n_heads + k.head * group + row_head[i]];
        }
        wait(W_RFREE + record, unit / WM_RECORDS & 1 ^ 1);
        wait(W_QFULL + unit % WM_FULL, unit / WM_FULL & 1);
        __syncwarp();
        float *rows = reinterpret_cast<float *>(smem + F::ROWS_AT) + record * 4 * WM_ROWS;
        // (every lane of four has the sums of two rows of each 16: one of them, of one group, is its own to write.  Two such
        // tiles at a time: a warp's chains of products, sums and roundings are its time)
#pragma unroll 1
        for (int m0 = 0; m0 < WM_ROWS / 16; m0 += 2) {
          uint32_t a[2][G][4][4];
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const int r = 16 * (m0 + m) + (lane & 15);  // of this lane's address: matrices of rows 0-7, 8-15, then their next 8 channels
            const uint32_t from = base + stage * F::STAGE + r * 128;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
              for (int i = 0; i < 4; ++i) ldmatrix_x4(a[m][g][i], from + g * (WM_ROWS * 128) + (((2 * i + (lane >> 4)) ^ (r & 7)) << 4));
          }
          float d[2][G][4] = {};
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
              for (int g = 0; g < G; ++g) mma_ones<BF16>(d[m][g], a[m][g][i]);
          const int g = lane & 1;
          if (g < G)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              const float low = g ? d[m][G - 1][0] : d[m][0][0], high = g ? d[m][G - 1][2] : d[m][0][2], sum = lane & 2 ? high : low;
              const int of = 16 * (m0 + m) + (lane >> 2) + 4 * (lane & 2);
              rows[g * WM_ROWS + of] = sum;
              if constexpr (BF16) {
                uint32_t s[3];
                three_terms(sum, s);
                const uint32_t to = base + F::QF_AT + (stage * G + g) * F::FOLD + of * 16;
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(s[0] | s[1] << 16), "r"(s[0] | s[2] << 16) : "memory");
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + 8), "r"(s[1] | s[0] << 16) : "memory");
              }
            }
        }
        bool other = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (a row that saw nothing adds nothing, whatever it holds; one behind the tokens is zero, or another's)
          const bool counts = lse[i] != -INFINITY;
          other = other || (!counts && 32 * i + lane < unit_rows);
          rows[2 * WM_ROWS + 32 * i + lane] = counts ? lse[i] * -1.44269504089f : -INFINITY;
          reinterpret_cast<int *>(rows)[3 * WM_ROWS + 32 * i + lane] = counts ? k.length - k.count + token0 + row_token[i] + 1 : -1;
          if constexpr (BF16) {
            // (no weight: one term, whose products with finite numbers are none that others cannot be added to)
            uint32_t n[3];
            three_terms(counts && lse[i] != INFINITY ? lse[i] * -1.44269504089f : -0x1p100f, n);
            const uint32_t to = base + F::QF_AT + stage * G * F::FOLD + (32 * i + lane) * 16;
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + 12), "r"(n[0] | n[1] << 16) : "memory");
            asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to + F::FOLD / 2), "r"(n[0] | n[2] << 16), "r"(n[1] | n[0] << 16)
                         : "memory");
          }
        }
        other = __any_sync(0xffffffffu, other);
        if (lane == 0) unlike[record] = other;
        if (BF16) fence_async_proxy();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(W_STATS + record));
          mbar_arrive(bar(W_QFREE + stage));
        }
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
        const unsigned stage = __shfl_sync(0xffffffffu, unit % WM_STAGES, 0), record = __shfl_sync(0xffffffffu, unit % WM_RECORDS, 0);
        ok = wait(W_QFULL + unit % WM_FULL, unit / WM_FULL & 1);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const unsigned buf = __shfl_sync(0xffffffffu, half * NB + unit % NB, 0);
          if (t == 0) ok = ok && wait(W_A + half, tiles & 1);
          ok = ok && wait(W_DFREE + buf, unit / NB & 1 ^ 1);
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
          tc_fence_after();
          const uint64_t q = sdesc_k_sw128(at + stage * F::STAGE), a = sdesc_k_sw128(at + F::K_AT + half * F::HALF);
          const uint64_t qf = sdesc_k_plain(at + F::QF_AT + stage * G * F::FOLD, F::FOLD / 2);
          const uint64_t af = sdesc_k_plain(at + F::KF_AT + half * G * F::FOLD, F::FOLD / 2);
          if (elect_one())
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
              for (int i = 0; i < 4; ++i)  // (descriptors count 16 bytes)
                mma_bf16_ss(tm + buf * F::D_COLS + g * WM_ROWS, a + g * (128 * 128 >> 4) + i * 2, q + g * (WM_ROWS * 128 >> 4) + i * 2,
                            idesc, i > 0);
          __syncwarp();
          if (BF16 && half == 0) {  // (the rows' sums are not needed before)
            if (!(ok = __all_sync(0xffffffffu, wait(W_STATS + record, unit / WM_RECORDS & 1)))) break;
            tc_fence_after();
          }
          if (elect_one()) {
            if (BF16)
#pragma unroll
              for (int g = 0; g < G; ++g)
                mma_bf16_ss(tm + buf * F::D_COLS + g * WM_ROWS, af + g * (F::FOLD >> 4), qf + g * (F::FOLD >> 4), idesc, 1);
            mma_commit(bar(W_DFULL + buf));
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
  const int smem = Many<HD>::SMEM + 1024, tokens = WM_ROWS / p.group;
  const cudaError_t e = opt_in(kernel, smem);
  if (e != cudaSuccess) return e;
  CUtensorMap map = {};
  const int use_map = p.q_wide && encode_heads_map(&map, p.q.data, HD, p.n_heads, p.n_tokens, p.q.head_bytes, p.q.token_bytes,
                                                   p.group, tokens) == 0;
  return launch_chained(kv4_weights_many_kernel<HD, BF16>, std::min(n_sm, FEW_BLOCKS), WM_THREADS, smem, s, p, map, use_map, tokens);
}

}  // namespace

cudaError_t launch_weights_many(const WeightParams &p, int n_sm, cudaStream_t s) {
  if (p.pool.head_dim == 128) return p.bf16 ? launch<128, true>(p, n_sm, s) : launch<128, false>(p, n_sm, s);
  return p.bf16 ? launch<64, true>(p, n_sm, s) : launch<64, false>(p, n_sm, s);
}

}  // namespace kfl
