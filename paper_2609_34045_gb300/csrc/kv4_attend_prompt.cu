// Attention over the 4-bit paged KV cache for many query rows per KV head (prompts, long drafts), on tcgen05.
//
// Mathematics.  The query rows (token, head of the group) of a KV head are the M of two matrix products,
//   S = Q K^T (128 rows x 128 keys), O += P V,  P = 2^(c S - m),
// with fp32 accumulators in tensor memory.  K and V are decoded once per block into fp16 operands in shared memory; P takes
// the place of S as the second product's fp16 operand.  The reference m of a row is the maximum of its first tiles and moves only
// when a tile's weights sum to more than 2^14 (P stays inside fp16), so that O is rarely rescaled and the maximum not looked for.
// A row of Q is brought into fp16's range by a power of two that its scores are multiplied back by.
//
// Roundings.  A number rounded to fp16 is 2.1e-4 of it off (root mean square).  The weights are, in P.  With bf16 outputs, whose own
// rounding is 1.66e-3, so are K and V: 4.3e-4 to 5e-4 in all, which the output's hides.  With fp16 outputs (2.1e-4) it would
// double their error: there a decoded value is the sum of two fp16 numbers (decode_row) and each product is taken twice; 2.8e-4
// in all, for 1.01 to 1.55 times the time.
//
// What bounds it.  4 head_dim flops per (query head, visible key): the tensor pipe, 2048 clocks for 256 rows by 128
// keys at head_dim 128.  2048 tokens over 8192 keys, 64/8 heads of 128, bf16: 452 us, 1.06 PFLOP/s of the 1.89 that a plain bf16
// product reaches, some 4670 clocks a tile.  Of these a half's softmax (64 scores a thread, 2.5 instructions each and as much again
// around them) takes about 1900 and its own products 1024, one after the other; the rest is not accounted for (waits
// between the roles, decoding: eight turns a tile of some 350 instructions on seven warps).  fp16: 700 us.  There the second
// terms' products cost 45 us, their decoding 40, both together 170, and the shorter tiles 90.
//
// Roles.  Warps 0-7 and 8-15: softmax of the two 128-row halves, two threads per row with half of a tile's keys each, and their Q
// and output; 16-22: decoding, a thread per key, 32 keys of K or V at a time in turn, raw codes straight from global memory
// ahead of their turn; 23: products.  While one half's softmax runs, the other half's products do.  (One thread per row:
// 531 us.  Four decoding warps: decoding takes as long as the rest.)
//
// Work split.  The (sequence, KV head, 256 rows) x (128 or 64 keys) tiles in sight form one list that the blocks share
// equally; a row block cut between thread blocks is merged by the last to arrive, in list order.
#include <algorithm>

#include "kv4_attend.cuh"
#include "prefill_tc.cuh"

namespace kfl {
namespace {

constexpr int PT_PARTS = 2;                  // threads of a row
constexpr int PT_SOFTMAX = 8 * PT_PARTS;     // warps 0 to 15
constexpr int PT_DECODERS = 7;               // 16 to 22
constexpr int PT_MMA_WARP = PT_SOFTMAX + PT_DECODERS;
constexpr int PT_THREADS = (PT_MMA_WARP + 1) * 32;
constexpr float PT_MOST = 16384.f;           // a row's weights in a tile may sum up to this: none is near fp16's end

// TERMS: fp16 numbers that a decoded value is the sum of.  One, rounded, on 128 keys a tile; or two, on 64, in the same bytes: with
// Q in the tensor memory that their narrower scores leave free (read from shared memory by each of twice as many products it
// held them up: 789 us for 700).
template <int HD, int TERMS>
struct Prompt {
  static constexpr int KEYS = 128 / TERMS;                 // of a tile
  static constexpr int COLS = KEYS / PT_PARTS;             // scores of a thread
  static constexpr int QUARTERS = KEYS / 32;               // what a decoding warp takes at once is one
  static constexpr int Q_COL = KEYS;                       // two terms: of Q, behind a half's scores
  static constexpr int KB = HD / 64;                       // 64-channel blocks of 128-byte rows
  static constexpr int TILE = 128 * HD * 2;                // bytes of 128 rows of Q in fp16, and of a tile's K or V
  static constexpr int TERM = TILE / TERMS;                // from a value's first term to its second
  static constexpr int Q_AT = 0, K_AT = TERMS == 1 ? 2 * TILE : 0, V_AT = K_AT + 2 * TILE;
  static constexpr int INFO_AT = V_AT + 2 * TILE;          // int4[FEW_SEQS], then int prefix[FEW_SEQS + 4]
  static constexpr int FLAG_AT = INFO_AT + FEW_SEQS * 16 + (FEW_SEQS + 4) * 4;  // uint4 [4][1 + KB]: keys of a tile
  static constexpr int ODD_AT = FLAG_AT + 4 * (1 + KB) * 16;    // uint32 [4][2]: a byte per 32 keys, K and V: not as usual
  static constexpr int PAIR_AT = ODD_AT + 4 * 2 * 4;  // float [2 halves][2][128]: what a row's two threads exchange
  static constexpr int BAR_AT = PAIR_AT + 2 * 2 * 128 * 4;
  static constexpr int SMEM = BAR_AT + 20 * 8 + 32;
  static_assert(SMEM + 1024 <= 232448, "shared memory of a block");
};

// Barriers, in 8-byte places behind BAR_AT.
enum { B_KFULL = 0, B_KFREE = 2, B_VFULL = 4, B_VFREE = 6, B_Q = 8, B_S = 10, B_P = 12, B_O = 14, B_READ = 16, B_DRAIN = 18 };

__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory descriptor of an operand whose N (channels) lies contiguous, 128-byte swizzled: rows of 64 channels, one
// per K (key), groups of 8 rows 1024 bytes apart (the stride byte offset), the next 64 channels `next` bytes on (the
// leading byte offset).
__device__ __forceinline__ uint64_t sdesc_mn_sw128(uint32_t addr, uint32_t next) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(next >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

__device__ __forceinline__ float pt_ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t pt_pack(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// A thread's scores of a row: w the weights 2^(score cf - top) in fp16 pairs, the second product's operand (bf16 would be eight
// times the rounding); returns their sum (taken in fp32 before the rounding: above PT_MOST one of them may have outgrown
// fp16).  Sixteen at a time: a load from tensor memory takes some 50 clocks, which the other warps fill, and more of them in
// flight would cost registers that the tile loop has not got.
template <int COLS>
__device__ __forceinline__ float weigh_scores(uint32_t t_s, float cf, float top, uint32_t (&w)[COLS / 2]) {
  const float2 scale = {cf, cf}, from = {-top, -top};
  float2 s[2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
  for (int c = 0; c < COLS / 16; ++c) {
    uint32_t v[16];
    tmem_ld16(t_s + 16 * c, v);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      float2 e = fma2({__uint_as_float(v[i]), __uint_as_float(v[i + 1])}, scale, from);
      e = {pt_ex2(e.x), pt_ex2(e.y)};
      s[i >> 1 & 1] = add2(s[i >> 1 & 1], e);
      w[8 * c + i / 2] = pt_pack(e.x, e.y);
    }
  }
  return s[0].x + s[0].y + (s[1].x + s[1].y);
}

// A barrier of the two warps that share 32 rows (pair 0 to 7); with any: whether any of their threads says so.
__device__ __forceinline__ void pair_sync(int pair) { named_bar_sync(1 + pair, 64); }
__device__ __forceinline__ bool pair_any(int pair, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)x), "r"(1 + pair)
      : "memory");
  return r != 0;
}

// A run of one row block's tiles: what a thread block works on at a time.
struct Piece {
  int seq, head, block;          // block: of rows_per_block query rows
  int user, length, first, count;
  int row0, rows;                // its query rows
  int tile0, n_tiles;            // its first tile (of KEYS keys) and how many it sees (at least one)
  int from, to;                  // this thread block's run of them
  int64_t flat;                  // place of its first tile in the list
};

template <int KEYS>
struct List {
  const int4 *info;
  const int *prefix;
  int n_seqs, heads, group, window, rows_per_block;
};

template <int KEYS>
__device__ __forceinline__ void tiles_of_block(int length, int count, int block, const List<KEYS> &l, int &tile0, int &n) {
  const int rows = count * l.group;
  const int tok0 = block * l.rows_per_block / l.group;
  const int tok1 = (min(rows, (block + 1) * l.rows_per_block) - 1) / l.group;
  const int end = length - count + tok1 + 1;
  const int begin = l.window > 0 ? max(0, length - count + tok0 + 1 - l.window) : 0;
  tile0 = begin / KEYS;
  n = max(1, (max(end, 0) + KEYS - 1) / KEYS - tile0);
}

template <int KEYS>
__device__ __forceinline__ void open_piece(Piece &pc, const List<KEYS> &l, int skip, int64_t limit) {
  // the block's tiles from `skip` on, as far as the list's place `limit`
  pc.row0 = pc.block * l.rows_per_block;
  pc.rows = min(l.rows_per_block, pc.count * l.group - pc.row0);
  tiles_of_block(pc.length, pc.count, pc.block, l, pc.tile0, pc.n_tiles);
  pc.from = skip;
  pc.to = (int)min((int64_t)pc.n_tiles, limit - pc.flat);
}

template <int KEYS>
__device__ __forceinline__ void open_sequence(Piece &pc, const List<KEYS> &l) {
  const int4 v = l.info[pc.seq];
  pc.user = v.x, pc.length = v.y, pc.first = v.z, pc.count = v.w;
}

// The piece at place `at` of the list (at < limit).  The whole warp calls it: lanes count the tiles of a block each.
template <int KEYS>
__device__ void find_piece(Piece &pc, const List<KEYS> &l, int64_t at, int64_t limit) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = l.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if ((int64_t)l.prefix[mid + 1] * l.heads > at)
      hi = mid;
    else
      lo = mid + 1;
  }
  pc.seq = lo;
  open_sequence(pc, l);
  const int64_t start = (int64_t)l.prefix[lo] * l.heads;
  const int per_head = l.prefix[lo + 1] - l.prefix[lo];
  pc.head = (int)((at - start) / per_head);
  int rest = (int)(at - start - (int64_t)pc.head * per_head), before = 0;
  const int n_blocks = (pc.count * l.group + l.rows_per_block - 1) / l.rows_per_block;
  for (int b0 = 0;; b0 += 32) {
    int tile0, n = 0;
    if (b0 + lane < n_blocks) tiles_of_block(pc.length, pc.count, b0 + lane, l, tile0, n);
    int sum = n;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, sum, off);
      if (lane >= off) sum += o;
    }
    const unsigned here = __ballot_sync(0xffffffffu, before + sum > rest);
    if (here != 0 || b0 + 32 >= n_blocks) {
      const int i = here ? __ffs(here) - 1 : 31;
      pc.block = b0 + i;
      before += __shfl_sync(0xffffffffu, sum - n, i);
      break;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  pc.flat = start + (int64_t)pc.head * per_head + before;
  open_piece(pc, l, (int)(at - pc.flat), limit);
}

template <int KEYS>
__device__ void next_piece(Piece &pc, const List<KEYS> &l, int64_t limit) {  // (the list goes on to `limit`)
  pc.flat += pc.n_tiles;
  if (++pc.block * l.rows_per_block >= pc.count * l.group) {
    pc.block = 0;
    if (++pc.head == l.heads) {
      pc.head = 0;
      do {
        ++pc.seq;
        open_sequence(pc, l);
      } while (pc.count == 0);
    }
  }
  open_piece(pc, l, 0, limit);
}

__device__ __forceinline__ uint32_t neg2(uint32_t x) {
  uint32_t r;
  asm("neg.f16x2 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// Codes and parameters of one row in fp16 [channel], in the order that the words' nibbles come in (0 4 1 5 2 6 3 7 of
// every eight), as a row of the swizzled operand.  One term: v = centre + (code - 8) scale, rounded once to fp16's 11 bits, 2.1e-4 of
// it (root mean square).  With two the second is what that rounding lost, to 2^-12 of a step: with the whole number k that leaves
// r = centre + k scale at half a step, and t = code - 8 - k, it is (t scale - v) + r, whose first difference
// is about -r and keeps its bits.  Where k would not fit (a group more than 1900 steps from zero) it is 0, and the
// second term t scale + (centre - v), whose difference is exact.
template <int HD, int TERMS>
__device__ __forceinline__ void decode_row(const uint4 (&raw)[HD / 32], const uint32_t (&par)[HD / 64], uint32_t tile, int row) {
  using F = Prompt<HD, TERMS>;
#pragma unroll
  for (int g = 0; g < HD / 64; ++g) {
    const uint32_t s = __byte_perm(par[g], 0, 0x1010);
    uint32_t c = __byte_perm(par[g], 0, 0x3232), from = 0xD480D480u;  // -72
    bool far = false, any_far = false;
    if constexpr (TERMS == 2) {
      const float scale = f16_to_f32((uint16_t)par[g]), centre = f16_to_f32((uint16_t)(par[g] >> 16));
      const float steps = scale > 0.f ? __fdividef(-centre, scale) : 0.f;
      far = !(fabsf(steps) <= 1900.f);  // (or NaN.  Whole numbers up to 2048 are exact in fp16)
      const float k = far ? 0.f : rintf(steps), r = far ? centre : fmaf(k, scale, centre);
      c = pt_pack(r, r), from = pt_pack(-72.f - k, -72.f - k);
      any_far = __any_sync(0xffffffffu, far);
    }
#pragma unroll
    for (int j = g * 8; j < g * 8 + 8; ++j) {
      const uint32_t w = j % 4 == 0 ? raw[j / 4].x : j % 4 == 1 ? raw[j / 4].y : j % 4 == 2 ? raw[j / 4].z : raw[j / 4].w;
      uint32_t v[4], rest[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = i == 0 ? w << 4 : i == 1 ? w : i == 2 ? w >> 4 : w >> 8;
        asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(v[i]) : "r"(x), "r"(0x00F000F0u), "r"(0x64006400u));  // 16 (64 + u)
        const uint32_t t = hfma2(v[i], 0x2C002C00u, from);                                                  // / 16 - 72 (- k): exact
        v[i] = hfma2(t, s, c);
        if constexpr (TERMS == 2) {
          rest[i] = hfma2(hfma2(t, s, neg2(v[i])), 0x3C003C00u, c);
          if (any_far) {
            const uint32_t other = hfma2(t, s, hfma2(v[i], 0xBC00BC00u, c));
            if (far) rest[i] = other;
          }
        }
      }
      const uint32_t at = tile + g * (F::KEYS * 128) + row * 128 + (((j & 7) ^ (row & 7)) << 4);
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
      if constexpr (TERMS == 2)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + F::TERM), "r"(rest[0]), "r"(rest[1]), "r"(rest[2]),
                     "r"(rest[3])
                     : "memory");
    }
  }
}

template <int HD, int TERMS>
__global__ void __launch_bounds__(PT_THREADS, 1) kv4_attend_prompt_kernel(const AttendParams p, int rows_per_block) {
  using F = Prompt<HD, TERMS>;
  constexpr int KB = F::KB, KEYS = F::KEYS, COLS = F::COLS, QUARTERS = F::QUARTERS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
  const uint32_t base = smem_addr(smem);
  int4 *info = reinterpret_cast<int4 *>(smem + F::INFO_AT);
  int *prefix = reinterpret_cast<int *>(info + FEW_SEQS);
  uint4 *flags = reinterpret_cast<uint4 *>(smem + F::FLAG_AT);  // [4][0: page there, 1 + g: group g reads as NaN]
  volatile uint32_t *odd = reinterpret_cast<volatile uint32_t *>(smem + F::ODD_AT);
  volatile uint32_t *words = reinterpret_cast<volatile uint32_t *>(smem + F::BAR_AT + 20 * 8);  // TMEM, abort, last
  const uint32_t bars = base + F::BAR_AT;
  const auto bar = [&](int b) { return bars + 8 * b; };
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int heads = p.pool.n_kv_heads, lp = p.pool.log2_tokens;
  const List<KEYS> list = {info, prefix, p.n_seqs, heads, p.group, p.window, rows_per_block};
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(B_KFULL + i), QUARTERS);
      mbar_init(bar(B_VFULL + i), QUARTERS);
      mbar_init(bar(B_KFREE + i), 1);
      mbar_init(bar(B_VFREE + i), 1);
      mbar_init(bar(B_Q + i), 4 * PT_PARTS);
      mbar_init(bar(B_S + i), 1);
      mbar_init(bar(B_P + i), 4 * PT_PARTS);
      mbar_init(bar(B_O + i), 1);
      mbar_init(bar(B_READ + i), 4 * PT_PARTS);
    }
    mbar_init(bar(B_DRAIN), 1);
    words[1] = 0;
    prefix[0] = 0;
  }
  fence_mbar_init();
  if (warp == PT_MMA_WARP) tmem_alloc(base + F::BAR_AT + 20 * 8, 512);
  pdl_wait();

  // ---- the list: every sequence's tiles per head, summed
  for (int s = warp; s < p.n_seqs; s += PT_THREADS / 32) {
    const int user = p.users ? p.users[s] : p.seq0 + s;
    const int first = p.q_start ? p.q_start[s] : p.seq0 + s;
    int count = p.q_start ? p.q_start[s + 1] - first : 1, length = 0;
    if (first < 0 || count < 0 || count > p.max_q || first > p.n_tokens - count) {
      if (blockIdx.x == 0 && lane == 0) report(p.status, KFL_BAD_POSITION);
      count = 0;
    }
    if (user < 0 || user >= p.map.n_users) {
      if (blockIdx.x == 0 && lane == 0) report(p.status, KFL_BAD_USER);
    } else {
      length = min(max(0, p.map.lengths[user]), p.map.max_pages << lp);
    }
    int64_t tiles = 0;
    for (int b = lane; b * rows_per_block < count * p.group; b += 32) {
      int tile0, n;
      tiles_of_block(length, count, b, list, tile0, n);
      tiles += n;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) tiles += __shfl_xor_sync(0xffffffffu, tiles, off);
    if (lane == 0) info[s] = make_int4(user, length, first, count), prefix[s + 1] = (int)min(tiles, (int64_t)0x7fffffff);
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
    // (a list of that many tiles would run for half a minute: refused)
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
  const size_t slot_floats = (size_t)rows_per_block * (HD + 2);

  // a wait that gives up lets no later one last
  const auto wait = [&](int b, uint32_t parity) {
    if (mbar_try_wait(bar(b), parity)) return true;
    if (words[1]) return false;
    if (wait_2s(bar(b), parity)) return true;
    words[1] = 1;
    report(p.status, KFL_TIMED_OUT);
    return false;
  };

  if (c0 < c1 && warp < PT_SOFTMAX) {
    // ---- softmax: two threads per query row, each with half of a tile's keys and half of the row's channels.  They meet in
    // barriers of the half, so where a wait has given up they go on to the list's end (no wait lasts then), their
    // results being of no account
    const int half = warp / (4 * PT_PARTS), part = warp / 4 % PT_PARTS, row = tid & 127;
    constexpr int CH = HD / PT_PARTS;                          // channels of a thread
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // TMEM lane 32 (warp mod 4), in bits 16 up
    const uint32_t t_s = tmem + lanes + half * 128 + part * COLS;
    const uint32_t t_o = tmem + lanes + 256 + half * 128 + part * CH;
    const uint32_t q_tile = base + F::Q_AT + half * F::TILE;
    const int twins = half * 4 + (warp & 3);
    float *pair = reinterpret_cast<float *>(smem + F::PAIR_AT) + half * 256;  // [part][row]
    // A value of both threads of the row
    const auto shared_by_row = [&](float x, auto join) {
      pair[part * 128 + row] = x;
      pair_sync(twins);
      x = join(x, pair[(part ^ 1) * 128 + row]);
      pair_sync(twins);  // (before the next exchange)
      return x;
    };
    const float log2_scale = fabsf(p.scale) * 1.44269504089f;
    constexpr uint32_t ODD = QUARTERS == 4 ? 0xffffffffu : 0xffffu;  // (a byte a quarter)
    uint32_t done = 0;  // tiles of this half so far
    unsigned tile = 0;  // tiles of the thread block so far (places of the flags)
    Piece pc;
    find_piece(pc, list, c0, c1);
    for (;;) {
      const int n = pc.to - pc.from;
      if (half * 128 < pc.rows) {
        const int r = half * 128 + row;
        const bool there = r < pc.rows;
        const int token = (pc.row0 + (there ? r : 0)) / p.group, head = pc.head * p.group + (pc.row0 + (there ? r : 0)) % p.group;
        const int end = there ? pc.length - pc.count + token + 1 : pc.length;  // keys below it are seen
        const int begin = p.window > 0 ? end - p.window : 0;
        // its query, in fp16 and the words' channel order
        float unit, inv;
        {
          const uint16_t *src = reinterpret_cast<const uint16_t *>(p.q.row(pc.first + token, head)) + part * CH;
          uint32_t w[CH / 2];
#pragma unroll
          for (int i = 0; i < CH / 8; ++i) {
            if (!there) {
              w[4 * i] = w[4 * i + 1] = w[4 * i + 2] = w[4 * i + 3] = 0;
            } else if (p.q_wide) {
              const uint4 v = *reinterpret_cast<const uint4 *>(src + 8 * i);
              w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j) w[4 * i + j] = src[8 * i + 2 * j] | ((uint32_t)src[8 * i + 2 * j + 1] << 16);
            }
          }
          const float sign = p.scale > 0.f ? 1.f : p.scale < 0.f ? -1.f : 0.f;
          float big = 0.f;
#pragma unroll
          for (int i = 0; i < CH / 2; ++i) {
            const float a = p.bf16 ? bf16_lo(w[i]) : f16_to_f32((uint16_t)w[i]);
            const float b = p.bf16 ? bf16_hi(w[i]) : f16_to_f32((uint16_t)(w[i] >> 16));
            big = fmaxf(big, fmaxf(fabsf(a), fabsf(b)));
          }
          unit = xchunk_scale(shared_by_row(big, [](float a, float b) { return fmaxf(a, b); }), &inv);
#pragma unroll
          for (int i = 0; i < CH / 8; ++i) {
            float f[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t v = w[4 * i + j];
              f[2 * j] = (p.bf16 ? bf16_lo(v) : f16_to_f32((uint16_t)v)) * inv * sign;
              f[2 * j + 1] = (p.bf16 ? bf16_hi(v) : f16_to_f32((uint16_t)(v >> 16))) * inv * sign;
            }
            if (p.scale == 0.f)
#pragma unroll
              for (int j = 0; j < 8; ++j) f[j] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * i + j] = pt_pack(f[j], f[j + 4]);
            if constexpr (TERMS == 1) {
              const int chunk = part * (CH / 8) + i;
              const uint32_t at = q_tile + (chunk / 8) * (128 * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[4 * i]), "r"(w[4 * i + 1]),
                           "r"(w[4 * i + 2]), "r"(w[4 * i + 3])
                           : "memory");
            }
          }
          if constexpr (TERMS == 2) {
#pragma unroll
            for (int c = 0; c < CH / 32; ++c)
              tmem_st16(tmem + lanes + half * 128 + F::Q_COL + part * (CH / 2) + 16 * c, reinterpret_cast<uint32_t(&)[16]>(w[16 * c]));
            tmem_wait_st();
            tc_fence_before();
          }
        }
        if (TERMS == 1) fence_async_proxy();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_Q + half));
        const float cf = p.scale == 0.f ? 1.f : fmaxf(unit * log2_scale, 1e-37f);
        float top = -INFINITY, sum = 0.f;  // top: the reference, in scores times cf; sum: of this thread's weights
        unsigned poison = 0;               // groups of which this row sees a NaN
        const auto see_poison = [&](int t) {
          const int key0 = (pc.tile0 + pc.from + t) * KEYS;
#pragma unroll 1
          for (int g = 0; g < KB; ++g) {
            const uint4 v = flags[((tile + t) & 3) * (1 + KB) + 1 + g];
#pragma unroll 1
            for (int k = 0; k < KEYS; ++k) {
              const uint32_t bits = k < 32 ? v.x : k < 64 ? v.y : k < 96 ? v.z : v.w;
              if ((bits >> (k & 31) & 1) && key0 + k < end && key0 + k >= begin) poison |= 1u << g;
            }
          }
        };
        // rows of this warp: the least end and the greatest begin decide whether a tile is seen whole
        const int least = __reduce_min_sync(0xffffffffu, end);
        const int greatest = __reduce_max_sync(0xffffffffu, begin);
        for (int t = 0; t < n; ++t) {
          const int key0 = (pc.tile0 + pc.from + t) * KEYS + part * COLS;  // of this thread's keys
          wait(B_S + half, done & 1);
          __syncwarp();
          tc_fence_after();
          const bool masked = key0 + COLS > least || (p.window > 0 && key0 < greatest);
          // (what the decoding has to say of the tiles comes while the scores are weighed: shared memory, busy with the
          // products' operands, takes hundreds of clocks)
          const uint32_t odd_k = odd[2 * ((tile + t) & 3)] & ODD, odd_v = t > 0 ? odd[2 * ((tile + t - 1) & 3) + 1] & ODD : 0;
          // The weights are taken against the reference that the row has; they stay in registers until both threads of the
          // row find that it holds.  Where it does not (the first tile, a row that outgrew it, scores that
          // are masked) the scores, still in place, are read again.
          uint32_t w[COLS / 2];
          float part_sum = 0.f;
          if (!masked && t > 0) part_sum = weigh_scores<COLS>(t_s, cf, top, w);
          if (odd_v) see_poison(t - 1);
          if (pair_any(twins, masked || odd_k || t == 0 || part_sum > PT_MOST || top == -INFINITY)) {
            const bool pick = masked || odd_k;
            const uint4 there4 = flags[((tile + t) & 3) * (1 + KB)];
            const auto sees = [&](int c, int i) {  // column 16 c + i
              const int key = key0 + 16 * c + i;
              const int k = part * COLS + 16 * c;
              const uint32_t pages = k < 32 ? there4.x : k < 64 ? there4.y : k < 96 ? there4.z : there4.w;
              return key < end && key >= begin && (pages >> ((c & 1) * 16 + i) & 1);
            };
            float most = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < COLS / 16; ++c) {
              uint32_t x[16];
              tmem_ld16(t_s + 16 * c, x);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (!pick || sees(c, i)) most = fmaxf(most, __uint_as_float(x[i]));
            }
            most = shared_by_row(most, [](float a, float b) { return fmaxf(a, b); });
            most = most == -INFINITY ? most : most * cf;
            float keep = 1.f;
            if (most > top) {
              keep = pt_ex2(top - most);
              top = most;
              sum *= keep;
            }
            if (t > 0 && __any_sync(0xffffffffu, keep != 1.f)) {
              wait(B_O + half, (done - 1) & 1);  // the last tile's product
              __syncwarp();
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < CH / 16; ++c) {
                uint32_t o[16];
                tmem_ld16(t_o + 16 * c, o);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * keep);
                tmem_st16(t_o + 16 * c, o);
              }
              tmem_wait_st();
            }
            const float ref = top == -INFINITY ? 0.f : top;
            part_sum = 0.f;
#pragma unroll
            for (int c = 0; c < COLS / 16; ++c) {
              uint32_t x[16];
              tmem_ld16(t_s + 16 * c, x);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; i += 2) {
                float a = fmaf(__uint_as_float(x[i]), cf, -ref), b = fmaf(__uint_as_float(x[i + 1]), cf, -ref);
                if (pick) {
                  if (!sees(c, i)) a = -INFINITY;
                  if (!sees(c, i + 1)) b = -INFINITY;
                }
                a = pt_ex2(a), b = pt_ex2(b);
                part_sum += a + b;
                w[8 * c + i / 2] = pt_pack(a, b);
              }
            }
          }
          sum += part_sum;
#pragma unroll
          for (int c = 0; c < COLS / 32; ++c) tmem_st16(t_s + 16 * c, reinterpret_cast<uint32_t(&)[16]>(w[16 * c]));
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_P + half));
          ++done;
        }
        // ---- the piece's end: O, divided and stored, or handed on
        wait(B_O + half, (done - 1) & 1);
        __syncwarp();
        tc_fence_after();
        if (odd[2 * ((tile + n - 1) & 3) + 1] & ODD) see_poison(n - 1);
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_READ + half));  // (the tiles' flags have been read)
        sum = shared_by_row(sum, [](float a, float b) { return a + b; });
        const bool whole = pc.from == 0 && pc.to == pc.n_tiles;
        const float inv_sum = sum == 0.f ? 0.f : 1.f / sum;
        float *slot = p.partials + ((size_t)blockIdx.x * 2 + (pc.from > 0 ? 0 : 1)) * slot_floats;
        float *to = slot + (size_t)r * HD + part * CH;
        uint16_t *out = reinterpret_cast<uint16_t *>(p.out.row(pc.first + token, head)) + part * CH;
#pragma unroll 1
        for (int c = 0; c < CH / 16; ++c) {
          uint32_t x[16];
          tmem_ld16(t_o + 16 * c, x);
          tmem_wait_ld();
          if (!there) continue;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float v[8];  // (back in the channels' own order)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              v[j] = __uint_as_float(x[8 * i + 2 * (j & 3) + (j >> 2)]);
              if (poison >> ((part * CH + 16 * c) / 64) & 1) v[j] = __uint_as_float(0x7fc00000u);
            }
            if (whole) {
              uint16_t h[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const float y = sum == 0.f ? 0.f : v[j] * inv_sum;
                h[j] = p.bf16 ? f32_to_bf16_rne(y) : f32_to_f16_rn(y);
              }
              if (p.out_wide) {
                *reinterpret_cast<uint4 *>(out + 16 * c + 8 * i) =
                    make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16,
                               h[6] | (uint32_t)h[7] << 16);
              } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) out[16 * c + 8 * i + j] = h[j];
              }
            } else {
              *reinterpret_cast<float4 *>(to + 16 * c + 8 * i) = make_float4(v[0], v[1], v[2], v[3]);
              *reinterpret_cast<float4 *>(to + 16 * c + 8 * i + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
          }
        }
        if (there && part == 0) {
          if (!whole)
            *reinterpret_cast<float2 *>(slot + (size_t)rows_per_block * HD + 2 * r) = make_float2(top, sum);
          else if (p.lse)
            p.lse[(int64_t)(pc.first + token) * p.n_heads + head] = sum == 0.f ? -INFINITY : 0.69314718056f * top + logf(sum);
        }
        tc_fence_before();
      }
      tile += n;
      if (pc.flat + pc.to >= c1) break;
      next_piece(pc, list, c1);
    }
  } else if (c0 < c1 && warp < PT_MMA_WARP) {
    // ---- decoding: a warp takes 32 keys of a tile's K or V, the warps in turn.  Its next keys' rows are loaded while
    // it decodes these, their page numbers one turn earlier still
    constexpr unsigned TURNS = 2 * QUARTERS;              // of a tile: (K or V, quarter)
    const unsigned n = (unsigned)(c1 - c0) * TURNS;
    Piece pc;
    find_piece(pc, list, c0, c1);
    int t_next = pc.from;
    unsigned tile_next = 0;
    int page = -2, slot = 0, head = 0;  // of the row of this warp's next turn (a page of -2: behind the user's rows)
    const auto find_page = [&](unsigned turn) {
      for (; tile_next < turn / TURNS; ++tile_next)
        if (++t_next == pc.to) {
          next_piece(pc, list, c1);
          t_next = pc.from;
        }
      const int key = (pc.tile0 + t_next) * KEYS + (turn % QUARTERS) * 32 + lane;
      page = key < pc.length ? p.map.table[(int64_t)pc.user * p.map.max_pages + (key >> lp)] : -2;
      slot = key & (p.pool.page_tokens() - 1), head = pc.head;
    };
    uint4 now[HD / 32], later[HD / 32];
    uint32_t now_p[KB], later_p[KB];
    const auto load_row = [&](int which, bool there) {
      if (!there) {
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) later[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < KB; ++i) later_p[i] = 0;
        return;
      }
      const uint8_t *b = p.pool.block(page, p.layer, head);
      const uint4 *codes = reinterpret_cast<const uint4 *>(b + which * p.pool.code_bytes() + slot * (HD / 2));
      const uint8_t *at = b + 2 * p.pool.code_bytes() + which * p.pool.param_bytes() + slot * (KB * 4);
      const uint32_t *params = reinterpret_cast<const uint32_t *>(at);
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) later[i] = codes[i];
#pragma unroll
      for (int i = 0; i < KB; ++i) later_p[i] = params[i];
    };
    unsigned turn = warp - PT_SOFTMAX;
    bool there = false;
    const auto load_turn = [&](unsigned t) {  // its page is known
      there = page >= 0 && page < p.pool.n_pages;
      if (page != -2 && !there) report(p.status, KFL_BAD_PAGE);
      load_row(t / QUARTERS & 1, there);
    };
    if (turn < n) {
      find_page(turn);
      load_turn(turn);
      if (turn + PT_DECODERS < n) find_page(turn + PT_DECODERS);
    }
#pragma unroll 1
    for (; turn < n; turn += PT_DECODERS) {
      const unsigned tile = turn / TURNS;
      const int which = turn / QUARTERS & 1, buf = tile & 1, quarter = turn % QUARTERS;
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) now[j] = later[j];
#pragma unroll
      for (int j = 0; j < KB; ++j) now_p[j] = later_p[j];
      uint32_t *flag = reinterpret_cast<uint32_t *>(flags + (tile & 3) * (1 + KB)) + quarter;
      const unsigned have = __ballot_sync(0xffffffffu, there);
      if (turn + PT_DECODERS < n) {
        load_turn(turn + PT_DECODERS);
        if (turn + 2 * PT_DECODERS < n) find_page(turn + 2 * PT_DECODERS);
      }
      if (!__all_sync(0xffffffffu, wait((which ? B_VFREE : B_KFREE) + buf, (tile >> 1 & 1) ^ 1))) break;
      unsigned any = which ? 0 : ~have;
      if (which) {
#pragma unroll
        for (int g = 0; g < KB; ++g) {  // (a NaN or an infinity in scale or centre: all exponent bits set)
          const bool nan = (now_p[g] & 0x7c00u) == 0x7c00u || (now_p[g] & 0x7c000000u) == 0x7c000000u;
          const unsigned bad = __ballot_sync(0xffffffffu, nan);
          if (lane == 0) flag[4 * (1 + g)] = bad;
          any |= bad;
          if (nan) now_p[g] = 0;
        }
      } else if (lane == 0) {
        flag[0] = have;
      }
      if (lane == 0) reinterpret_cast<volatile uint8_t *>(odd + 2 * (tile & 3) + which)[quarter] = any != 0;
      decode_row<HD, TERMS>(now, now_p, base + (which ? F::V_AT : F::K_AT) + buf * F::TILE, quarter * 32 + lane);
      fence_async_proxy();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar((which ? B_VFULL : B_KFULL) + buf));
    }
  } else if (c0 < c1) {
    // ---- products, issued by an elected lane.  Descriptors are the same in every lane and known to be: through
    // shuffles, or the compiler moves them lane by lane, which takes longer than a product
    constexpr uint32_t idesc_s = idesc_kind_f16(128, KEYS, false);
    constexpr uint32_t idesc_o = idesc_kind_f16(128, HD, false) | (1u << 16);  // B is N-major
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), at = __shfl_sync(0xffffffffu, base, 0);
    unsigned tile = 0, done[2] = {}, pieces[2] = {};
    int before = 0;
    bool ok = true;
    Piece pc;
    find_piece(pc, list, c0, c1);
    const auto scores = [&](int half, int buf) {
      const uint64_t q = sdesc_k_sw128(at + F::Q_AT + half * F::TILE), k = sdesc_k_sw128(at + F::K_AT + buf * F::TILE);
      if (elect_one()) {
#pragma unroll
        for (int term = 0; term < TERMS; ++term)
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) {  // (descriptors count 16 bytes)
            const int at_q = (i / 4) * (128 * 128 >> 4) + (i % 4) * 2, at_k = (i / 4) * (KEYS * 128 >> 4) + (i % 4) * 2;
            if (TERMS == 1)
              mma_bf16_ss(tm + half * 128, q + at_q, k + at_k, idesc_s, i > 0);
            else
              mma_ts(tm + half * 128, tm + half * 128 + F::Q_COL + i * 8, k + (term * F::TERM >> 4) + at_k, idesc_s, term > 0 || i > 0);
          }
        mma_commit(bar(B_S + half));
      }
      __syncwarp();
    };
    const auto values = [&](int half, int buf, bool first) {
      const uint64_t v = sdesc_mn_sw128(at + F::V_AT + buf * F::TILE, KB == 2 ? KEYS * 128 : 1024);
      if (elect_one()) {
#pragma unroll
        for (int term = 0; term < TERMS; ++term)
#pragma unroll
          for (int i = 0; i < KEYS / 16; ++i)
            mma_ts(tm + 256 + half * 128, tm + half * 128 + i / (COLS / 16) * COLS + i % (COLS / 16) * 8,
                   v + (term * F::TERM >> 4) + i * 128, idesc_o, !first || term > 0 || i > 0);
        mma_commit(bar(B_O + half));
      }
      __syncwarp();
    };
    for (;;) {
      const int halves = __shfl_sync(0xffffffffu, pc.rows > 128 ? 2 : 1, 0), n = __shfl_sync(0xffffffffu, pc.to - pc.from, 0);
      // the halves that worked on the last piece have read its flags (decoding runs ahead), and the ones that work
      // on this one have their queries in place
      for (int h = 0; h < before; ++h) ok = ok && wait(B_READ + h, (pieces[h] - 1) & 1);
      for (int h = 0; h < halves; ++h) ok = ok && wait(B_Q + h, pieces[h]++ & 1);
      before = halves;
      ok = ok && wait(B_KFULL + (tile & 1), tile >> 1 & 1);
      if (!(ok = __all_sync(0xffffffffu, ok))) break;
      tc_fence_after();
      const int buf0 = __shfl_sync(0xffffffffu, (int)(tile & 1), 0);
      for (int h = 0; h < halves; ++h) scores(h, buf0);
      if (elect_one()) mma_commit(bar(B_KFREE + buf0));
      __syncwarp();
      for (int t = 0; t < n; ++t, ++tile) {
        const int buf = __shfl_sync(0xffffffffu, (int)(tile & 1), 0);
        const bool more = t + 1 < n;
        ok = wait(B_VFULL + buf, tile >> 1 & 1) && (!more || wait(B_KFULL + (buf ^ 1), (tile + 1) >> 1 & 1));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (h >= halves) break;
          ok = ok && wait(B_P + h, done[h]++ & 1);
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
          tc_fence_after();
          values(h, buf, t == 0);
          if (more) scores(h, buf ^ 1);
        }
        if (!ok) break;
        if (elect_one()) {
          mma_commit(bar(B_VFREE + buf));
          if (more) mma_commit(bar(B_KFREE + (buf ^ 1)));
        }
        __syncwarp();
      }
      if (!ok || pc.flat + pc.to >= c1) break;
      next_piece(pc, list, c1);
    }
    // every product has to be done before the tensor memory goes
    if (elect_one()) mma_commit(bar(B_DRAIN));
    __syncwarp();
    wait_2s(bar(B_DRAIN), 0);
  }
  tc_fence_before();
  __threadfence();
  __syncthreads();
  tc_fence_after();
  if (warp == PT_MMA_WARP) tmem_dealloc(tmem, 512);
  if (c0 >= c1 || words[1]) return;

  // ---- row blocks that other thread blocks have parts of: this one's first, its last
  for (int i = 0; i < 2; ++i) {
    Piece pc;
    find_piece(pc, list, i == 0 ? c0 : c1 - 1, c1);
    const int64_t sa = pc.flat, sb = sa + pc.n_tiles;
    if (!(i == 0 ? sa < c0 : sb > c1 && sa >= c0)) continue;
    const int from = (int)(sa / quota), to = (int)((sb - 1) / quota);
    __syncthreads();
    if (tid == 0) {
      unsigned *ticket = p.tickets + from;  // (a row block that is cut begins in one thread block, as its last one)
      const unsigned before = atom_add_acq_rel(ticket, 1u);
      words[2] = before == (unsigned)(to - from);
      if (words[2]) atomicExch(ticket, 0u);
    }
    __syncthreads();
    if (!words[2]) continue;
    // (the thread block where the row block begins has it as its last part, the others as their first)
    const float *first = p.partials + ((size_t)from * 2 + 1) * slot_floats;
    const auto slot_of = [&](int i) { return first + (i == 0 ? 0 : (size_t)(2 * i - 1) * slot_floats); };
    // sixteen lanes per row: a part's maximum and sum to a lane, then every lane its channels of all parts, four parts'
    // loads together
    constexpr int C = HD / 16;
    const int sub = lane & 15, n = to - from + 1;
    for (int r0 = warp * 2; r0 < pc.rows; r0 += PT_THREADS / 16) {
      const int r = min(r0 + (lane >> 4), pc.rows - 1);
      const size_t stats = (size_t)rows_per_block * HD + 2 * r;
      float top = -INFINITY;
      for (int i = sub; i < n; i += 16) top = fmaxf(top, slot_of(i)[stats]);
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f, v[C] = {};
      for (int i0 = 0; i0 < n; i0 += 16) {
        float w = 0.f;
        if (i0 + sub < n) {
          const float2 ms = *reinterpret_cast<const float2 *>(slot_of(i0 + sub) + stats);
          w = pt_ex2(ms.x - ref);
          sum = fmaf(ms.y, w, sum);
        }
        for (int i = 0; i < min(16, n - i0); i += 4) {
          float4 x[4][C / 4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < C / 4; ++j)
              x[k][j] = reinterpret_cast<const float4 *>(slot_of(min(i0 + i + k, n - 1)) + (size_t)r * HD + sub * C)[j];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float wk = __shfl_sync(0xffffffffu, w, (lane & 16) + i + k);
            if (i0 + i + k >= n) break;
#pragma unroll
            for (int j = 0; j < C / 4; ++j) {
              v[4 * j] = fmaf(x[k][j].x, wk, v[4 * j]), v[4 * j + 1] = fmaf(x[k][j].y, wk, v[4 * j + 1]);
              v[4 * j + 2] = fmaf(x[k][j].z, wk, v[4 * j + 2]), v[4 * j + 3] = fmaf(x[k][j].w, wk, v[4 * j + 3]);
            }
          }
        }
      }
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      if (r0 + (lane >> 4) >= pc.rows) continue;
      const int token = (pc.row0 + r) / p.group, head = pc.head * p.group + (pc.row0 + r) % p.group;
      uint16_t *out = reinterpret_cast<uint16_t *>(p.out.row(pc.first + token, head)) + sub * C;
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const float y = sum == 0.f ? 0.f : v[j] / sum;
        out[j] = p.bf16 ? f32_to_bf16_rne(y) : f32_to_f16_rn(y);
      }
      if (p.lse && sub == 0)
        p.lse[(int64_t)(pc.first + token) * p.n_heads + head] = sum == 0.f ? -INFINITY : 0.69314718056f * top + logf(sum);
    }
  }
}

template <int HD, int TERMS>
cudaError_t launch(const AttendParams &p, int n_sm, cudaStream_t s) {
  static SmemOptIn opt_in;
  const void *kernel = reinterpret_cast<const void *>(&kv4_attend_prompt_kernel<HD, TERMS>);
  const int smem = Prompt<HD, TERMS>::SMEM + 1024;
  const cudaError_t e = opt_in(kernel, smem);
  if (e != cudaSuccess) return e;
  return launch_chained(kv4_attend_prompt_kernel<HD, TERMS>, std::min(n_sm, FEW_BLOCKS), PT_THREADS, smem, s, p,
                        prompt_rows(p.max_q * p.group));
}

}  // namespace

size_t attend_prompt_partials(int head_dim, int64_t rows) {
  return (size_t)FEW_BLOCKS * 2 * prompt_rows(rows) * (head_dim + 2) * sizeof(float);
}

cudaError_t launch_attend_prompt(const AttendParams &p, int n_sm, cudaStream_t s) {
  // (two terms for fp16 outputs, whose own rounding is no larger than that of a decoded value; bf16's is eight times it)
  if (p.pool.head_dim == 128) return p.bf16 ? launch<128, 1>(p, n_sm, s) : launch<128, 2>(p, n_sm, s);
  return p.bf16 ? launch<64, 1>(p, n_sm, s) : launch<64, 2>(p, n_sm, s);
}

}  // namespace kfl
