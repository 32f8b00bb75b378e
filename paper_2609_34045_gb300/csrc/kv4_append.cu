// Rows into and out of the 4-bit paged KV cache (include/kafila_kv4.h): kfl_kv4_append, kfl_kv4_read.
//
// Memory bound in bytes (a 16-bit value read and 4.5 bits written, or the reverse), if the instructions per value stay
// below some 12: at 41 (eight channels a thread, integer divisions of 64 bits, a code's clamp and shift one by one) 16384 rows
// of 8 heads took 49 us against 13 for their bytes.  So sixteen channels of a k row and of its v row to a thread, four
// threads to a group of 64, whose ends meet in two shuffles; a code is four operations, its place in the word the last of
// them, and two more where a group's ends need a clamp.  19 us for these rows unrotated, 25 rotated in neighbouring
// pairs, 31 in halves, 18 for reading them back, all with rows that the L2 still holds; rows of four prompts that come from HBM, rotated in
// halves, 34 to 36 and 20.  The difference is the angles: 8 bytes for each pair, which the L1 looks up a
// line at a time.  Through shared memory they cost a barrier that waits for them (29 and 28 us); with the next rows' loads
// under way in a loop the registers leave half the warps (34 us).  The rotation's partner channels are read once more,
// from L1, rather than exchanged: the partner may lie in any other thread or in the same one, depending on layout and rope_dim.
#include "kv4.cuh"

namespace kfl {
namespace {

constexpr int ROW_THREADS = 256;

struct RowsParams {
  Kv4Pool pool;
  Kv4Map map;
  int layer;
  HeadsView k, v;
  const int32_t *users, *positions;
  int n_tokens;
  const float2 *cos_sin;  // NULL: no rotation
  int n_pos, rope_half, rope_layout;
  int32_t *status;
};

// Where row t goes: its place in the table (NULL: out of range, reported once per row), its slot in the page.
__device__ __forceinline__ const int32_t *place(const RowsParams &p, int user, int pos, bool reports, int &slot) {
  int bad = 0;
  if (user < 0 || user >= p.map.n_users)
    bad = KFL_BAD_USER;
  else if (pos < 0 || (pos >> p.pool.log2_tokens) >= p.map.max_pages || (p.cos_sin && pos >= p.n_pos))
    bad = KFL_BAD_POSITION;
  if (bad && reports) report(p.status, bad);
  slot = pos & (p.pool.page_tokens() - 1);
  return bad ? nullptr : p.map.table + (int64_t)user * p.map.max_pages + (pos >> p.pool.log2_tokens);
}
__device__ __forceinline__ bool page_ok(const RowsParams &p, int page, bool reports) {
  if (page >= 0 && page < p.pool.n_pages) return true;
  if (reports) report(p.status, page == -1 ? KFL_BAD_POSITION : KFL_BAD_PAGE);
  return false;
}

// Sixteen channels as they lie in memory.
constexpr int CH = 16;
template <class T>
struct alignas(16) Raw {
  T e[CH];
};
template <class T, bool WIDE>
__device__ __forceinline__ Raw<T> load_raw(const T *p) {
  Raw<T> r;
  if constexpr (WIDE) {
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < CH; i += W) move_pack<W>(r.e + i, p + i);
  } else {
#pragma unroll
    for (int i = 0; i < CH; ++i) r.e[i] = p[i];
  }
  return r;
}
template <class T>
__device__ __forceinline__ void unpack(const Raw<T> &r, float (&x)[CH]) {
#pragma unroll
  for (int i = 0; i < CH; ++i) x[i] = to_f32(r.e[i]);
}

// x, channels [c, c + 16) of a k row, rotated.
template <class T, bool WIDE>
__device__ __forceinline__ void rotate(const RowsParams &p, const T *row, int c, int pos, float (&x)[CH]) {
  const int half = p.rope_half;
  if (c >= 2 * half) return;
  const float2 *cs = p.cos_sin + (int64_t)pos * half;
  if (p.rope_layout == KFL_ROPE_INTERLEAVED) {
#pragma unroll
    for (int i = 0; i < CH; i += 2) {
      if (c + i >= 2 * half) break;  // (rope_dim is even: a pair is inside or outside as a whole)
      const float2 f = cs[(c + i) / 2];
      const float a = x[i], b = x[i + 1];
      x[i] = rope_first(a, b, f), x[i + 1] = rope_second(a, b, f);
    }
  } else if (half % CH == 0) {  // the sixteen channels have their partners in sixteen others
    float y[CH];
    const bool second = c >= half;
    unpack(load_raw<T, WIDE>(row + (second ? c - half : c + half)), y);
    const float4 *f4 = reinterpret_cast<const float4 *>(cs + (second ? c - half : c));
    const float sign = second ? 1.f : -1.f;  // x cos - y sin, or x cos + y sin
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) {
      const float4 f = f4[i];
      x[2 * i] = __fadd_rn(__fmul_rn(x[2 * i], f.x), __fmul_rn(y[2 * i], f.y * sign));
      x[2 * i + 1] = __fadd_rn(__fmul_rn(x[2 * i + 1], f.z), __fmul_rn(y[2 * i + 1], f.w * sign));
    }
  } else {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int e = c + i;
      if (e >= 2 * half) break;
      x[i] = e < half ? rope_first(x[i], to_f32(row[e + half]), cs[e])
                      : rope_second(to_f32(row[e - half]), x[i], cs[e - half]);
    }
  }
}

// Smallest and largest of three, NaN if one is.
__device__ __forceinline__ float min_nan(float a, float b, float c) {
  float r;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Two rounded sums or products in one instruction.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// Eight codes from t = (x - centre) / scale: clamp(rint(t) + 8, 0, 15).  t is clamped first (to whole numbers: the order is
// of no account), and its sum with 1.5 2^23 + 8, rounded to whole numbers, has rint(t) + 8 as its last bits.  The other
// bits of the eight sums, one on the other at 16 times the place, are a constant.
template <bool CLAMPS>
__device__ __forceinline__ uint32_t codes8(const float *x, float centre, float inv) {
  constexpr uint32_t MAGIC = 0x4B400000u;
  uint32_t w = 0;
#pragma unroll
  for (int i = 6; i >= 0; i -= 2) {
    float2 t = mul2(add2({x[i], x[i + 1]}, {-centre, -centre}), {inv, inv});
    if (CLAMPS) t = {fminf(fmaxf(t.x, -8.f), 7.f), fminf(fmaxf(t.y, -8.f), 7.f)};
    // (not add2: two-fold, the product and this sum come out as one operation, and ties go elsewhere)
    w = w * 16 + __float_as_uint(__fadd_rn(t.y, 12582920.f));
    w = w * 16 + __float_as_uint(__fadd_rn(t.x, 12582920.f));
  }
  return w - MAGIC * 0x11111111u;
}

// Codes of sixteen channels; their group is the warp's aligned four lanes, which all call.
__device__ __forceinline__ uint2 quantise(const float (&x)[CH], uint32_t &params) {
  float lo = min_nan(x[0], x[1], x[2]), hi = max_nan(x[0], x[1], x[2]);
#pragma unroll
  for (int i = 3; i < CH - 1; i += 2) lo = min_nan(lo, x[i], x[i + 1]), hi = max_nan(hi, x[i], x[i + 1]);
  lo = min_nan(lo, x[CH - 1], x[CH - 1]), hi = max_nan(hi, x[CH - 1], x[CH - 1]);
#pragma unroll
  for (int off = 2; off > 0; off >>= 1) {
    const float l = __shfl_xor_sync(0xffffffffu, lo, off), h = __shfl_xor_sync(0xffffffffu, hi, off);
    lo = min_nan(lo, l, l), hi = max_nan(hi, h, h);
  }
  if (!(hi <= KV4_LIMIT && lo >= -KV4_LIMIT)) {  // (or NaN)
    params = 0x7FFF7FFFu;
    return make_uint2(0x88888888u, 0x88888888u);
  }
  const __half scale_h = __float2half_rn(__fdiv_rn(hi - lo, 15.f));
  const float scale = __half2float(scale_h);
  const __half centre_h = __float2half_rn(__fadd_rn(lo, 8.f * scale));
  const float centre = __half2float(centre_h);
  const float inv = scale > 0.f ? __frcp_rn(scale) : 0.f;
  params = (uint32_t)__half_as_ushort(scale_h) | ((uint32_t)__half_as_ushort(centre_h) << 16);
  // the group's ends have the ends of t: where those need no clamp (a centre whose rounding to fp16 is far below a step),
  // none does
  if (__fmul_rn(__fsub_rn(lo, centre), inv) >= -8.5f && __fmul_rn(__fsub_rn(hi, centre), inv) < 7.5f)
    return make_uint2(codes8<false>(x, centre, inv), codes8<false>(x + 8, centre, inv));
  return make_uint2(codes8<true>(x, centre, inv), codes8<true>(x + 8, centre, inv));
}

// The (token, head) of a unit: below 2^31 of them (checked by the host).
struct Unit {
  int64_t t;
  int head;
};
__device__ __forceinline__ Unit unit_of(const RowsParams &p, unsigned u) {
  const unsigned t = u / (unsigned)p.pool.n_kv_heads;
  return {(int64_t)t, (int)(u - t * (unsigned)p.pool.n_kv_heads)};
}

template <class T, bool WIDE>
__global__ void __launch_bounds__(ROW_THREADS, 4) kv4_append_kernel(const RowsParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int lanes = p.pool.head_dim / CH, shift = p.pool.head_dim == 128 ? 3 : 2;  // threads of a row
  const unsigned n_units = (unsigned)p.n_tokens * (unsigned)p.pool.n_kv_heads;
  const unsigned unit = blockIdx.x * (unsigned)(ROW_THREADS >> shift) + (threadIdx.x >> shift);
  // (threads behind the last row repeat it without storing it: the shuffles take whole warps)
  const Unit u = unit_of(p, min(unit, n_units - 1));
  const int c = (threadIdx.x & (lanes - 1)) * CH;
  const int pos = p.positions[u.t], user = p.users ? p.users[u.t] : (int)u.t;
  const T *k_row = reinterpret_cast<const T *>(p.k.row(u.t, u.head));
  const Raw<T> v_raw = load_raw<T, WIDE>(reinterpret_cast<const T *>(p.v.row(u.t, u.head)) + c);
  const Raw<T> k_raw = load_raw<T, WIDE>(k_row + c);
  const bool reports = u.head == 0 && c == 0 && unit < n_units;
  int slot, page = -2;
  const int32_t *at = place(p, user, pos, reports, slot);
  if (at) page = *at;
  float x[CH];
  unpack(k_raw, x);
  if (p.cos_sin && at) rotate<T, WIDE>(p, k_row, c, pos, x);
  uint32_t kp, vp;
  const uint2 kw = quantise(x, kp);
  unpack(v_raw, x);
  const uint2 vw = quantise(x, vp);
  if (unit >= n_units || !at || !page_ok(p, page, reports)) return;
  uint8_t *block = p.pool.block(page, p.layer, u.head);
  const int to = slot * (p.pool.head_dim / 2) + c / 2;
  *reinterpret_cast<uint2 *>(block + to) = kw;
  *reinterpret_cast<uint2 *>(block + p.pool.code_bytes() + to) = vw;
  if (c % KV4_GROUP == 0) {
    uint8_t *params = block + 2 * p.pool.code_bytes() + (slot * (p.pool.head_dim / KV4_GROUP) + c / KV4_GROUP) * 4;
    *reinterpret_cast<uint32_t *>(params) = kp;
    *reinterpret_cast<uint32_t *>(params + p.pool.param_bytes()) = vp;
  }
}

template <class T, bool WIDE>
__device__ __forceinline__ void store_values(uint2 codes, uint32_t params, T *dst) {
  const __half2 par = *reinterpret_cast<const __half2 *>(&params);
  const float scale = __low2float(par), centre = __high2float(par);
  Raw<T> v;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const uint32_t w = i < 8 ? codes.x : codes.y;
    // (2^23 + code, less 2^23 + 8: exact; so is the product, of 4 by 11 bits)
    const float u = __uint_as_float((w >> (4 * (i & 7)) & 15) | 0x4B000000u) - 8388616.f;
    v.e[i] = from_f32<T>(fmaf(u, scale, centre));
  }
  if constexpr (WIDE) {
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < CH; i += W) move_pack<W>(dst + i, v.e + i);
  } else {
#pragma unroll
    for (int i = 0; i < CH; ++i) dst[i] = v.e[i];
  }
}

template <class T, bool WIDE>
__global__ void __launch_bounds__(ROW_THREADS) kv4_read_kernel(const RowsParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int lanes = p.pool.head_dim / CH, shift = p.pool.head_dim == 128 ? 3 : 2;
  const unsigned unit = blockIdx.x * (unsigned)(ROW_THREADS >> shift) + (threadIdx.x >> shift);
  if (unit >= (unsigned)p.n_tokens * (unsigned)p.pool.n_kv_heads) return;
  const Unit u = unit_of(p, unit);
  const int c = (threadIdx.x & (lanes - 1)) * CH;
  const bool reports = u.head == 0 && c == 0;
  int slot;
  const int32_t *at = place(p, p.users ? p.users[u.t] : (int)u.t, p.positions[u.t], reports, slot);
  if (!at) return;
  const int page = *at;
  if (!page_ok(p, page, reports)) return;
  const uint8_t *block = p.pool.block(page, p.layer, u.head);
  const int from = slot * (p.pool.head_dim / 2) + c / 2;
  const uint8_t *params = block + 2 * p.pool.code_bytes() + (slot * (p.pool.head_dim / KV4_GROUP) + c / KV4_GROUP) * 4;
  const uint2 kw = *reinterpret_cast<const uint2 *>(block + from);
  const uint2 vw = *reinterpret_cast<const uint2 *>(block + p.pool.code_bytes() + from);
  const uint32_t kp = *reinterpret_cast<const uint32_t *>(params);
  const uint32_t vp = *reinterpret_cast<const uint32_t *>(params + p.pool.param_bytes());
  store_values<T, WIDE>(kw, kp, reinterpret_cast<T *>(p.k.row(u.t, u.head)) + c);
  store_values<T, WIDE>(vw, vp, reinterpret_cast<T *>(p.v.row(u.t, u.head)) + c);
}

template <class T>
cudaError_t launch_rows(const RowsParams &p, bool reads, bool wide, cudaStream_t s) {
  const int rows = ROW_THREADS / (p.pool.head_dim / CH);
  const unsigned grid = (unsigned)(((int64_t)p.n_tokens * p.pool.n_kv_heads + rows - 1) / rows);
  if (reads)
    return wide ? launch_chained(kv4_read_kernel<T, true>, grid, ROW_THREADS, 0, s, p)
                : launch_chained(kv4_read_kernel<T, false>, grid, ROW_THREADS, 0, s, p);
  return wide ? launch_chained(kv4_append_kernel<T, true>, grid, ROW_THREADS, 0, s, p)
              : launch_chained(kv4_append_kernel<T, false>, grid, ROW_THREADS, 0, s, p);
}

int rows_call(const char *me, bool reads, const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer,
              const kfl_heads *k, const kfl_heads *v, const int32_t *users, const int32_t *positions, int n_tokens,
              const kfl_rope_plan *rope, int32_t *status, void *cuda_stream) {
  int rc = check_pool(pool, true, me);
  if (rc == KFL_OK) rc = check_map(map, me);
  if (rc == KFL_OK) rc = check_layer(pool, layer, me);
  if (rc != KFL_OK) return rc;
  if (!heads_valid(k, n_tokens) || !heads_valid(v, n_tokens)) return bad_arg(me, "k and v are needed");
  if (k->n_heads != pool->n_kv_heads || v->n_heads != pool->n_kv_heads || k->dtype != v->dtype)
    return bad_arg(me, "k and v have the pool's heads and one type");
  if (rope && (!rope_valid(rope) || rope->rope_dim > pool->head_dim)) return bad_arg(me, "not a rotation of these heads");
  if (n_tokens < 0 || (n_tokens > 0 && !positions)) return bad_arg(me, "positions are needed");
  if (n_tokens == 0) return KFL_OK;
  if ((int64_t)n_tokens * pool->n_kv_heads > 0x7fffffff) {
    bad_arg(me, "more than 2^31 - 1 rows in one call");
    return KFL_ERR_RANGE;
  }
  RowsParams p = {};
  p.pool = pool_of(*pool), p.map = map_of(*map), p.layer = layer;
  p.k = view_of(*k), p.v = view_of(*v);
  p.users = users, p.positions = positions, p.n_tokens = n_tokens;
  if (rope) {
    p.cos_sin = reinterpret_cast<const float2 *>(rope->cos_sin);
    p.n_pos = rope->n_pos, p.rope_half = rope->rope_dim / 2, p.rope_layout = rope->layout;
  }
  p.status = status;
  const bool wide = rows_aligned16(*k) && rows_aligned16(*v);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  switch (k->dtype) {
    case KFL_DT_BF16: e = launch_rows<__nv_bfloat16>(p, reads, wide, s); break;
    case KFL_DT_FP16: e = launch_rows<__half>(p, reads, wide, s); break;
    default: e = launch_rows<float>(p, reads, wide, s); break;
  }
  return cuda_result(e, me);
}

}  // namespace
}  // namespace kfl

extern "C" int kfl_kv4_page_bytes(const kfl_kv4_pool *pool, size_t *out) {
  const int rc = kfl::check_pool(pool, false, "kfl_kv4_page_bytes");
  if (rc != KFL_OK) return rc;
  if (!out) return kfl::bad_arg("kfl_kv4_page_bytes", "NULL pointer");
  *out = kfl::pool_of(*pool).page_bytes();
  return KFL_OK;
}

extern "C" int kfl_kv4_append(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const kfl_heads *k,
                              const kfl_heads *v, const int32_t *users, const int32_t *positions, int n_tokens,
                              const kfl_rope_plan *rope, int32_t *status, void *cuda_stream) {
  return kfl::rows_call("kfl_kv4_append", false, pool, map, layer, k, v, users, positions, n_tokens, rope, status,
                        cuda_stream);
}

extern "C" int kfl_kv4_read(const kfl_kv4_pool *pool, const kfl_kv4_map *map, int layer, const int32_t *users,
                            const int32_t *positions, int n_tokens, const kfl_heads *k_out, const kfl_heads *v_out,
                            int32_t *status, void *cuda_stream) {
  return kfl::rows_call("kfl_kv4_read", true, pool, map, layer, k_out, v_out, users, positions, n_tokens, nullptr,
                        status, cuda_stream);
}
