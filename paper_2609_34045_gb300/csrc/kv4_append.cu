// Rows into and out of the 4-bit paged KV cache (include/kafila_kv4.h): kfl_kv4_append, kfl_kv4_read.
//
// Memory bound: a 16-bit value read and 4.5 bits written (or the reverse), some 10 flops.  Eight channels of one
// row to a thread (one 16-byte load, one 4-byte word of codes), eight threads to a group of 64, whose ends
// meet in three shuffles; a thread has its k and its v in flight together.  The rotation's partner channels
// are read once more, from L1, rather than exchanged: the partner may lie in any other thread or
// in the same one, depending on layout and rope_dim.
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

// Eight channels as they lie in memory.
template <class T>
struct alignas(16) Raw8 {
  T e[8];
};
template <class T, bool WIDE>
__device__ __forceinline__ Raw8<T> load_raw(const T *p) {
  Raw8<T> r;
  if constexpr (WIDE) {
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8; i += W) *reinterpret_cast<Pack<T, W> *>(r.e + i) = *reinterpret_cast<const Pack<T, W> *>(p + i);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.e[i] = p[i];
  }
  return r;
}
template <class T>
__device__ __forceinline__ void unpack8(const Raw8<T> &r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = to_f32(r.e[i]);
}

// x, channels [c, c + 8) of a k row, rotated.
template <class T, bool WIDE>
__device__ __forceinline__ void rotate8(const RowsParams &p, const T *row, int c, int pos, float (&x)[8]) {
  const int half = p.rope_half;
  if (c >= 2 * half) return;
  const float2 *cs = p.cos_sin + (int64_t)pos * half;
  if (p.rope_layout == KFL_ROPE_INTERLEAVED) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      if (c + i >= 2 * half) break;  // (rope_dim is even: a pair is inside or outside as a whole)
      const float2 f = cs[(c + i) / 2];
      const float a = x[i], b = x[i + 1];
      x[i] = rope_first(a, b, f), x[i + 1] = rope_second(a, b, f);
    }
  } else if (half % 8 == 0) {  // the eight channels have their partners in eight others
    float y[8];
    const bool second = c >= half;
    unpack8(load_raw<T, WIDE>(row + (second ? c - half : c + half)), y);
    const float4 *f4 = reinterpret_cast<const float4 *>(cs + (second ? c - half : c));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 f = f4[i];
      const float2 f0 = {f.x, f.y}, f1 = {f.z, f.w};
      x[2 * i] = second ? rope_second(y[2 * i], x[2 * i], f0) : rope_first(x[2 * i], y[2 * i], f0);
      x[2 * i + 1] = second ? rope_second(y[2 * i + 1], x[2 * i + 1], f1) : rope_first(x[2 * i + 1], y[2 * i + 1], f1);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = c + i;
      if (e >= 2 * half) break;
      x[i] = e < half ? rope_first(x[i], to_f32(row[e + half]), cs[e])
                      : rope_second(to_f32(row[e - half]), x[i], cs[e - half]);
    }
  }
}

// Codes of eight channels; their group is the warp's aligned eight lanes, which all call.
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], int lane, uint32_t &params) {
  float lo = x[0], hi = x[0];
  bool ok = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, x[i]), hi = fmaxf(hi, x[i]);
    ok = ok && fabsf(x[i]) <= KV4_LIMIT;  // (false for NaN, which fminf and fmaxf pass over)
  }
#pragma unroll
  for (int off = 4; off > 0; off >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, off));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, off));
  }
  ok = ((__ballot_sync(0xffffffffu, ok) >> (lane & 24)) & 0xff) == 0xff;
  if (!ok) {
    params = 0x7FFF7FFFu;
    return 0x88888888u;
  }
  const __half scale_h = __float2half_rn(__fdiv_rn(hi - lo, 15.f));
  const float scale = __half2float(scale_h);
  const __half centre_h = __float2half_rn(__fadd_rn(lo, 8.f * scale));
  const float centre = __half2float(centre_h);
  const float inv = scale > 0.f ? __fdiv_rn(1.f, scale) : 0.f;
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int u = __float2int_rn(__fmul_rn(__fsub_rn(x[i], centre), inv)) + 8;
    w |= (uint32_t)min(15, max(0, u)) << (4 * i);
  }
  params = (uint32_t)__half_as_ushort(scale_h) | ((uint32_t)__half_as_ushort(centre_h) << 16);
  return w;
}

// U rows a thread, in flight together.
template <class T, bool WIDE, int U>
__global__ void __launch_bounds__(ROW_THREADS) kv4_append_kernel(const RowsParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int lanes = p.pool.head_dim / 8, rows = ROW_THREADS / lanes;  // threads of a row, rows of a block at a time
  const int64_t n_units = (int64_t)p.n_tokens * p.pool.n_kv_heads;
  const int c = threadIdx.x % lanes * 8;
  Raw8<T> k_raw[U], v_raw[U];
  int pos[U], user[U], head[U];
  bool mine[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int64_t unit = ((int64_t)blockIdx.x * U + j) * rows + threadIdx.x / lanes;
    // (threads behind the last row repeat it without storing it: the shuffles take whole warps)
    mine[j] = unit < n_units;
    const int64_t u = min(unit, n_units - 1), t = u / p.pool.n_kv_heads;
    head[j] = (int)(u - t * p.pool.n_kv_heads);
    pos[j] = p.positions[t];
    user[j] = p.users ? p.users[t] : (int)t;
    v_raw[j] = load_raw<T, WIDE>(reinterpret_cast<const T *>(p.v.row(t, head[j])) + c);
    k_raw[j] = load_raw<T, WIDE>(reinterpret_cast<const T *>(p.k.row(t, head[j])) + c);
  }
  int slot[U], page[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const bool reports = head[j] == 0 && c == 0 && mine[j];
    const int32_t *at = place(p, user[j], pos[j], reports, slot[j]);
    page[j] = at ? *at : -2;
    if (at && !page_ok(p, page[j], reports)) page[j] = -2;
    mine[j] = mine[j] && page[j] >= 0;
  }
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int64_t unit = min(((int64_t)blockIdx.x * U + j) * rows + threadIdx.x / lanes, n_units - 1);
    const T *row = reinterpret_cast<const T *>(p.k.row(unit / p.pool.n_kv_heads, head[j]));
    float x[8];
    unpack8(k_raw[j], x);
    if (p.cos_sin && mine[j]) rotate8<T, WIDE>(p, row, c, pos[j], x);
    uint32_t kp, vp;
    const uint32_t kw = quantise8(x, threadIdx.x & 31, kp);
    unpack8(v_raw[j], x);
    const uint32_t vw = quantise8(x, threadIdx.x & 31, vp);
    if (!mine[j]) continue;
    uint8_t *block = p.pool.block(page[j], p.layer, head[j]);
    const int at = slot[j] * (p.pool.head_dim / 2) + c / 2;
    *reinterpret_cast<uint32_t *>(block + at) = kw;
    *reinterpret_cast<uint32_t *>(block + p.pool.code_bytes() + at) = vw;
    if (c % KV4_GROUP == 0) {
      uint8_t *params = block + 2 * p.pool.code_bytes() + (slot[j] * (p.pool.head_dim / KV4_GROUP) + c / KV4_GROUP) * 4;
      *reinterpret_cast<uint32_t *>(params) = kp;
      *reinterpret_cast<uint32_t *>(params + p.pool.param_bytes()) = vp;
    }
  }
}

template <class T, bool WIDE>
__device__ __forceinline__ void store_values(uint32_t w, uint32_t params, T *dst) {
  const float scale = __half2float(__ushort_as_half((uint16_t)params));
  const float centre = __half2float(__ushort_as_half((uint16_t)(params >> 16)));
  T v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)  // (the product is exact: 4 by 11 bits)
    v[i] = from_f32<T>(fmaf((float)((int)((w >> (4 * i)) & 15) - 8), scale, centre));
  if constexpr (WIDE) {
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8; i += W) {
      Pack<T, W> o;
#pragma unroll
      for (int j = 0; j < W; ++j) o.e[j] = v[i + j];
      *reinterpret_cast<Pack<T, W> *>(dst + i) = o;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[i] = v[i];
  }
}

template <class T, bool WIDE, int U>
__global__ void __launch_bounds__(ROW_THREADS) kv4_read_kernel(const RowsParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int lanes = p.pool.head_dim / 8, rows = ROW_THREADS / lanes;
  const int64_t n_units = (int64_t)p.n_tokens * p.pool.n_kv_heads;
  const int c = threadIdx.x % lanes * 8;
  int64_t t[U];
  int head[U], page[U], slot[U], user[U], pos[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int64_t unit = ((int64_t)blockIdx.x * U + j) * rows + threadIdx.x / lanes;
    t[j] = unit < n_units ? unit / p.pool.n_kv_heads : -1;
    if (t[j] < 0) continue;
    head[j] = (int)(unit - t[j] * p.pool.n_kv_heads);
    pos[j] = p.positions[t[j]];
    user[j] = p.users ? p.users[t[j]] : (int)t[j];
  }
#pragma unroll
  for (int j = 0; j < U; ++j) {
    if (t[j] < 0) continue;
    const int32_t *at = place(p, user[j], pos[j], head[j] == 0 && c == 0, slot[j]);
    if (at)
      page[j] = *at;
    else
      t[j] = -1;
  }
  uint32_t kw[U], vw[U], kp[U], vp[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    if (t[j] >= 0 && !page_ok(p, page[j], head[j] == 0 && c == 0)) t[j] = -1;
    if (t[j] < 0) continue;
    const uint8_t *block = p.pool.block(page[j], p.layer, head[j]);
    const int at = slot[j] * (p.pool.head_dim / 2) + c / 2;
    const uint8_t *params = block + 2 * p.pool.code_bytes() + (slot[j] * (p.pool.head_dim / KV4_GROUP) + c / KV4_GROUP) * 4;
    kw[j] = *reinterpret_cast<const uint32_t *>(block + at);
    vw[j] = *reinterpret_cast<const uint32_t *>(block + p.pool.code_bytes() + at);
    kp[j] = *reinterpret_cast<const uint32_t *>(params);
    vp[j] = *reinterpret_cast<const uint32_t *>(params + p.pool.param_bytes());
  }
#pragma unroll
  for (int j = 0; j < U; ++j) {
    if (t[j] < 0) continue;
    store_values<T, WIDE>(kw[j], kp[j], reinterpret_cast<T *>(p.k.row(t[j], head[j])) + c);
    store_values<T, WIDE>(vw[j], vp[j], reinterpret_cast<T *>(p.v.row(t[j], head[j])) + c);
  }
}

template <class T, bool WIDE, int U>
cudaError_t launch_units(const RowsParams &p, bool reads, cudaStream_t s) {
  const int rows = ROW_THREADS / (p.pool.head_dim / 8) * U;
  const int64_t grid = ((int64_t)p.n_tokens * p.pool.n_kv_heads + rows - 1) / rows;
  if (grid > 0x7fffffff) return cudaErrorInvalidValue;
  return reads ? launch_chained(kv4_read_kernel<T, WIDE, U>, (unsigned)grid, ROW_THREADS, 0, s, p)
               : launch_chained(kv4_append_kernel<T, WIDE, U>, (unsigned)grid, ROW_THREADS, 0, s, p);
}

// Rows that fill the SMs many times over: two or four a thread.  Few, or off 16 bytes: one, spread as widely as they go.
template <class T>
cudaError_t launch_rows(const RowsParams &p, bool reads, bool wide, cudaStream_t s) {
  const int64_t threads = (int64_t)p.n_tokens * p.pool.n_kv_heads * (p.pool.head_dim / 8);
  if (!wide) return launch_units<T, false, 1>(p, reads, s);
  if (threads < 8 * 152 * 2048) return launch_units<T, true, 1>(p, reads, s);
  return reads ? launch_units<T, true, 4>(p, reads, s) : launch_units<T, true, 2>(p, reads, s);
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
