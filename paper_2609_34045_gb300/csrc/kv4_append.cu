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

// The page and slot of row t, or a page of -1 (reported once per row).
__device__ __forceinline__ int locate(const RowsParams &p, int64_t t, int pos, bool reports, int &slot) {
  const int user = p.users ? p.users[t] : (int)t;
  int bad = 0, page = -1;
  if (user < 0 || user >= p.map.n_users) {
    bad = KFL_BAD_USER;
  } else if (pos < 0 || (pos >> p.pool.log2_tokens) >= p.map.max_pages || (p.cos_sin && pos >= p.n_pos)) {
    bad = KFL_BAD_POSITION;
  } else {
    page = p.map.table[(int64_t)user * p.map.max_pages + (pos >> p.pool.log2_tokens)];
    if (page < 0 || page >= p.pool.n_pages) bad = page == -1 ? KFL_BAD_POSITION : KFL_BAD_PAGE, page = -1;
  }
  if (bad && reports) report(p.status, bad);
  slot = pos & (p.pool.page_tokens() - 1);
  return page;
}

template <class T, bool WIDE>
__device__ __forceinline__ void load8(const T *p, float (&x)[8]) {
  if constexpr (WIDE) {
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8; i += W) {
      const Pack<T, W> w = *reinterpret_cast<const Pack<T, W> *>(p + i);
#pragma unroll
      for (int j = 0; j < W; ++j) x[i + j] = to_f32(w.e[j]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f32(p[i]);
  }
}

// Channels [c, c + 8) of a k row, rotated.
template <class T, bool WIDE>
__device__ __forceinline__ void load8_rotated(const RowsParams &p, const T *row, int c, int pos, float (&x)[8]) {
  load8<T, WIDE>(row + c, x);
  const int half = p.rope_half;
  if (!p.cos_sin || c >= 2 * half) return;
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
    load8<T, WIDE>(row + (second ? c - half : c + half), y);
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

template <class T, bool WIDE>
__global__ void __launch_bounds__(ROW_THREADS) kv4_append_kernel(const RowsParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int lanes = p.pool.head_dim / 8;  // threads of a row
  const int64_t unit = (int64_t)blockIdx.x * (ROW_THREADS / lanes) + threadIdx.x / lanes;
  const int64_t n_units = (int64_t)p.n_tokens * p.pool.n_kv_heads;
  const int c = threadIdx.x % lanes * 8;
  // (a block's last threads repeat the last row without storing it: the shuffles take whole warps)
  const int64_t u = min(unit, n_units - 1);
  const int64_t t = u / p.pool.n_kv_heads;
  const int head = (int)(u % p.pool.n_kv_heads);
  const int pos = p.positions[t];
  int slot;
  const int page = locate(p, t, pos, head == 0 && c == 0 && unit < n_units, slot);
  float x[8], y[8];
  load8<T, WIDE>(reinterpret_cast<const T *>(p.v.row(t, head)) + c, y);
  const T *k_row = reinterpret_cast<const T *>(p.k.row(t, head));
  if (page >= 0)
    load8_rotated<T, WIDE>(p, k_row, c, pos, x);
  else
    load8<T, WIDE>(k_row + c, x);
  uint32_t kp, vp;
  const uint32_t kw = quantise8(x, threadIdx.x & 31, kp);
  const uint32_t vw = quantise8(y, threadIdx.x & 31, vp);
  if (unit >= n_units || page < 0) return;
  uint8_t *block = p.pool.block(page, p.layer, head);
  const int row = slot * (p.pool.head_dim / 2) + c / 2;
  *reinterpret_cast<uint32_t *>(block + row) = kw;
  *reinterpret_cast<uint32_t *>(block + p.pool.code_bytes() + row) = vw;
  if (c % KV4_GROUP == 0) {
    uint8_t *params = block + 2 * p.pool.code_bytes() + (slot * (p.pool.head_dim / KV4_GROUP) + c / KV4_GROUP) * 4;
    *reinterpret_cast<uint32_t *>(params) = kp;
    *reinterpret_cast<uint32_t *>(params + p.pool.param_bytes()) = vp;
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

template <class T, bool WIDE>
__global__ void __launch_bounds__(ROW_THREADS) kv4_read_kernel(const RowsParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int lanes = p.pool.head_dim / 8;
  const int64_t unit = (int64_t)blockIdx.x * (ROW_THREADS / lanes) + threadIdx.x / lanes;
  if (unit >= (int64_t)p.n_tokens * p.pool.n_kv_heads) return;
  const int c = threadIdx.x % lanes * 8;
  const int64_t t = unit / p.pool.n_kv_heads;
  const int head = (int)(unit % p.pool.n_kv_heads);
  int slot;
  const int page = locate(p, t, p.positions[t], head == 0 && c == 0, slot);
  if (page < 0) return;
  const uint8_t *block = p.pool.block(page, p.layer, head);
  const int row = slot * (p.pool.head_dim / 2) + c / 2;
  const uint8_t *params = block + 2 * p.pool.code_bytes() + (slot * (p.pool.head_dim / KV4_GROUP) + c / KV4_GROUP) * 4;
  const uint32_t kw = *reinterpret_cast<const uint32_t *>(block + row);
  const uint32_t vw = *reinterpret_cast<const uint32_t *>(block + p.pool.code_bytes() + row);
  const uint32_t kp = *reinterpret_cast<const uint32_t *>(params);
  const uint32_t vp = *reinterpret_cast<const uint32_t *>(params + p.pool.param_bytes());
  store_values<T, WIDE>(kw, kp, reinterpret_cast<T *>(p.k.row(t, head)) + c);
  store_values<T, WIDE>(vw, vp, reinterpret_cast<T *>(p.v.row(t, head)) + c);
}

template <class T>
cudaError_t launch_rows(const RowsParams &p, bool reads, bool wide, cudaStream_t s) {
  const int rows = ROW_THREADS / (p.pool.head_dim / 8);
  const int64_t grid = ((int64_t)p.n_tokens * p.pool.n_kv_heads + rows - 1) / rows;
  if (grid > 0x7fffffff) return cudaErrorInvalidValue;
  if (reads)
    return wide ? launch_chained(kv4_read_kernel<T, true>, (unsigned)grid, ROW_THREADS, 0, s, p)
                : launch_chained(kv4_read_kernel<T, false>, (unsigned)grid, ROW_THREADS, 0, s, p);
  return wide ? launch_chained(kv4_append_kernel<T, true>, (unsigned)grid, ROW_THREADS, 0, s, p)
              : launch_chained(kv4_append_kernel<T, false>, (unsigned)grid, ROW_THREADS, 0, s, p);
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
