// Rows of heads that callers keep themselves (kfl_heads): views, loads and stores of their three types, and
// what the entry points of include/kafila_rope.h and include/kafila_kv4.h check alike.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdio.h>

#include "../../include/kafila_rope.h"
#include "common.cuh"

namespace kfl {

void set_error_detail(const char *msg);  // what kfl_last_error_detail returns

// An argument error with its text.
inline int bad_arg(const char *where, const char *what) {
  char msg[256];
  snprintf(msg, sizeof(msg), "%s: %s", where, what);
  set_error_detail(msg);
  return KFL_ERR_ARG;
}
inline int cuda_result(cudaError_t e, const char *where) {
  if (e == cudaSuccess) return KFL_OK;
  char msg[256];
  snprintf(msg, sizeof(msg), "%s: %s", where, cudaGetErrorString(e));
  set_error_detail(msg);
  return KFL_ERR_CUDA;
}

// Launch with the attribute that lets the grid come up while the kernel before it ends: every kernel launched
// through here executes pdl_wait() before it touches memory.
template <class... P, class... A>
cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, A... args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid, cfg.blockDim = block, cfg.dynamicSmemBytes = smem, cfg.stream = s;
  cfg.attrs = attr, cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

struct HeadsView {
  char *data;
  int64_t token_bytes, head_bytes;
  __device__ __forceinline__ char *row(int64_t t, int h) const { return data + t * token_bytes + h * head_bytes; }
};

inline int dtype_size(int dtype) { return dtype == KFL_DT_FP32 ? 4 : 2; }
inline HeadsView view_of(const kfl_heads &h) {
  const int64_t sz = dtype_size(h.dtype);
  return {static_cast<char *>(h.data), h.token_stride * sz, h.head_stride * sz};
}
// Wide accesses: every row starts on 16 bytes.
inline bool rows_aligned16(const kfl_heads &h) {
  const HeadsView v = view_of(h);
  return ((reinterpret_cast<uintptr_t>(h.data) | (uintptr_t)v.token_bytes | (uintptr_t)v.head_bytes) & 15) == 0;
}
// (a call without tokens may come without data)
inline bool heads_valid(const kfl_heads *h, int n_tokens) {
  return h && (h->data || n_tokens == 0) && h->n_heads >= 1 && h->n_heads <= (1 << 16) && h->dtype >= KFL_DT_BF16 &&
         h->dtype <= KFL_DT_FP32 && reinterpret_cast<uintptr_t>(h->data) % dtype_size(h->dtype) == 0;
}
inline bool rope_valid(const kfl_rope_plan *r) {
  return r && r->cos_sin && (reinterpret_cast<uintptr_t>(r->cos_sin) & 15) == 0 && r->n_pos >= 1 && r->rope_dim >= 2 &&
         r->rope_dim % 2 == 0 && r->rope_dim <= 512 &&
         (r->layout == KFL_ROPE_HALF || r->layout == KFL_ROPE_INTERLEAVED);
}

__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }
template <class T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) {
  return __float2half_rn(x);
}
template <>
__device__ __forceinline__ float from_f32<float>(float x) {
  return x;
}

// V elements, moved as one access when V is more than one.
template <class T, int V>
struct alignas(V == 1 ? sizeof(T) : 16) Pack {
  T e[V];
};
// Moves one as one access (assigned, its elements may be moved one by one).
template <int V, class T>
__device__ __forceinline__ void move_pack(T *dst, const T *src) {
  static_assert(V == 1 || V * sizeof(T) == 16, "an element or 16 bytes");
  if constexpr (V == 1)
    *dst = *src;
  else
    *reinterpret_cast<uint4 *>(dst) = *reinterpret_cast<const uint4 *>(src);
}

// a' = a c - b s and b' = b c + a s with every product and sum rounded: the same values whatever the
// compiler would fuse, so that a cache's codes do not hang on it.
__device__ __forceinline__ float rope_first(float a, float b, float2 cs) {
  return __fsub_rn(__fmul_rn(a, cs.x), __fmul_rn(b, cs.y));
}
__device__ __forceinline__ float rope_second(float a, float b, float2 cs) {
  return __fadd_rn(__fmul_rn(b, cs.x), __fmul_rn(a, cs.y));
}

__device__ __forceinline__ void report(int32_t *status, int bits) {
  if (status) atomicOr(status, bits);
}

}  // namespace kfl
