// Rotary positions of callers' q and k heads (include/kafila_rope.h).
//
// A pass reads and writes every element once and the angles' row once per token: memory bound, 2 flops a byte.
// A thread keeps one vector of angles in registers and turns that vector's pairs in every head of its token that
// falls to it, so the table's row (8 bytes an angle, against 4 a 16-bit pair) is read once per CTA and not once
// per head; its loads, up to four heads', are issued together and before the position is known.  8192 tokens of 28 + 4 heads
// of 128, half of each turned, in fp16: 24.5 us, 5.6 TB/s (vectors assigned as structs, which the compiler moves in parts: 31; one head a thread and
// the position first: 49 us).
#include <math.h>

#include <algorithm>

#include "heads.cuh"

namespace kfl {
namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_AHEAD = 4;  // heads whose loads a thread issues together

struct RopeParams {
  HeadsView in[2], out[2];  // q, k
  int n_q, n_heads;         // query heads, all heads
  int copies[2];            // an output that is not its input gets the channels behind rope_dim too
  const float2 *cos_sin;
  const int32_t *positions;
  int n_pos, rope_half, head_dim;
  int n_rot, n_items;       // vector pairs of a head that turn; and those that are copied with them
  int heads_per_block, heads_per_step;
  float sign;
  int32_t *status;
};

template <class T, int V, bool HALF>
__global__ void __launch_bounds__(ROPE_THREADS) rope_kernel(const RopeParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int64_t t = blockIdx.x;
  const int pos = p.positions[t];
  using Vec = Pack<T, V>;
  const int item = threadIdx.x % p.n_items, head0 = threadIdx.x / p.n_items;
  const bool turns = item < p.n_rot;
  // the item's two vectors: elements [a, a + V) and [b, b + V) of a head
  int a, b;
  if (turns) {
    a = HALF ? item * V : 2 * item * V;
    b = HALF ? p.rope_half + item * V : a + V;
  } else {
    a = 2 * p.rope_half + 2 * (item - p.n_rot) * V;
    b = a + V;
  }
  const bool has_b = b < p.head_dim;
  const int first = blockIdx.y * p.heads_per_block;
  const int last = min(p.n_heads, first + p.heads_per_block);
  Vec x[ROPE_AHEAD], y[ROPE_AHEAD];
  const auto load = [&](int h0) {
#pragma unroll
    for (int j = 0; j < ROPE_AHEAD; ++j) {
      const int h = h0 + j * p.heads_per_step;
      if (h >= last) break;
      const int which = h >= p.n_q;
      if (!turns && !p.copies[which]) continue;
      const T *src = reinterpret_cast<const T *>(p.in[which].row(t, h - (which ? p.n_q : 0)));
      move_pack<V>(x[j].e, src + a);
      if (has_b) move_pack<V>(y[j].e, src + b);
    }
  };
  load(first + head0);  // (under way before the position is known)
  if (pos < 0 || pos >= p.n_pos) {
    if (blockIdx.y == 0 && threadIdx.x == 0) report(p.status, KFL_BAD_POSITION);
    return;
  }
  float2 cs[V];
  if (turns) {
    const float2 *row = p.cos_sin + (int64_t)pos * p.rope_half + item * V;
#pragma unroll
    for (int i = 0; i < V; i += V > 1 ? 2 : 1) {
      if constexpr (V > 1) {
        const float4 f = *reinterpret_cast<const float4 *>(row + i);
        cs[i] = {f.x, f.y * p.sign}, cs[i + 1] = {f.z, f.w * p.sign};
      } else {
        cs[i] = {row[i].x, row[i].y * p.sign};
      }
    }
  }
  for (int h0 = first + head0; h0 < last; h0 += ROPE_AHEAD * p.heads_per_step) {
    if (h0 != first + head0) load(h0);
#pragma unroll
    for (int j = 0; j < ROPE_AHEAD; ++j) {
      const int h = h0 + j * p.heads_per_step;
      if (h >= last) break;
      const int which = h >= p.n_q;
      if (!turns && !p.copies[which]) continue;
      if (turns) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          // pair i of the item: (x[i], y[i]), or neighbours within the two vectors laid end to end
          T *fa, *fb;
          if constexpr (HALF) {
            fa = &x[j].e[i], fb = &y[j].e[i];
          } else if constexpr (V == 1) {
            fa = &x[j].e[0], fb = &y[j].e[0];
          } else {
            fa = 2 * i < V ? &x[j].e[2 * i] : &y[j].e[2 * i - V];
            fb = fa + 1;
          }
          const float u = to_f32(*fa), v = to_f32(*fb);
          *fa = from_f32<T>(rope_first(u, v, cs[i]));
          *fb = from_f32<T>(rope_second(u, v, cs[i]));
        }
      }
      T *dst = reinterpret_cast<T *>(p.out[which].row(t, h - (which ? p.n_q : 0)));
      move_pack<V>(dst + a, x[j].e);
      if (has_b) move_pack<V>(dst + b, y[j].e);
    }
  }
}

struct RopeFreqs {
  double f[256];
};

__global__ void rope_table_kernel(const RopeFreqs freqs, int half, double magnitude, int n_pos, float2 *out) {
  pdl_launch_dependents();
  pdl_wait();
  const int64_t n = (int64_t)n_pos * half;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
    double s, c;
    sincos((double)(i / half) * freqs.f[i % half], &s, &c);
    out[i] = {(float)(c * magnitude), (float)(s * magnitude)};
  }
}

bool same_rows(const kfl_heads &a, const kfl_heads &b) {
  return a.data == b.data && a.token_stride == b.token_stride && a.head_stride == b.head_stride;
}

template <class T>
cudaError_t launch_rope(RopeParams &p, bool wide, bool half, int n_tokens, cudaStream_t s) {
  constexpr int W = 16 / sizeof(T);
  const int V = wide ? W : 1;
  p.n_rot = p.rope_half / V;
  const int rest = (p.copies[0] || p.copies[1]) ? (p.head_dim - 2 * p.rope_half) / V : 0;
  p.n_items = p.n_rot + (rest + 1) / 2;
  // Few tokens: a head or two per thread, so that the rows spread over the SMs (4 tokens of 72 heads of 128: 36
  // blocks).  Many: a block per token with up to four heads per thread, whose loads are in flight together.
  const bool few = n_tokens < 304;
  const int most = std::max(1, (few ? 64 : ROPE_THREADS) / p.n_items);
  // (a grid has at most 65535 rows of blocks: of 2 x 65536 heads a block may take more than its threads do at once)
  p.heads_per_block = few ? std::min(p.n_heads, std::max(most, (p.n_heads + 65534) / 65535)) : p.n_heads;
  const int steps = std::max((p.heads_per_block + most - 1) / most, few ? 1 : std::min(p.heads_per_block, ROPE_AHEAD));
  p.heads_per_step = (p.heads_per_block + steps - 1) / steps;
  const dim3 grid(n_tokens, (p.n_heads + p.heads_per_block - 1) / p.heads_per_block);
  const int threads = p.heads_per_step * p.n_items;
  if (wide)
    return half ? launch_chained(rope_kernel<T, W, true>, grid, threads, 0, s, p)
                : launch_chained(rope_kernel<T, W, false>, grid, threads, 0, s, p);
  return half ? launch_chained(rope_kernel<T, 1, true>, grid, threads, 0, s, p)
              : launch_chained(rope_kernel<T, 1, false>, grid, threads, 0, s, p);
}

}  // namespace
}  // namespace kfl

extern "C" int kfl_rope_table(const kfl_rope_cfg *cfg, int n_pos, float *cos_sin, void *cuda_stream) {
  using namespace kfl;
  const char *me = "kfl_rope_table";
  if (!cfg || !cos_sin || n_pos < 1) return bad_arg(me, "NULL pointer or no positions");
  if (reinterpret_cast<uintptr_t>(cos_sin) & 7) return bad_arg(me, "the table is 8-byte aligned (16 for a rotation)");
  if (cfg->rope_dim < 2 || cfg->rope_dim > 512 || cfg->rope_dim % 2) return bad_arg(me, "rope_dim is even, 2..512");
  if (!(cfg->theta > 1.0) || !std::isfinite(cfg->theta)) return bad_arg(me, "theta is above 1");
  if (cfg->scaling < KFL_ROPE_PLAIN || cfg->scaling > KFL_ROPE_RAMP) return bad_arg(me, "unknown scaling");
  if (cfg->scaling != KFL_ROPE_PLAIN && !(cfg->factor >= 1.0 && std::isfinite(cfg->factor)))
    return bad_arg(me, "factor is at least 1");
  if (cfg->scaling == KFL_ROPE_BASE && cfg->rope_dim == 2) return bad_arg(me, "KFL_ROPE_BASE needs a rope_dim above 2");
  const bool bands = cfg->scaling == KFL_ROPE_BANDS || cfg->scaling == KFL_ROPE_RAMP;
  if (bands && !(cfg->low > 0.0 && cfg->high > cfg->low && std::isfinite(cfg->high) && cfg->original_ctx > 0.0 &&
                 std::isfinite(cfg->original_ctx)))
    return bad_arg(me, "0 < low < high and an original_ctx are needed");
  if (!(cfg->magnitude >= 0.0) || !std::isfinite(cfg->magnitude)) return bad_arg(me, "magnitude is not negative");
  const int half = cfg->rope_dim / 2;
  const double pi = 3.14159265358979323846, r = cfg->rope_dim;
  double theta = cfg->theta, magnitude = cfg->magnitude > 0.0 ? cfg->magnitude : 1.0;
  if (cfg->scaling == KFL_ROPE_BASE) theta *= pow(cfg->factor, r / (r - 2.0));
  double ramp0 = 0.0, ramp1 = 0.0;
  if (cfg->scaling == KFL_ROPE_RAMP) {
    const auto index = [&](double turns) { return r * log(cfg->original_ctx / (2.0 * pi * turns)) / (2.0 * log(theta)); };
    ramp0 = std::max(0.0, floor(index(cfg->high)));
    ramp1 = std::min(r - 1.0, ceil(index(cfg->low)));
    if (!(ramp1 > ramp0)) ramp1 = ramp0 + 1e-3;
    if (cfg->magnitude == 0.0) magnitude = 0.1 * log(cfg->factor) + 1.0;
  }
  RopeFreqs freqs;
  for (int i = 0; i < half; ++i) {
    double f = pow(theta, -2.0 * i / r), keep = 1.0;
    if (cfg->scaling == KFL_ROPE_LINEAR) keep = 0.0;
    if (cfg->scaling == KFL_ROPE_BANDS)
      keep = std::min(1.0, std::max(0.0, (cfg->original_ctx * f / (2.0 * pi) - cfg->low) / (cfg->high - cfg->low)));
    if (cfg->scaling == KFL_ROPE_RAMP) keep = 1.0 - std::min(1.0, std::max(0.0, (i - ramp0) / (ramp1 - ramp0)));
    freqs.f[i] = keep == 1.0 ? f : f * keep + f / cfg->factor * (1.0 - keep);
  }
  const int64_t blocks = ((int64_t)n_pos * half + 255) / 256;
  return cuda_result(launch_chained(rope_table_kernel, (unsigned)std::min<int64_t>(blocks, 152 * 16), 256, 0,
                                    static_cast<cudaStream_t>(cuda_stream), freqs, half, magnitude, n_pos,
                                    reinterpret_cast<float2 *>(cos_sin)),
                     me);
}

extern "C" int kfl_rope(const kfl_rope_plan *plan, const kfl_heads *q, const kfl_heads *q_out, const kfl_heads *k,
                        const kfl_heads *k_out, const int32_t *positions, int n_tokens, int head_dim, int inverse,
                        int32_t *status, void *cuda_stream) {
  using namespace kfl;
  const char *me = "kfl_rope";
  if (!rope_valid(plan)) return bad_arg(me, "not a rotation (16-byte aligned table, even rope_dim of 2..512, layout)");
  if (!heads_valid(q, n_tokens) || !heads_valid(q_out, n_tokens)) return bad_arg(me, "q and q_out are needed");
  if (!k != !k_out || (k && (!heads_valid(k, n_tokens) || !heads_valid(k_out, n_tokens))))
    return bad_arg(me, "k and k_out go together");
  if (q->n_heads != q_out->n_heads || q->dtype != q_out->dtype) return bad_arg(me, "q and q_out differ");
  if (k && (k->n_heads != k_out->n_heads || k->dtype != k_out->dtype || k->dtype != q->dtype))
    return bad_arg(me, "k and k_out differ, or k has another type than q");
  if (head_dim < plan->rope_dim || head_dim > 512 || head_dim % 2)
    return bad_arg(me, "head_dim is even, rope_dim..512");
  if (n_tokens < 0 || (n_tokens > 0 && !positions)) return bad_arg(me, "positions are needed");
  if (n_tokens == 0) return KFL_OK;
  RopeParams p = {};
  p.in[0] = view_of(*q), p.out[0] = view_of(*q_out);
  p.in[1] = view_of(k ? *k : *q), p.out[1] = view_of(k ? *k_out : *q_out);
  p.n_q = q->n_heads, p.n_heads = q->n_heads + (k ? k->n_heads : 0);
  const bool rest = head_dim > plan->rope_dim;
  p.copies[0] = rest && !same_rows(*q, *q_out), p.copies[1] = rest && k && !same_rows(*k, *k_out);
  p.cos_sin = reinterpret_cast<const float2 *>(plan->cos_sin);
  p.positions = positions;
  p.n_pos = plan->n_pos, p.rope_half = plan->rope_dim / 2, p.head_dim = head_dim;
  p.sign = inverse ? -1.f : 1.f;
  p.status = status;
  // wide: rows on 16 bytes, and both parts of a head whole vectors
  const int W = 16 / dtype_size(q->dtype);
  const bool wide = rows_aligned16(*q) && rows_aligned16(*q_out) && (!k || (rows_aligned16(*k) && rows_aligned16(*k_out))) &&
                    p.rope_half % W == 0 && head_dim % W == 0;
  const bool half = plan->layout == KFL_ROPE_HALF;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  switch (q->dtype) {
    case KFL_DT_BF16: e = launch_rope<__nv_bfloat16>(p, wide, half, n_tokens, s); break;
    case KFL_DT_FP16: e = launch_rope<__half>(p, wide, half, n_tokens, s); break;
    default: e = launch_rope<float>(p, wide, half, n_tokens, s); break;
  }
  return cuda_result(e, me);
}
