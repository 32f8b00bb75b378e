/* Rotary positions (RoPE) on their own (sm_103a), for callers that keep q and k themselves.
 *
 * A pair (a, b) of a head's channels at position P is turned by the angle P f_i:
 *   a' = a cos - b sin,  b' = b cos + a sin,   i < rope_dim / 2
 * in fp32, each product and sum rounded, then rounded once to the output's type.  Channels from rope_dim
 * on are copied.  The stage's own kernels (kafila_stage.h) rotate whole heads in the half layout; this is
 * the general form: both layouts, part of the head, frequencies scaled for long contexts, the gradient.
 * The model family that the paper serves (section VI) is read as rotate-half over the whole head.
 *
 * Conventions as in kafila_stage.h.
 */
#ifndef KAFILA_ROPE_H
#define KAFILA_ROPE_H

#include <stdint.h>

#include "kafila_stage.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- element types of the callers' activations ---- */
#define KFL_DT_BF16 0
#define KFL_DT_FP16 1
#define KFL_DT_FP32 2

/* Rows of heads [token][head][head_dim]: strides in elements, the channels of a head contiguous.  data is
 * aligned to the element.  16-byte aligned data and strides (in bytes) take wide loads. */
typedef struct {
  void *data;
  int64_t token_stride, head_stride;
  int n_heads, dtype;
} kfl_heads;

/* ---- bits of a device status word (int32, may be NULL): OR-ed in by the kernels, cleared by the caller.
 * A row that raises one is skipped; the others are computed. ---- */
#define KFL_BAD_POSITION 1 /* a position outside the table, or behind the user's pages */
#define KFL_BAD_USER 2     /* a user outside [0, n_users), or named twice in one call */
#define KFL_BAD_PAGE 4     /* a page number outside [0, n_pages) */
#define KFL_NO_PAGES 8     /* the pool has no free page left, or the user's table row is full */
#define KFL_TIMED_OUT 16   /* a bounded wait inside a kernel gave up: the call's outputs are not valid */

/* ---- pairs of channels ---- */
#define KFL_ROPE_HALF 0        /* (i, i + rope_dim / 2) */
#define KFL_ROPE_INTERLEAVED 1 /* (2 i, 2 i + 1) */

/* ---- frequencies: f_i = theta^(-2 i / rope_dim), then ---- */
#define KFL_ROPE_PLAIN 0
#define KFL_ROPE_LINEAR 1 /* f_i / factor */
#define KFL_ROPE_BASE 2   /* theta * factor^(rope_dim / (rope_dim - 2)) in place of theta */
#define KFL_ROPE_BANDS 3  /* by wavelength w = 2 pi / f_i: kept below original_ctx / high, divided by factor above
                             original_ctx / low, in between blended by (original_ctx / w - low) / (high - low) */
#define KFL_ROPE_RAMP 4   /* by index (Peng et al., arXiv 2309.00071): with d(b) = rope_dim ln(original_ctx / (2 pi b)) /
                             (2 ln theta), kept for i <= floor(d(high)), divided by factor for i >= ceil(d(low)),
                             blended linearly in between; cos and sin times 0.1 ln(factor) + 1 */
typedef struct {
  int rope_dim; /* even, 2..512 */
  int scaling;
  double theta, factor;
  double low, high;    /* BANDS (for example 1, 4), RAMP (for example 1, 32) */
  double original_ctx; /* BANDS, RAMP: the context that the model was trained at */
  double magnitude;    /* cos and sin times this; 0: 1, or RAMP's own */
} kfl_rope_cfg;

/* cos and sin of the angles of positions [0, n_pos): device fp32 [n_pos][rope_dim / 2][2], 8-byte aligned (a
 * kfl_rope_plan wants 16), computed in fp64.  Enqueued on cuda_stream.  Errors: KFL_ERR_ARG, KFL_ERR_CUDA. */
int kfl_rope_table(const kfl_rope_cfg *cfg, int n_pos, float *cos_sin, void *cuda_stream);

/* A rotation: a table of kfl_rope_table (16-byte aligned) and how its pairs lie in a head. */
typedef struct {
  const float *cos_sin;
  int n_pos, rope_dim, layout;
} kfl_rope_plan;

/* Rotates n_tokens rows of q and of k, in one launch, by their positions (device int32 [n_tokens]).  k and
 * k_out may both be NULL.  An output is either its input (same data and strides) or does not overlap it; input
 * and output have the same heads and type.  q and k may differ in heads, not in type.  inverse = 1 turns by
 * the negative angles: the gradient of the rotation (with a magnitude m, m times the transposed matrix).
 *   head_dim  even, rope_dim..512
 * A token whose position is outside [0, n_pos) is left out (its output rows are not written) and reported
 * in status.  Enqueued on cuda_stream, returns without waiting.
 * Errors: KFL_ERR_ARG (NULL, sizes, types), KFL_ERR_CUDA. */
int kfl_rope(const kfl_rope_plan *plan, const kfl_heads *q, const kfl_heads *q_out, const kfl_heads *k,
             const kfl_heads *k_out, const int32_t *positions, int n_tokens, int head_dim, int inverse,
             int32_t *status, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* KAFILA_ROPE_H */
