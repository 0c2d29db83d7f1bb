/*
 * Rotary positions of packed rows, beside ce_router.h.
 *
 * A routed layer packs the retained tokens into a shorter sequence (section 3.4),
 * but a retained token keeps its own position: text tokens one number, the tokens of
 * images and videos time, height and width. Queries and keys are turned by these
 * before attention (and before ce_kv_append).
 */
#ifndef CE_ROUTER_ROTARY_H
#define CE_ROUTER_ROTARY_H

#include "ce_router.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { CE_ROTARY_HALVES = 0, CE_ROTARY_PAIRS = 1 };

/*
 * Of every head's head_dim values the first 2 n_pairs are turned, pair i by the angle
 * a = freq[i] * position[axis[i]] of the row's token:
 *   y1 = x1 cos a - x2 sin a,  y2 = x1 sin a + x2 cos a
 * with x1, x2 = x[i], x[i + n_pairs] (CE_ROTARY_HALVES) or x[2 i], x[2 i + 1]
 * (CE_ROTARY_PAIRS). The others stay as they are.
 *   freq      host double [n_pairs]: radians a position, |freq| <= 64
 *   axis      host int32 [n_pairs] in [0, n_axes), or NULL: all 0
 *   inverse   1: turned by -a, which undoes the turn and is its gradient
 *   positions device int32 [n_axes x n_positions]
 *   index     device int32 [rows] or NULL: row r is token index[r] (ce_topk_compact's
 *             kept_idx); NULL: token r. A row whose token is outside [0, n_positions)
 *             is not turned
 * Limits: head_dim even, at most 256, 1 <= n_pairs <= head_dim / 2, 1 <= n_axes <= 4,
 * n_heads < 2^16, rows * n_heads < 2^31, and fewer than 2^32 threads (rows * ceil(n_heads / 4) below
 * 2^24 - 1 needs no more at any width; pairs by eights allow 2^29).
 */
typedef struct ce_rotary_desc {
  int32_t rows;
  int32_t n_heads;
  int32_t head_dim;
  int32_t n_pairs;
  int32_t n_axes;
  int32_t layout;
  int32_t inverse;
  int32_t dtype; /* CE_BF16 or CE_F32 */
  int32_t n_positions;
  const double* freq;
  const int32_t* axis;
  const int32_t* positions;
  const int32_t* index;
} ce_rotary_desc;

/*
 *   x, y   device dtype: row r at r * x_ld (y_ld) elements, its n_heads x head_dim values
 *          contiguous (a part of a fused projection's rows); the strides are
 *          multiples of 8 elements. y may be x (in place, with the same stride), else
 *          they must not overlap
 * The angle is reduced to a turn in 64-bit fixed point, exact to 2^-28 of a turn at any
 * position; cosine, sine and products are float32, rounded once to the output.
 * Errors: CE_ERR_INVALID_ARG for null pointers, sizes, a frequency that is not finite or
 * an axis, layout or inverse out of range; CE_ERR_UNSUPPORTED outside the limits, CE_ERR_HIP.
 */
int ce_rotary(const ce_rotary_desc* desc, const void* x, int64_t x_ld, void* y, int64_t y_ld, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CE_ROUTER_ROTARY_H */
