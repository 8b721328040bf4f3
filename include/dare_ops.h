/*
 * libdare — stand-alone operators of a transformer block, for callers that build a pass of their own around (or instead of)
 * the DARE layer of dare.h: models with grouped key/value heads, projection biases, other rotary layouts or positions scaled
 * past the trained ones, prompts of different lengths in one batch, causal prefixes.  The attention half of a block is
 *
 *     dare_rmsnorm -> dare_linear (queries, keys, values; biases) -> dare_rope -> dare_attention -> dare_linear (+ residual)
 *
 * Conventions of dare.h: plain C, device pointers, dare_status_t, work is enqueued on the given stream and the call returns;
 * nothing is allocated; calls may be captured into a CUDA graph (once a call of the same types has run outside a capture).
 * Strides are in elements; the elements of a row (of a head) lie side by side.  Unlike weights of a layer handle, every
 * operand may be what the kernel before on the stream writes.  Outputs must not overlap inputs, except where it is said.
 *
 * `status`: a device int32 of the caller's (or NULL), written only when a kernel sees a problem: DARE_ERR_DEVICE_CHECK (a
 * position, a row index or a length that is out of range: what it would have addressed is left alone) or DARE_ERR_TIMEOUT (a
 * bounded wait ran out, results are not to be relied on).  A recorded value stays until the caller clears it.
 *
 * The calls keep nothing between them and may run on several streams at once, each with its own workspace and outputs.
 */
#ifndef DARE_OPS_H_
#define DARE_OPS_H_

#include "dare.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions ------------------------------------------------------------------------------------------------
 * Pair j of rotary_dim / 2 turns by p * f_j at position p, f_j = theta^(-2 j / rotary_dim), scaled for contexts longer than
 * the trained ones (`factor` = s >= 1):
 *   NONE     f_j
 *   LINEAR   f_j / s                                       (positions squeezed into the trained range)
 *   BASE     theta * s^(r / (r - 2)) in theta's place      (r = rotary_dim > 2)
 *   TURNS    keep f_j + (1 - keep) f_j / s,  keep = clip((t_j - low) / (high - low), 0, 1),  t_j = trained f_j / 2 pi: the turns
 *            that the pair makes over the `trained` positions
 *   INDEX    the same with keep falling linearly in j, from 1 at the index of `high` turns (rounded down, at least 0) to 0 at
 *            that of `low` turns (rounded up, at most r - 1)
 * `magnitude` multiplies cosines and sines (1 for none). */
enum {
  DARE_ROPE_SCALE_NONE = 0,
  DARE_ROPE_SCALE_LINEAR = 1,
  DARE_ROPE_SCALE_BASE = 2,
  DARE_ROPE_SCALE_TURNS = 3,
  DARE_ROPE_SCALE_INDEX = 4
};
/* HALF: element j turns with j + rotary_dim / 2 (as in the layer); INTERLEAVED: 2 j with 2 j + 1. */
enum { DARE_ROPE_HALF = 0, DARE_ROPE_INTERLEAVED = 1 };

typedef struct {
  uint32_t struct_size; /* sizeof(dare_rope_config_t) */
  int32_t rotary_dim;   /* even, at most 256 */
  double theta;         /* > 0 */
  int32_t scaling;      /* DARE_ROPE_SCALE_* */
  int32_t trained;      /* TURNS, INDEX: positions the model was trained on */
  double factor;        /* s >= 1 (ignored by NONE) */
  double low, high;     /* TURNS, INDEX: 0 < low < high */
  double magnitude;
} dare_rope_config_t;

/* table[p][j] = magnitude * (cos, sin)(p f_j) for positions [0, positions), float32 [positions, rotary_dim / 2, 2]; worked out in
 * float64.  8-byte aligned; positions <= 2^24. */
dare_status_t dare_rope_table(const dare_rope_config_t* cfg, float* table, int64_t positions, void* cuda_stream);

typedef struct {
  uint32_t struct_size; /* sizeof(dare_rope_apply_t) */
  int32_t dtype;        /* dare_dtype_t of x and y */
  int64_t tokens;       /* <= 2^30 */
  int32_t heads;
  int32_t head_dim;     /* <= 65536 */
  int32_t rotary_dim;   /* even, <= head_dim and 256: the leading elements of a head, the rest are copied */
  int32_t layout;       /* DARE_ROPE_HALF / _INTERLEAVED */
  int32_t transpose;    /* 1: angles negated: the gradient of the forward call (magnitude 1: also its inverse) */
  int32_t pos_begin;    /* positions == NULL: token t has position pos_begin + t */
  int64_t x_token, x_head, y_token, y_head; /* strides */
  int64_t table_positions;                  /* rows of the table */
} dare_rope_apply_t;

/* y = x with every head's pairs turned by the table's row of the token's position.  positions: int32 [tokens] or NULL.  A token
 * whose position is outside the table is left as y had it (DARE_ERR_DEVICE_CHECK).  y may be x with the same strides. */
dare_status_t dare_rope(const dare_rope_apply_t* cfg, const void* x, const int32_t* positions, const float* table, void* y,
                        int32_t* status, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* DARE_OPS_H_ */
