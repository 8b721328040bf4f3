/*
 * libdare — stand-alone operators of a transformer block, for callers that build a pass of their own around (or instead of)
 * the DARE layer of dare.h: models with grouped key/value heads, projection biases, other rotary layouts or positions scaled
 * past the trained ones, prompts of different lengths in one batch, causal prefixes.  The attention half of a block is
 *
 *     dare_rmsnorm -> dare_linear (queries, keys, values; biases) -> dare_rope -> dare_attention -> dare_linear (+ residual)
 *
 * Conventions of dare.h: plain C, device pointers, dare_status_t, work is enqueued on the given stream and the call returns;
 * nothing is allocated; calls may be captured into a CUDA graph (once a call of the same types has run outside a capture).
 * Strides are in elements, not negative, below 2^38; the elements of a row (of a head) lie side by side.  Rows of an input may overlap or repeat
 * (stride 0), places of an output may not.  Unlike weights of a layer handle, every
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
 * whose position is outside the table is left as y had it (DARE_ERR_DEVICE_CHECK).  y may be x with the same strides.
 * By 16 bytes where addresses, strides, the copied part and rotary_dim / 2 (INTERLEAVED: rotary_dim) are multiples of that, else by single
 * elements (pairs): 16384 tokens x 40 heads x 128 in bf16 53 us, with 64 of the 128 turned 68, with 58 175. */
dare_status_t dare_rope(const dare_rope_apply_t* cfg, const void* x, const int32_t* positions, const float* table, void* y,
                        int32_t* status, void* cuda_stream);

/* ---- y = act(x W^T + bias) + resid ----------------------------------------------------------------------------------- */
enum { DARE_ACT_NONE = 0, DARE_ACT_RELU = 1, DARE_ACT_SILU = 2, DARE_ACT_GELU = 3 /* x Phi(x) */, DARE_ACT_GELU_TANH = 4 };

typedef struct {
  uint32_t struct_size; /* sizeof(dare_linear_config_t) */
  int32_t dtype;        /* dare_dtype_t of x, W, resid and y; sums in float32 */
  int64_t rows;         /* <= 2^24; rows * out_features <= 2^38 */
  int32_t in_features;  /* 1 .. 2^20 */
  int32_t out_features; /* 1 .. 2^24 */
  int32_t activation;   /* DARE_ACT_* */
  int32_t reserved;     /* 0 */
  int64_t x_row, w_row, resid_row, y_row; /* strides */
} dare_linear_config_t;

/* x [rows, in_features], w [out_features, in_features] (the layer's convention, y = W x), bias float32 [out_features] or NULL, resid
 * [rows, out_features] or NULL; resid may be y with the same stride.
 * Activations are right to a few units of their value, small ones too; GELU in bf16 to 2^-24 of its argument.
 * bf16 with x, w 16-byte aligned and their strides multiples of 8 runs on the tensor cores, float32 with x, w 16-byte aligned,
 * strides and in_features multiples of 4 too where that is faster (operands split into three bf16 parts, fp32 accuracy); everything
 * else on the CUDA cores, many times slower where rows are many (bf16, 8192 x 1000 x 4096: 62 us; with rows 1004 apart 2.1 ms, 128 x 1001
 * x 4096 51 us instead of 8): rows are worth padding to a multiple of 8. */
dare_status_t dare_linear(const dare_linear_config_t* cfg, const void* x, const void* w, const float* bias, const void* resid,
                          void* y, int32_t* status, void* cuda_stream);

/* ---- softmax attention over packed sequences --------------------------------------------------------------------------
 * Sequence b has the query rows [q_begin[b], q_begin[b + 1]) and the key rows k_begin[b] + [0, n_b), n_b = k_len[b], or without k_len
 * k_begin[b + 1] - k_begin[b].  Query head h reads key/value head h / (n_heads / n_kv_heads).
 *     out_i = sum_j softmax_j(scale q_i . k_j) v_j    over j < n_b and, if causal, j <= i + n_b - (query rows of b)
 * (the last query sees every key).  A row that sees no key gets zeros, and -inf as its lse = log sum_j exp(scale q_i . k_j).
 * Rows of q, out and lse outside every sequence are not touched; k and v are never read into results outside their sequence.
 * The rows (query, head of the group) of a sequence are worked on in tiles of at most 256, in that order from its first: a key and value that
 * causality hides from all of a tile's queries never come into its results; a v row that it hides from some of them only must be
 * finite (its weight there is 0).  One query a sequence is a decoding step; a sequence may be empty. */
typedef struct {
  uint32_t struct_size; /* sizeof(dare_attention_config_t) */
  int32_t dtype;        /* dare_dtype_t of q, k, v and out; softmax in float32 */
  int32_t batch;        /* sequences, 1 .. 65536 */
  int32_t n_heads;      /* a multiple of n_kv_heads */
  int32_t n_kv_heads;
  int32_t head_dim;     /* 32, 64, 128 or 256 */
  int32_t causal;
  float scale;          /* > 0 */
  int64_t q_rows;       /* rows of q, out and lse, <= 2^24; q_rows * n_heads < 2^31 */
  int64_t k_rows;       /* rows of k and v, <= 2^30 */
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head; /* strides */
} dare_attention_config_t;

/* Bytes of device workspace a call needs (16-byte aligned); 0 if the configuration is invalid.  It holds nothing between calls. */
size_t dare_attention_workspace_bytes(const dare_attention_config_t* cfg);

/* q_begin int32 [batch + 1]; k_begin int32 [batch + 1], or [batch] with k_len int32 [batch]; lse float32 [q_rows, n_heads] or NULL.
 * A sequence whose slices are not inside q_rows / k_rows is skipped (DARE_ERR_DEVICE_CHECK); query slices must not overlap (where
 * q_begin runs back and forth, rows may be left out, all of them where the work passes 2^31 units).
 * bf16 with head_dim 64 or 128, q, k, v, out 16-byte aligned and strides multiples of 8 runs on the tensor cores, everything else on
 * the CUDA cores, many times slower on prompts (two of 1500 tokens, 8 and 4 heads of 128: 26 us, of 256: 1.06 ms).
 * On the tensor cores softmax weights meet v as bf16, with head_dim 64 in two parts (16 bits), with 128 in one (8 bits). */
dare_status_t dare_attention(const dare_attention_config_t* cfg, const void* q, const void* k, const void* v,
                             const int32_t* q_begin, const int32_t* k_begin, const int32_t* k_len, void* out, float* lse,
                             void* workspace, size_t workspace_bytes, int32_t* status, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* DARE_OPS_H_ */
