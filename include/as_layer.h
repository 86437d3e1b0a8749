/*
 * as_layer.h - C ABI of the bf16 steps around the hybrid attention, for NVIDIA B200 (sm_100a).
 *
 * Between a layer's products and its attention stand the norms of queries and keys and their rotation by the tokens' positions; behind
 * the attention, and in the feed-forward half, linear layers with what follows them.  These calls are those steps, with their gradients:
 *
 *   as_rotary_table             cos and sin of every position of every axis
 *   as_qk_norm_rotary           queries and keys: norm for each head or over a token's heads, rotation, both or either; one tensor or two
 *   as_qk_norm_rotary_backward  the gradients of its inputs and weights
 *   as_linear                   out = residual + gate * act(x w^T + bias)
 *   as_linear_backward          the gradients of x, w, bias and gate
 *
 * Conventions as in as_fp8.h: device pointers, the caller's buffers and stream, nothing allocated, no synchronisation, calls can be
 * captured; on error nothing has been launched.  Sums are fp32 in an order that depends on sizes, types, layouts, the alignment of
 * addresses and the device alone: results are run-to-run identical.
 */
#ifndef AS_LAYER_H_
#define AS_LAYER_H_

#include "as_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- rotation
 * Pair i of a head is turned by the angle of its axis's position: (a, b) -> (a cos - b sin, a sin + b cos).  A head's first 2 P elements
 * are P pairs, (2 i, 2 i + 1) or (i, i + P); the elements behind them stay as they are.  The pairs belong to up to four axes in turn. */
enum { AS_ROTARY_INTERLEAVED = 0, AS_ROTARY_HALF = 1 };
enum { AS_ROTARY_PLAIN = 0, AS_ROTARY_LINEAR = 1, AS_ROTARY_NTK = 2, AS_ROTARY_YARN = 3 };
enum { AS_ROTARY_MAX_AXES = 4 };

/* Pair i of an axis of n pairs turns by position * f: f = base^(-i / n), for longer contexts than a model was trained on changed by `scaling`:
 *   LINEAR  f / factor                                             (positions are interpolated)
 *   NTK     the base becomes base * factor^(n / (n - 1))           (n == 1: f = 1)
 *   YARN    r = original * f / 2 pi turns over the trained context, g = clamp((r - 1) / 31, 0, 1): f g + (f / factor) (1 - g), and cos and
 *           sin times 0.1 ln(factor) + 1 */
typedef struct {
  int32_t size;             /* positions 0 .. size - 1, >= 1 */
  int32_t pairs;            /* >= 1 */
  int32_t scaling;
  int32_t reserved;         /* 0 */
  double base;              /* > 0, finite */
  double factor;            /* >= 1, finite; PLAIN: not looked at */
  double original;          /* > 0, finite: YARN only */
} as_rotary_axis_t;

/* table [sum of sizes][sum of pairs][2] fp32, 16-byte aligned: (cos, sin); axis a's positions are the rows behind those of the axes before it, in which
 * its own pairs are filled and the others are 0.  Angles are taken in 64 bits.  Up to 2^31 - 1 rows, 8192 pairs. */
AS_API as_status_t as_rotary_table(const as_rotary_axis_t* axes, int32_t n_axes, float* table, void* cuda_stream);

typedef struct {
  const float* table;       /* as above, 8-byte aligned (16: vectors); NULL: nothing is turned */
  int32_t n_axes;           /* 1 .. 4 */
  int32_t size[AS_ROTARY_MAX_AXES];
  int32_t pairs[AS_ROTARY_MAX_AXES];   /* their sum: up to head_dim / 2 */
  int32_t layout;           /* AS_ROTARY_INTERLEAVED | AS_ROTARY_HALF */
  int32_t inverse;          /* 1: the transposed rotation */
  int32_t position_bytes;   /* 4 or 8: of an element of `positions` */
  const void* positions;    /* [entries][tokens][n_axes] whole numbers; an element turned by one outside of its axis is NaN.  NULL: token t of every entry is
                               at `first + t` in the axes' raster order (the last axis fastest), which has to lie in the grid */
  int64_t positions_stride; /* elements from one entry's positions to the next one's; 0: they share them */
  int64_t first;
} as_rotation_t;

enum { AS_NORM_NONE = 0, AS_NORM_HEAD = 1, AS_NORM_ROW = 2 };

/* out = R (x * rsqrt(mean(x^2) + eps) * weight), the mean over a head (weight: [head_dim]) or over all heads of a token (weight: [heads * head_dim]).
 * Matrices are as_rows_t of `rows` tokens (rows / tokens entries) and heads * head_dim columns, head_dim the same in all of them, q and k of as many rows
 * and tokens; types bf16 or fp32, the same for all of a call.  A result may be its own input itself in the same layout, and overlaps no other tensor.  fp32 throughout, one rounding at the end.  Holds for every finite x,
 * whatever its squares are in fp32; a head (row) of zeros with eps == 0 is NaN. */
typedef struct {
  uint32_t struct_size;     /* sizeof(as_qk_norm_rotary_t) */
  int32_t norm;             /* AS_NORM_*; NONE: eps and the weights are not looked at */
  int64_t rows;             /* 0 .. 2^31 - 1 */
  int32_t head_dim;         /* 1 .. 1024; norm over rows: heads * head_dim up to 16384 */
  int32_t q_heads, k_heads; /* >= 1; k_heads is not looked at where k.data == NULL */
  float eps;                /* >= 0 */
  as_rows_t q, k;           /* k.data == NULL: q alone */
  as_rows_t q_out, k_out;
  const void *q_weight, *k_weight;   /* NULL: ones */
  int32_t weight_dtype;
  int32_t reserved;         /* 0 */
  as_rotation_t rotation;
} as_qk_norm_rotary_t;
AS_API as_status_t as_qk_norm_rotary(const as_qk_norm_rotary_t* args, void* cuda_stream);

/* From the gradients of its outputs and its inputs: with n = x * r, r = rsqrt(mean(x^2) + eps), d = R^T dy:
 *   dx = r (d w - n mean(d w n)),   dw = sum of d n over tokens (and heads, where they share w), in the weights' type.
 * `fwd`: the forward call's arguments, of which q_out and k_out are not looked at; the norm is not NONE.  dw pointers are NULL where no gradient is wanted or there is no weight.
 * dq_out may be dq or q itself in the same layout. */
typedef struct {
  uint32_t struct_size;     /* sizeof(as_qk_norm_rotary_backward_t) */
  int32_t reserved;         /* 0 */
  const as_qk_norm_rotary_t* fwd;
  as_rows_t dq, dk;         /* gradients of q_out, k_out */
  as_rows_t dq_out, dk_out; /* gradients of q, k */
  void *dq_weight, *dk_weight;
  void* workspace;          /* 16-byte aligned, as_qk_norm_rotary_backward_workspace_bytes */
  uint64_t workspace_bytes;
} as_qk_norm_rotary_backward_t;
AS_API as_status_t as_qk_norm_rotary_backward_workspace_bytes(const as_qk_norm_rotary_backward_t* args, uint64_t* bytes);
AS_API as_status_t as_qk_norm_rotary_backward(const as_qk_norm_rotary_backward_t* args, void* cuda_stream);

/* ---------------------------------------------------------------- linear layers */
enum { AS_ACT_NONE = -1 /* AS_ACT_RELU = 0 */, AS_ACT_SILU = 1, AS_ACT_GELU = 2 /* by the error function */, AS_ACT_GELU_TANH = 3 };

/* z = x w^T + bias, out = residual + gate * act(z): products of bf16 values summed in fp32, everything behind them in fp32 from the unrounded z, one rounding
 * into out and one into pre (z itself, for the backward pass).  rows == 0 launches nothing. */
typedef struct {
  uint32_t struct_size;     /* sizeof(as_linear_t) */
  int32_t activation;
  int64_t rows;             /* M, 0 .. 2^30 */
  int64_t cols, out_cols;   /* K, N: 1 .. 2^20 */
  as_rows_t x;              /* [M, K] bf16 */
  as_rows_t w;              /* [N, K] bf16, rows (head_dim == cols) */
  as_rows_t residual;       /* [M, N] bf16 or fp32, or data == NULL */
  as_rows_t out;            /* [M, N] bf16 or fp32; may be the residual itself in the same layout; out and pre overlap nothing else */
  as_rows_t pre;            /* [M, N] bf16, or data == NULL */
  const void* bias;         /* [N], or NULL */
  const void* gate;         /* [gates][N], gate_stride elements apart, or NULL; rows / gates rows in turn share one */
  int32_t bias_dtype, gate_dtype;
  int64_t gates, gate_stride;   /* gates: 1 .. 65534, a divisor of rows */
  void* workspace;          /* 256-byte aligned, as_linear_workspace_bytes of it (which may be 0); calls in flight at once have one each */
  uint64_t workspace_bytes;
} as_linear_t;
AS_API as_status_t as_linear_workspace_bytes(as_fp8_context_t ctx, const as_linear_t* args, uint64_t* bytes);
AS_API as_status_t as_linear(as_fp8_context_t ctx, const as_linear_t* args, void* cuda_stream);

/* With z = pre as it was kept and u = act(z): dz = dy * gate * act'(z), rounded to bf16 as an operand of the two products,
 *   dx = dz w,  dw = dz^T x  (bf16),  dbias = sum of dz over the rows,  dgate = sum of dy * u over the rows that share it  (from the unrounded ones).
 * The residual's gradient is dy itself.  Outputs with data == NULL are not computed. */
typedef struct {
  uint32_t struct_size;     /* sizeof(as_linear_backward_t) */
  int32_t activation;
  int64_t rows, cols, out_cols;
  as_rows_t dy;             /* [M, N] bf16 or fp32 */
  as_rows_t x, w;           /* as in as_linear_t; x is looked at for dw alone, w for dx alone */
  as_rows_t pre;            /* [M, N] bf16; required with an activation or where dgate is asked for */
  as_rows_t dx;             /* [M, K] bf16, or NULL */
  as_rows_t dw;             /* [N, K] bf16, rows, or NULL */
  const void* gate;
  void* dbias;              /* [N], or NULL */
  void* dgate;              /* [gates][N], N elements apart, or NULL */
  int32_t bias_dtype, gate_dtype;   /* of dbias; of gate and dgate */
  int64_t gates, gate_stride;
  void* workspace;
  uint64_t workspace_bytes;
} as_linear_backward_t;
AS_API as_status_t as_linear_backward_workspace_bytes(as_fp8_context_t ctx, const as_linear_backward_t* args, uint64_t* bytes);
AS_API as_status_t as_linear_backward(as_fp8_context_t ctx, const as_linear_backward_t* args, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif  /* AS_LAYER_H_ */
