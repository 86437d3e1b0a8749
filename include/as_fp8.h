/*
 * as_fp8.h - C ABI of the 8-bit projections around the hybrid attention, for NVIDIA B200 (sm_100a).
 *
 * A converted layer's attention stands between linear layers with frozen weights: the projections of queries, keys and
 * values ahead of it, the output projection behind it.  These calls run them in 8 bits on the tensor cores:
 *
 *   as_rms_norm       t = x + residual,  y = t * rsqrt(mean(t^2) + eps) * weight     (and t itself, the new residual)
 *   as_quantize_fp8   the 8-bit form of a matrix that is there already (attention's output, weights)
 *   as_matmul_fp8     out = a w^T + bias of two matrices in 8-bit form
 *
 * The 8-bit form of a matrix [rows, cols]: e4m3 values q and one scale 2^e for every 128 columns of a row (of 128 rows,
 * where weights are quantised); element (r, c) stands for q[r, c] * 2^e[r, c / 128], and
 *
 *   e = the smallest whole number with max |y| <= 448 * 2^e over the block (448: the largest e4m3 value), at least -127.
 *
 * A scale that is a power of two costs an 8-bit floating type no accuracy, its product with a value is exact, and the
 * tensor cores take it as it is.  A block that holds an infinity or NaN has the scale NaN (byte 255).
 *
 * Conventions (as in as_hybrid_attn.h): tensor pointers are DEVICE pointers; the caller owns every buffer and the stream;
 * every call is asynchronous on it, allocates nothing, does not synchronise, and can be captured into a graph; nothing
 * aborts and no kernel traps.  On error nothing has been launched and the outputs are untouched.  Sums are fp32, in an order
 * that depends on the sizes alone: results are run-to-run identical.  These operators serve a model whose weights stay as they are: there are
 * no gradients (the value distillation of a layer takes q, k, v and the teacher's output as constants).
 */
#ifndef AS_FP8_H_
#define AS_FP8_H_

#include "as_hybrid_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { AS_DTYPE_BF16 = 0, AS_DTYPE_F32 = 1 };

/* A matrix [rows, cols] as it lies in memory.  Row r is token r % tokens of batch entry r / tokens; column c is column
 * c % head_dim of head c / head_dim:
 *
 *   address = data + (r / tokens) * stride_batch + (c / head_dim) * stride_head + (r % tokens) * stride_token + c % head_dim
 *
 * in elements.  [rows, cols] with a row stride: tokens = rows, head_dim = cols.  The attention's [B, H, N, d]: tokens = N,
 * head_dim = d, its strides.  tokens divides rows and head_dim divides cols; strides are not negative, and those of an output
 * keep its elements apart; an output shares no memory with another one, nor with an input in another layout.  data == NULL: no
 * such matrix.  Where head_dim, the strides and the address are all multiples of 8 elements (16 bytes), rows move 16 bytes at a
 * time; otherwise element by element. */
typedef struct {
  void* data;
  int32_t dtype;            /* AS_DTYPE_BF16 | AS_DTYPE_F32 */
  int32_t head_dim;
  int64_t tokens;
  int64_t stride_batch, stride_head, stride_token;
} as_rows_t;

/* A matrix in 8-bit form. */
typedef struct {
  void* data;               /* e4m3 [rows][pitch], 16-byte aligned; columns cols .. pitch-1 are neither read nor written     */
  int64_t pitch;            /* bytes from row to row, a multiple of 16, >= cols                                               */
  void* scales;             /* uint8 [ceil(cols / 512)][scale_rows][4], 4-byte aligned: byte k % 4 of [k / 4][r] is e + 127 of
                               row r, columns 128 k .. 128 k + 127; bytes behind the last block are written as 0, not read    */
  int64_t scale_rows;       /* >= rows                                                                                        */
} as_fp8_matrix_t;

typedef struct {
  uint32_t struct_size;     /* sizeof(as_rms_norm_t) */
  int32_t cols;             /* 1 .. 16384 */
  int64_t rows;             /* 0 .. 2^31 - 1 */
  as_rows_t x;              /* bf16 or fp32 */
  as_rows_t residual;       /* optional (data == NULL: t = x); bf16 or fp32; with x in fp32: fp32 */
  as_rows_t residual_out;   /* t in the residual's type; required with a residual (may be the residual itself), NULL without */
  as_rows_t out;            /* y in bf16, or NULL */
  as_fp8_matrix_t out8;     /* y in 8-bit form, a scale for each row and 128 columns, or data == NULL; exactly one of the two */
  const void* weight;       /* [cols], or NULL for ones */
  int32_t weight_dtype;
  float eps;                /* >= 0 */
} as_rms_norm_t;

typedef struct {
  uint32_t struct_size;     /* sizeof(as_quantize_fp8_t) */
  int32_t cols;             /* 1 .. 16384 */
  int64_t rows;             /* 0 .. 2^31 - 1; with block_rows == 128 up to 65535 * 128 */
  as_rows_t x;              /* bf16 or fp32 */
  as_fp8_matrix_t out;
  int32_t block_rows;       /* rows that share a scale: 1 (activations) or 128 (weights) */
  int32_t reserved;         /* 0 */
} as_quantize_fp8_t;

typedef struct {
  uint32_t struct_size;     /* sizeof(as_matmul_fp8_t) */
  int32_t cols;             /* K, 1 .. 2^20 */
  int64_t rows;             /* M, 0 .. 2^30 */
  int64_t out_cols;         /* N, 1 .. 2^24 */
  as_fp8_matrix_t a;        /* [M, K] */
  as_fp8_matrix_t w;        /* [N, K] */
  const void* bias;         /* [N] bf16, 2-byte aligned, or NULL */
  as_rows_t out;            /* [M, N] bf16; heads that lie apart: N * head_dim up to 2^32 */
} as_matmul_fp8_t;

/* t = x + residual in fp32; y = t * rsqrt(mean(t^2) + eps) * weight from the unrounded t; t is rounded once into residual_out, y
 * once into out or out8.  Holds for every finite t and every y within the output's range, whatever their squares or t * weight are in fp32; a row of
 * zeros with eps == 0 is NaN, as in the formula.  rows == 0 launches nothing. */
AS_API as_status_t as_rms_norm(const as_rms_norm_t* args, void* cuda_stream);

/* The 8-bit form of x. */
AS_API as_status_t as_quantize_fp8(const as_quantize_fp8_t* args, void* cuda_stream);

/* What as_matmul_fp8 keeps on a device: the status word of its bounded waits.  Create it on the device that the calls run on
 * (AS_ERR_ARCH when that is not sm_100); calls that use one context may overlap. */
typedef struct as_fp8_context_s* as_fp8_context_t;
AS_API as_status_t as_fp8_create(as_fp8_context_t* out);
AS_API as_status_t as_fp8_destroy(as_fp8_context_t ctx);

/* Synchronises the stream, then reads and clears the context's status word: AS_OK, AS_ERR_DEVICE_TIMEOUT (a wait inside a
 * product since the last read ran out: that product's output is undefined, the context stays usable and later calls run) or
 * AS_ERR_CUDA. */
AS_API as_status_t as_fp8_last_status(as_fp8_context_t ctx, void* cuda_stream);

/* Test aid: enqueues a one-CTA kernel whose bounded wait, the one that the products use, runs out after about limit_cycles SM clocks
 * (1 .. 1e8) and sets the context's status word as a time-out inside a product does; no copy and no tensor-core operation is in
 * flight.  Like the products it lets the launch behind it set up before it waits. */
AS_API as_status_t as_fp8_debug_expire_wait(as_fp8_context_t ctx, int64_t limit_cycles, void* cuda_stream);

/* out[m, n] = sum_k a[m, k] w[n, k] + bias[n], products of the 8-bit values times both scales, summed in fp32, rounded once to
 * bf16.  A scale byte of 255 makes the row's (column's) results NaN.  rows == 0 launches nothing. */
AS_API as_status_t as_matmul_fp8(as_fp8_context_t ctx, const as_matmul_fp8_t* args, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif  /* AS_FP8_H_ */
