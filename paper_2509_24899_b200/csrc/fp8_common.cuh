// Pieces shared by the kernels of the 8-bit projections: addresses of a matrix in rows or heads, and the e4m3 form with a
// power-of-two scale for every 128 columns.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "as_fp8.h"
#include "as_internal.h"
#include "sm100_ptx.cuh"

namespace as_fp8 {

// as_rows_t as the kernels use it: c / head_dim is a product with ceil(2^32 / head_dim), exact for c and head_dim below 2^16
// (c * (head_dim - 1) < 2^32); wider matrices without heads have head_dim == cols, where `split` is false and nothing is divided.
struct Rows {
  void* data;
  long long sb, sh, st;
  unsigned tokens;
  int hd;
  unsigned long long magic;
  bool split, batched;

  __device__ __forceinline__ long long row(unsigned r) const {
    if (!batched) return (long long)r * st;
    const unsigned b = r / tokens;
    return (long long)b * sb + (long long)(r - b * tokens) * st;
  }
  __device__ __forceinline__ long long col(unsigned c) const {
    if (!split) return c;
    const unsigned h = (unsigned)((c * magic) >> 32);
    return (long long)h * sh + (c - h * (unsigned)hd);
  }
};

// ---------------------------------------------------------------- host: checks, and the form above
// What a call returns when one of CUDA's has failed; the error does not stay behind for the library's next launch, which would report it as its own.
inline as_status_t failed(as_status_t status = AS_ERR_CUDA) { cudaGetLastError(); return status; }

inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline bool rows_ok(const as_rows_t& x, long long rows, long long cols) {
  if (x.data == nullptr || (x.dtype != AS_DTYPE_BF16 && x.dtype != AS_DTYPE_F32)) return false;
  if (!aligned(x.data, x.dtype == AS_DTYPE_BF16 ? 2 : 4)) return false;
  if (x.head_dim <= 0 || cols % x.head_dim != 0) return false;
  if (rows > 0 && (x.tokens <= 0 || rows % x.tokens != 0)) return false;
  return x.stride_batch >= 0 && x.stride_head >= 0 && x.stride_token >= 0;
}

// Whether no two elements of an output share an address, by the strides that are in use: sorted by size, each is at least as long
// as all that lies within it.
inline bool apart(const as_rows_t& x, long long rows, long long cols) {
  struct Dim { __int128 n, s; } d[3] = {{cols / x.head_dim, x.stride_head}, {x.tokens, x.stride_token}, {x.tokens > 0 ? rows / x.tokens : 0, x.stride_batch}};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (d[j].s > d[j + 1].s) { const Dim t = d[j]; d[j] = d[j + 1]; d[j + 1] = t; }
  __int128 span = x.head_dim;                                // elements from the first to the last one, both counted
  for (const Dim& e : d) {
    if (e.n <= 1) continue;
    if (e.s < span) return false;
    span += (e.n - 1) * e.s;
  }
  return true;
}

// Whether an output at an input's address is that input itself, element by element; elsewhere it is taken to lie apart from it.
inline bool in_place_ok(const as_rows_t& out, const as_rows_t& in, long long rows, long long cols) {
  if (out.data != in.data || out.data == nullptr || rows == 0) return true;
  return out.dtype == in.dtype && out.head_dim == in.head_dim && out.tokens == in.tokens && (out.tokens == 1 || out.stride_token == in.stride_token) &&
         (cols == out.head_dim || out.stride_head == in.stride_head) && (rows == out.tokens || out.stride_batch == in.stride_batch);
}

// Whether rows can move `bytes` at a time (16, 32), with 8 or 16 bf16 columns: address, strides and heads are multiples of as much.
inline bool rows_vec(const as_rows_t& x, int bytes) {
  return aligned(x.data, bytes) && ((x.head_dim | x.stride_batch | x.stride_head | x.stride_token) & (bytes / 2 - 1)) == 0;
}

inline Rows rows_of(const as_rows_t& x, long long rows, long long cols) {
  Rows r{};
  r.data = x.data;
  r.sb = x.stride_batch; r.sh = x.stride_head; r.st = x.stride_token;
  r.tokens = (unsigned)x.tokens;
  r.hd = x.head_dim;
  r.magic = ((1ull << 32) + x.head_dim - 1) / x.head_dim;
  r.split = x.head_dim != cols && x.stride_head != x.head_dim;
  r.batched = x.tokens != rows;
  return r;
}

inline bool matrix_ok(const as_fp8_matrix_t& m, long long rows, long long cols) {
  return m.data != nullptr && m.scales != nullptr && aligned(m.data, 16) && aligned(m.scales, 4) && m.pitch >= cols && m.pitch % 16 == 0 && m.scale_rows >= rows;
}

// ---------------------------------------------------------------- device: the 8-bit form
// The scale's byte e + 127 from the bits of a block's largest |y| = 1.m * 2^(E - 127): 448 = 1.75 * 2^8, so e + 127 = E - 8, and one more where
// 1.m > 1.75, which is where adding 2^21 - 1 to the bits carries into the exponent.  Infinity and NaN: 255.  Below 2^-119: 0.
AS_DEV uint32_t scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return 255u;
  const int e = (int)((amax_bits + 0x1fffffu) >> 23) - 8;
  return (uint32_t)max(e, 0);
}
// 2^-e (NaN for the byte 255).
AS_DEV float inverse_scale(uint32_t byte) { return __uint_as_float(byte == 255u ? 0x7fc00000u : (254u - byte) << 23); }

// Two values as e4m3, round to nearest even, lo in the low byte.
AS_DEV uint32_t pack_e4m3(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

}  // namespace as_fp8
