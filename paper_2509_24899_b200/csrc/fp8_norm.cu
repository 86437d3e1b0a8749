// Root-mean-square norm with the residual's addition, and the 8-bit form of a matrix.
//
// Both read a row once, keep it in registers and write it once: bound by HBM bytes.  A row belongs to W warps (one up to 2048 columns), a lane holds
// NV vectors of 8 columns, and a block of 128 columns lies in half a warp's vector (where rows move 16 bytes at a time) or in four of a warp's
// 32-column runs (where they move element by element): its largest value is a shuffle away, and so is the sum of squares.
#include "fp8_common.cuh"

namespace {

using namespace as_fp8;
using sm100::griddep_launch;
using sm100::griddep_wait;

constexpr int THREADS = 256;

struct NormParams {
  Rows x, r, ro, o;                        // x, residual, t rounded, y in bf16
  uint8_t* q;
  uint8_t* scales;
  long long pitch, scale_rows;
  const void* w;
  bool w_f32;
  float eps;
  int rows, cols, W;                       // W: warps of a row
};


// Pairs of fp32 values, added and multiplied two at a time.
AS_DEV float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
AS_DEV float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
AS_DEV float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// The largest of |a|, |b|, |c|; NaN if one of them is.
AS_DEV float max_abs(float a, float b, float c) {
  float d;
  asm("{\n\t.reg .f32 x, y, z;\n\tabs.f32 x, %1;\n\tabs.f32 y, %2;\n\tabs.f32 z, %3;\n\tmax.NaN.f32 %0, x, y, z;\n\t}" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// 8 elements of a row as they come: a vector where VEC, else elements 32 columns apart, 0 where there is no column.
template <typename T, bool VEC> struct Raw { T e[8]; };
template <> struct Raw<__nv_bfloat16, true> { uint4 a; };
template <> struct Raw<float, true> { float4 a, b; };

template <typename T, bool VEC>
AS_DEV void fetch(const Rows& m, long long row, int c0, int cols, Raw<T, VEC>& v) {
  const T* base = static_cast<const T*>(m.data) + row;
  if constexpr (VEC) {
    v = Raw<T, VEC>{};
    if (c0 < cols) {
      const T* at = base + m.col(c0);
      if constexpr (sizeof(T) == 2) v.a = *reinterpret_cast<const uint4*>(at);
      else { v.a = *reinterpret_cast<const float4*>(at); v.b = *reinterpret_cast<const float4*>(at + 4); }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = c0 + 32 * i;
      v.e[i] = c < cols ? base[m.col(c)] : (T)0.f;
    }
  }
}
template <typename T, bool VEC>
AS_DEV void values(const Raw<T, VEC>& v, float2 (&f)[4]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2((float)v.e[2 * i], (float)v.e[2 * i + 1]);
  } else if constexpr (sizeof(T) == 2) {
    const uint32_t w[4] = {v.a.x, v.a.y, v.a.z, v.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  } else {
    f[0] = make_float2(v.a.x, v.a.y); f[1] = make_float2(v.a.z, v.a.w); f[2] = make_float2(v.b.x, v.b.y); f[3] = make_float2(v.b.z, v.b.w);
  }
}
template <typename T, bool VEC>
AS_DEV void load8(const Rows& m, long long row, int c0, int cols, float2 (&f)[4]) {
  Raw<T, VEC> v;
  fetch<T, VEC>(m, row, c0, cols, v);
  values<T, VEC>(v, f);
}

template <typename T, bool VEC>
AS_DEV void store8(const Rows& m, long long row, int c0, int cols, const float2 (&v)[4]) {
  T* base = static_cast<T*>(m.data) + row;
  if constexpr (VEC) {
    if (c0 >= cols) return;
    T* at = base + m.col(c0);
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4*>(at) = make_uint4(sm100::pack_bf16(v[0].x, v[0].y), sm100::pack_bf16(v[1].x, v[1].y), sm100::pack_bf16(v[2].x, v[2].y), sm100::pack_bf16(v[3].x, v[3].y));
    } else {
      *reinterpret_cast<float4*>(at) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
      *reinterpret_cast<float4*>(at + 4) = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = c0 + 32 * i;
      const float f = i % 2 ? v[i / 2].y : v[i / 2].x;
      if (c >= cols) continue;
      if constexpr (sizeof(T) == 2) base[m.col(c)] = __float2bfloat16_rn(f);
      else base[m.col(c)] = f;
    }
  }
}

// The largest |value| of each of the two blocks of 128 columns in a warp's vector, as bits (NaN is above infinity), for every lane.
template <bool VEC>
AS_DEV void block_max(const float2 (&v)[4], int lane, uint32_t (&top)[2]) {
  const float lo = max_abs(v[0].x, v[0].y, v[1].x), hi = max_abs(v[2].x, v[2].y, v[3].x);
  if constexpr (VEC) {                        // lanes 0-15 hold the first one
    const uint32_t t = __float_as_uint(max_abs(max_abs(lo, v[1].y, v[3].y), hi, 0.f));
    top[0] = __reduce_max_sync(0xffffffffu, lane < 16 ? t : 0u);
    top[1] = __reduce_max_sync(0xffffffffu, lane < 16 ? 0u : t);
  } else {                                    // every lane holds four values of each
    top[0] = __reduce_max_sync(0xffffffffu, __float_as_uint(max_abs(lo, v[1].y, 0.f)));
    top[1] = __reduce_max_sync(0xffffffffu, __float_as_uint(max_abs(hi, v[3].y, 0.f)));
  }
}

// NORM: y = t * rsqrt(mean t^2 + eps) * w, else y = x.  R: the residual's type (void: none).  FP8: y in 8-bit form, else in bf16.
//
// The weights multiply t while the sum of squares is on its way between the lanes, and so do the blocks' largest values go round: both turns of a row's reductions
// overlap, and the row's scale enters last.  (In the formula's order, with one value an instruction, a row took 850 instructions instead of 450 and the norm of 32760 x 1536
// with a residual in bf16 131 us: the arithmetic, not memory, was the bound.)
template <typename X, typename R, bool NORM, bool FP8, bool VEC, int NV>
__global__ void __launch_bounds__(THREADS) norm_kernel(const __grid_constant__ NormParams p) {
  griddep_launch();
  __shared__ float part[THREADS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (THREADS / 32) / p.W;                       // rows of a CTA
  const int slot = warp / p.W, piece = warp - slot * p.W;
  const long long row = (long long)blockIdx.x * per + slot;
  const bool live = slot < per && row < p.rows;
  const unsigned r = live ? (unsigned)row : 0u;
  const int cols = live ? p.cols : 0;                         // of a row that is not there nothing is read or written
  const int first = piece * (NV * 256);                       // columns of this warp
  const int c0 = first + (VEC ? lane * 8 : lane);
  float2 v[NV][4];
  griddep_wait();
  {
    Raw<X, VEC> x[NV];
    const long long xr = p.x.row(r);
#pragma unroll
    for (int j = 0; j < NV; ++j) fetch<X, VEC>(p.x, xr, c0 + j * 256, cols, x[j]);
    if constexpr (!__is_same(R, void)) {
      Raw<R, VEC> t[NV];
      const long long rr = p.r.row(r), wr = p.ro.row(r);
#pragma unroll
      for (int j = 0; j < NV; ++j) fetch<R, VEC>(p.r, rr, c0 + j * 256, cols, t[j]);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float2 u[4];
        values<X, VEC>(x[j], v[j]);
        values<R, VEC>(t[j], u);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j][i] = add2(v[j][i], u[i]);
        store8<R, VEC>(p.ro, wr, c0 + j * 256, cols, v[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) values<X, VEC>(x[j], v[j]);
    }
  }
  float scale = 1.f;
  float2 sum2 = make_float2(0.f, 0.f);
  if constexpr (NORM) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum2 = fma2(v[j][i], v[j][i], sum2);
    if (p.w != nullptr) {
      Rows m{};
      m.data = const_cast<void*>(p.w);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float2 w[4];
        if (p.w_f32) load8<float, VEC>(m, 0, c0 + j * 256, cols, w);
        else load8<__nv_bfloat16, VEC>(m, 0, c0 + j * 256, cols, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j][i] = mul2(v[j][i], w[i]);
      }
    }
  }
  uint32_t top[NV][2];
  if constexpr (FP8) {
#pragma unroll
    for (int j = 0; j < NV; ++j) block_max<VEC>(v[j], lane, top[j]);
  }
  if constexpr (NORM) {
    float sum = sum2.x + sum2.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (p.W > 1) {                                            // the same for every thread of the launch
      if (lane == 0) part[warp] = sum;
      __syncthreads();
      sum = 0.f;
      for (int i = 0; i < p.W; ++i) sum += part[min(slot * p.W + i, THREADS / 32 - 1)];
    }
    scale = rsqrtf(sum / (float)p.cols + p.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[j][i] = mul2(v[j][i], make_float2(scale, scale));
  }
  if (!live) return;
  if constexpr (!FP8) {
    const long long wr = p.o.row(r);
#pragma unroll
    for (int j = 0; j < NV; ++j) store8<__nv_bfloat16, VEC>(p.o, wr, c0 + j * 256, cols, v[j]);
  } else {
    uint8_t* q = p.q + (long long)r * p.pitch;
    uint32_t pair[NV];                                        // the bytes of a vector's two blocks, the first one's in the low byte
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + j * 256;
      uint32_t byte[2];
      float inv[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if constexpr (NORM) top[j][b] = __float_as_uint(__uint_as_float(top[j][b]) * scale);
        byte[b] = scale_byte(top[j][b]);
        inv[b] = inverse_scale(byte[b]);
      }
      if constexpr (VEC) {
        const float f = lane < 16 ? inv[0] : inv[1];
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 y = mul2(v[j][i], make_float2(f, f)); w[i] = pack_e4m3(y.x, y.y); }
        if (c < cols) *reinterpret_cast<uint2*>(q + c) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + 32 * i < cols) q[c + 32 * i] = (uint8_t)pack_e4m3((i % 2 ? v[j][i / 2].y : v[j][i / 2].x) * inv[i / 4], 0.f);
      }
      // blocks behind the last column keep the byte 0
      const int k = first + j * 256;
      pair[j] = k + 128 < p.cols ? byte[0] | byte[1] << 8 : k < p.cols ? byte[0] : 0u;
    }
    // four blocks' bytes are a word: lane g writes the one of this warp's group g
#pragma unroll
    for (int g = 0; g < (NV + 1) / 2; ++g) {
      const uint32_t word = pair[2 * g] | (2 * g + 1 < NV ? pair[2 * g + 1] << 16 : 0u);
      const long long group = first / 512 + g;
      if (lane == g && 512 * group < p.cols) *reinterpret_cast<uint32_t*>(p.scales + (group * p.scale_rows + r) * 4) = word;
    }
  }
}

// A scale for 128 rows and 128 columns: a CTA per block, a thread's 64 elements in registers.  VEC: 16 lanes a row and 16 bytes a lane; else a warp
// a row and an element a lane.  The CTA of a group's last block writes the bytes behind it as well.
template <typename X, bool VEC>
__global__ void __launch_bounds__(THREADS) quantize_block_kernel(const __grid_constant__ NormParams p) {
  griddep_launch();
  __shared__ uint32_t part[THREADS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = blockIdx.x * 128, row0 = blockIdx.y * 128;
  float2 v[8][4];
  uint32_t top = 0u;
  griddep_wait();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (VEC) {
      const int row = row0 + j * 16 + warp * 2 + lane / 16;
      load8<X, true>(p.x, row < p.rows ? p.x.row(row) : 0, c0 + lane % 16 * 8, row < p.rows ? p.cols : 0, v[j]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = row0 + warp * 16 + j * 2 + i / 4, c = c0 + i % 4 * 32 + lane;
        const float f = row < p.rows && c < p.cols ? (float)static_cast<const X*>(p.x.data)[p.x.row(row) + p.x.col(c)] : 0.f;
        if (i % 2) v[j][i / 2].y = f; else v[j][i / 2].x = f;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(max_abs(v[j][i].x, v[j][i].y, 0.f)));
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if (lane == 0) part[warp] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < THREADS / 32; ++i) top = max(top, part[i]);
  const uint32_t byte = scale_byte(top);
  const float inv = inverse_scale(byte);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (VEC) {
      const int row = row0 + j * 16 + warp * 2 + lane / 16, c = c0 + lane % 16 * 8;
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pack_e4m3(v[j][i].x * inv, v[j][i].y * inv);
      if (row < p.rows && c < p.cols) *reinterpret_cast<uint2*>(p.q + (long long)row * p.pitch + c) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = row0 + warp * 16 + j * 2 + i / 4, c = c0 + i % 4 * 32 + lane;
        if (row < p.rows && c < p.cols) p.q[(long long)row * p.pitch + c] = (uint8_t)pack_e4m3((i % 2 ? v[j][i / 2].y : v[j][i / 2].x) * inv, 0.f);
      }
    }
  }
  if (threadIdx.x < 128 && row0 + (int)threadIdx.x < p.rows) {
    uint8_t* at = p.scales + ((long long)(blockIdx.x / 4) * p.scale_rows + row0 + threadIdx.x) * 4;
    at[blockIdx.x % 4] = (uint8_t)byte;
    if (blockIdx.x + 1 == gridDim.x)
      for (int k = blockIdx.x % 4 + 1; k < 4; ++k) at[k] = 0;
  }
}

// Warps of a row and vectors of a lane: one warp up to 2048 columns (a row then needs no barrier), then as many as keep 8 vectors a lane.  An odd number
// of vectors is only used with one warp: a warp's columns begin with a group of scales.
struct Split { int W, NV; };
Split split_of(int cols) {
  const int W = (cols + 2047) / 2048, need = (cols + 256 * W - 1) / (256 * W);
  if (W == 1 && need == 1) return {1, 1};
  return {W, (need + 1) / 2 * 2};
}

template <typename X, typename R, bool NORM, bool FP8, bool VEC>
cudaError_t launch_rows(const NormParams& p, int NV, cudaStream_t st) {
  const long long per = (THREADS / 32) / p.W;
  const dim3 grid((unsigned)((p.rows + per - 1) / per));
  if constexpr (!VEC) {
    // element by element: fewer forms, the columns that are not there cost only their comparison
    if (p.W == 1 && NV <= 2) return as_launch_dependent(norm_kernel<X, R, NORM, FP8, VEC, 2>, grid, dim3(THREADS), 0, st, p);
    if (p.W == 1 && NV <= 4) return as_launch_dependent(norm_kernel<X, R, NORM, FP8, VEC, 4>, grid, dim3(THREADS), 0, st, p);
    return as_launch_dependent(norm_kernel<X, R, NORM, FP8, VEC, 8>, grid, dim3(THREADS), 0, st, p);
  } else {
    switch (NV) {
      case 1: return as_launch_dependent(norm_kernel<X, R, NORM, FP8, VEC, 1>, grid, dim3(THREADS), 0, st, p);
      case 2: return as_launch_dependent(norm_kernel<X, R, NORM, FP8, VEC, 2>, grid, dim3(THREADS), 0, st, p);
      case 4: return as_launch_dependent(norm_kernel<X, R, NORM, FP8, VEC, 4>, grid, dim3(THREADS), 0, st, p);
      case 6: return as_launch_dependent(norm_kernel<X, R, NORM, FP8, VEC, 6>, grid, dim3(THREADS), 0, st, p);
      default: return as_launch_dependent(norm_kernel<X, R, NORM, FP8, VEC, 8>, grid, dim3(THREADS), 0, st, p);
    }
  }
}

template <typename X, typename R, bool NORM>
cudaError_t launch_out(const NormParams& p, bool fp8, bool vec, int NV, cudaStream_t st) {
  if constexpr (NORM)
    if (!fp8) return vec ? launch_rows<X, R, NORM, false, true>(p, NV, st) : launch_rows<X, R, NORM, false, false>(p, NV, st);
  return vec ? launch_rows<X, R, NORM, true, true>(p, NV, st) : launch_rows<X, R, NORM, true, false>(p, NV, st);
}

as_status_t arch_ok() {
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return AS_ERR_CUDA;
  return major == 10 ? AS_OK : AS_ERR_ARCH;
}

}  // namespace

extern "C" as_status_t as_rms_norm(const as_rms_norm_t* a, void* cuda_stream) {
  if (a == nullptr || a->struct_size != sizeof(as_rms_norm_t)) return AS_ERR_INVALID_ARG;
  if (a->cols < 1 || a->rows < 0 || a->rows > 0x7fffffffll || !(a->eps >= 0.f)) return AS_ERR_INVALID_ARG;
  if (a->weight != nullptr && ((a->weight_dtype != AS_DTYPE_BF16 && a->weight_dtype != AS_DTYPE_F32) || !aligned(a->weight, a->weight_dtype == AS_DTYPE_BF16 ? 2 : 4)))
    return AS_ERR_INVALID_ARG;
  const bool res = a->residual.data != nullptr, fp8 = a->out8.data != nullptr;
  if (!rows_ok(a->x, a->rows, a->cols) || fp8 == (a->out.data != nullptr) || res != (a->residual_out.data != nullptr)) return AS_ERR_INVALID_ARG;
  if (fp8 ? !matrix_ok(a->out8, a->rows, a->cols) : !(rows_ok(a->out, a->rows, a->cols) && a->out.dtype == AS_DTYPE_BF16 && apart(a->out, a->rows, a->cols)))
    return AS_ERR_INVALID_ARG;
  if (res && !(rows_ok(a->residual, a->rows, a->cols) && rows_ok(a->residual_out, a->rows, a->cols) && a->residual.dtype == a->residual_out.dtype &&
               apart(a->residual_out, a->rows, a->cols)))
    return AS_ERR_INVALID_ARG;
  if (a->cols > 16384 || (res && a->x.dtype == AS_DTYPE_F32 && a->residual.dtype == AS_DTYPE_BF16)) return AS_ERR_UNSUPPORTED;
  if (a->rows == 0) return AS_OK;
  if (const as_status_t s = arch_ok(); s != AS_OK) return s;
  NormParams p{};
  p.rows = (int)a->rows; p.cols = a->cols; p.eps = a->eps;
  p.x = rows_of(a->x, a->rows, a->cols);
  bool vec = rows_vec(a->x) && (a->weight == nullptr || aligned(a->weight, 16));
  if (res) {
    p.r = rows_of(a->residual, a->rows, a->cols);
    p.ro = rows_of(a->residual_out, a->rows, a->cols);
    vec = vec && rows_vec(a->residual) && rows_vec(a->residual_out);
  }
  if (fp8) {
    p.q = static_cast<uint8_t*>(a->out8.data); p.pitch = a->out8.pitch;
    p.scales = static_cast<uint8_t*>(a->out8.scales); p.scale_rows = a->out8.scale_rows;
  } else {
    p.o = rows_of(a->out, a->rows, a->cols);
    vec = vec && rows_vec(a->out);
  }
  p.w = a->weight; p.w_f32 = a->weight_dtype == AS_DTYPE_F32;
  const Split s = split_of(a->cols);
  p.W = s.W;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  typedef __nv_bfloat16 bf;
  if (a->x.dtype == AS_DTYPE_F32) e = res ? launch_out<float, float, true>(p, fp8, vec, s.NV, st) : launch_out<float, void, true>(p, fp8, vec, s.NV, st);
  else if (!res) e = launch_out<bf, void, true>(p, fp8, vec, s.NV, st);
  else e = a->residual.dtype == AS_DTYPE_BF16 ? launch_out<bf, bf, true>(p, fp8, vec, s.NV, st) : launch_out<bf, float, true>(p, fp8, vec, s.NV, st);
  return e == cudaSuccess ? AS_OK : AS_ERR_CUDA;
}

extern "C" as_status_t as_quantize_fp8(const as_quantize_fp8_t* a, void* cuda_stream) {
  if (a == nullptr || a->struct_size != sizeof(as_quantize_fp8_t) || a->reserved != 0) return AS_ERR_INVALID_ARG;
  if (a->cols < 1 || a->rows < 0 || a->rows > 0x7fffffffll || (a->block_rows != 1 && a->block_rows != 128)) return AS_ERR_INVALID_ARG;
  if (!rows_ok(a->x, a->rows, a->cols) || !matrix_ok(a->out, a->rows, a->cols)) return AS_ERR_INVALID_ARG;
  if (a->cols > 16384 || (a->block_rows == 128 && a->rows > 65535ll * 128)) return AS_ERR_UNSUPPORTED;
  if (a->rows == 0) return AS_OK;
  if (const as_status_t s = arch_ok(); s != AS_OK) return s;
  NormParams p{};
  p.rows = (int)a->rows; p.cols = a->cols;
  p.x = rows_of(a->x, a->rows, a->cols);
  p.q = static_cast<uint8_t*>(a->out.data); p.pitch = a->out.pitch;
  p.scales = static_cast<uint8_t*>(a->out.scales); p.scale_rows = a->out.scale_rows;
  const bool vec = rows_vec(a->x), f32 = a->x.dtype == AS_DTYPE_F32;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  typedef __nv_bfloat16 bf;
  if (a->block_rows == 1) {
    const Split s = split_of(a->cols);
    p.W = s.W;
    e = f32 ? launch_out<float, void, false>(p, true, vec, s.NV, st) : launch_out<bf, void, false>(p, true, vec, s.NV, st);
  } else {
    const dim3 grid((unsigned)((a->cols + 127) / 128), (unsigned)((a->rows + 127) / 128));
    e = f32 ? (vec ? as_launch_dependent(quantize_block_kernel<float, true>, grid, dim3(THREADS), 0, st, p) : as_launch_dependent(quantize_block_kernel<float, false>, grid, dim3(THREADS), 0, st, p))
            : (vec ? as_launch_dependent(quantize_block_kernel<bf, true>, grid, dim3(THREADS), 0, st, p) : as_launch_dependent(quantize_block_kernel<bf, false>, grid, dim3(THREADS), 0, st, p));
  }
  return e == cudaSuccess ? AS_OK : AS_ERR_CUDA;
}
