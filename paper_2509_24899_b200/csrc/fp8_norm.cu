// Root-mean-square norm with the residual's addition, and the 8-bit form of a matrix.
//
// Both read a row once, keep it in registers and write it once: bound by HBM bytes, with the arithmetic of unpacking, scaling and packing close behind.
// A lane holds NV vectors of 16 columns, 8 lanes a block of 128 columns, a warp's vector a group of four blocks, whose scales are one word.  A row has 8 or
// 16 lanes where that is enough (up to 128 or 256 columns: norms of single heads), else one warp up to 1536 columns, which needs no barrier, else W warps.
//
// MOVE says how rows move: 32 or 16 bytes an instruction, by what all addresses and strides of the call allow, or 2: element by element, where a lane's 16 columns are 32
// apart, so that a warp's access is one run, and every lane holds four columns of each block.
#include <algorithm>

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
  int sms;
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
// The largest of both |a| and c >= 0; NaN if one of them is.
AS_DEV float max_abs2(float2 a, float c) {
  float d;
  asm("{\n\t.reg .f32 x, y;\n\tabs.f32 x, %1;\n\tabs.f32 y, %2;\n\tmax.NaN.f32 %0, x, y, %3;\n\t}" : "=f"(d) : "f"(a.x), "f"(a.y), "f"(c));
  return d;
}

constexpr int MOVE32 = 0, MOVE16 = 1, MOVE_ELEMENT = 2;      // the slower, the larger

AS_DEV void load32(const void* at, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(at) : "memory");
}
AS_DEV void store32(void* at, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

// 16 columns of a row as they come, from c0 on (or c0, c0 + 32, ...), 0 where there is no column.
template <typename T, int MOVE> struct Raw { uint32_t w[4 * sizeof(T)]; };
template <typename T> struct Raw<T, MOVE_ELEMENT> { T e[16]; };

// SPLIT: whether columns may belong to heads that lie apart.  It is asked once for all loads of a row: asked at each, element by element the loads waited for one another
// (32760 x 1537 with a residual 197 us, so 117), and vectors did a little (7800 x 1536 with a residual 16.8, 16.2).
template <typename T, int MOVE, bool SPLIT = true>
AS_DEV void fetch(const Rows& m, long long row, int c0, int cols, Raw<T, MOVE>& v) {
  const T* base = static_cast<const T*>(m.data) + row;
  if constexpr (MOVE == MOVE_ELEMENT) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int c = c0 + 32 * i;
      v.e[i] = c < cols ? base[SPLIT ? m.col(c) : c] : (T)0.f;
    }
  } else {
    v = Raw<T, MOVE>{};
    if constexpr (MOVE == MOVE32) {           // head_dim and cols are multiples of 16
      if (c0 < cols) {
        const T* at = base + (SPLIT ? m.col(c0) : c0);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) load32(reinterpret_cast<const uint8_t*>(at) + 32 * i, reinterpret_cast<uint32_t(&)[8]>(v.w[8 * i]));
      }
    } else {                                  // of 8
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (c0 + 8 * h < cols) {
          const uint4* at = reinterpret_cast<const uint4*>(base + (SPLIT ? m.col(c0 + 8 * h) : c0 + 8 * h));
#pragma unroll
          for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(v.w)[h * (int)sizeof(T) / 2 + i] = at[i];
        }
    }
  }
}
// All vectors of a row, 512 columns apart.
template <typename T, int MOVE, int NV>
AS_DEV void fetch_row(const Rows& m, long long row, int c0, int cols, Raw<T, MOVE> (&v)[NV]) {
  if ((MOVE == MOVE_ELEMENT || NV > 1) && !m.split) {
#pragma unroll
    for (int j = 0; j < NV; ++j) fetch<T, MOVE, false>(m, row, c0 + j * 512, cols, v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) fetch<T, MOVE, true>(m, row, c0 + j * 512, cols, v[j]);
  }
}
template <typename T, int MOVE>
AS_DEV void values(const Raw<T, MOVE>& v, float2 (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (MOVE == MOVE_ELEMENT) f[i] = make_float2((float)v.e[2 * i], (float)v.e[2 * i + 1]);
    else if constexpr (sizeof(T) == 2) f[i] = make_float2(__uint_as_float(v.w[i] << 16), __uint_as_float(v.w[i] & 0xffff0000u));
    else f[i] = make_float2(__uint_as_float(v.w[2 * i]), __uint_as_float(v.w[2 * i + 1]));
  }
}
// f += v
template <typename T, int MOVE>
AS_DEV void add_values(const Raw<T, MOVE>& v, float2 (&f)[8]) {
  if constexpr (MOVE != MOVE_ELEMENT && sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sm100::add_bf16x2(f[i].x, f[i].y, v.w[i]);
  } else {
    float2 u[8];
    values<T, MOVE>(v, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = add2(f[i], u[i]);
  }
}
// f *= v
template <typename T, int MOVE>
AS_DEV void scale_values(const Raw<T, MOVE>& v, float2 (&f)[8]) {
  float2 u[8];
  values<T, MOVE>(v, u);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = mul2(f[i], u[i]);
}

template <typename T, int MOVE>
AS_DEV void store16(const Rows& m, long long row, int c0, int cols, const float2 (&f)[8]) {
  T* base = static_cast<T*>(m.data) + row;
  if constexpr (MOVE == MOVE_ELEMENT) {
    auto store = [&](auto at) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = c0 + 32 * i;
        const float x = i % 2 ? f[i / 2].y : f[i / 2].x;
        if (c < cols) base[at(c)] = (T)x;
      }
    };
    if (m.split) store([&](int c) { return m.col(c); });
    else store([](int c) { return c; });
  } else {
    uint32_t w[4 * sizeof(T)];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 2) w[i] = sm100::pack_bf16(f[i].x, f[i].y);
      else { w[2 * i] = __float_as_uint(f[i].x); w[2 * i + 1] = __float_as_uint(f[i].y); }
    }
    if constexpr (MOVE == MOVE32) {
      if (c0 < cols) {
        T* at = base + m.col(c0);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) store32(reinterpret_cast<uint8_t*>(at) + 32 * i, reinterpret_cast<const uint32_t(&)[8]>(w[8 * i]));
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (c0 + 8 * h < cols) {
          uint4* at = reinterpret_cast<uint4*>(base + m.col(c0 + 8 * h));
#pragma unroll
          for (int i = 0; i < (int)sizeof(T) / 2; ++i) at[i] = reinterpret_cast<const uint4*>(w)[h * (int)sizeof(T) / 2 + i];
        }
    }
  }
}

// The bits of a block's largest |value| (NaN is above infinity): of the lane's own block, the eight lanes' columns.
AS_DEV uint32_t block_max(const float2 (&f)[8]) {
  float t = max_abs2(f[0], 0.f);
#pragma unroll
  for (int i = 1; i < 8; ++i) t = max_abs2(f[i], t);
  uint32_t u = __float_as_uint(t);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) u = max(u, __shfl_xor_sync(0xffffffffu, u, o));
  return u;
}
// Element by element: of block b of the warp's four, for all lanes.
AS_DEV uint32_t block_max_elements(const float2 (&f)[8], int b) { return __reduce_max_sync(0xffffffffu, __float_as_uint(max_abs2(f[2 * b], max_abs2(f[2 * b + 1], 0.f)))); }

constexpr float DOWN = 8.271806126e-25f;       // 2^-80: |t| below 2^128 becomes 2^48 at most, and the sum of 16384 squares 2^110
constexpr float UP = 1.267650600e30f;          // 2^100: fp32's smallest number becomes 2^-49, and what LEAST lets through 2^57 at most
constexpr float LEAST = 7.888609052e-31f;      // 2^-100: squares that fp32 rounds below its normal numbers are 2^-150 off, 2^-50 of it
constexpr float MOST = 3.402823466e38f;

// NORM: y = t * rsqrt(mean t^2 + eps) * w, else y = x.  R: the residual's type (void: none).  FP8: y in 8-bit form, else in bf16.  LANES: of a row
// in a warp (8, 16: with one vector).
//
// The order is the formula's: sum of squares, the row's scale times t, the weights, the blocks' largest values.  (Weights ahead of the scale let the block's reductions run beside
// the row's, which gained 0.4 us of 29, 0.3 of 56 and nothing of 82; but t * w may lie beyond fp32 where the normed value times w does not.)  What counts is the number of
// instructions: with 8 columns a lane, one value an instruction, a row of 1536 columns with a residual in bf16 took 131 us for 32760 rows, in pairs 62 us; with 16 columns a lane, whose
// loads are half as many and whose scales are a third as much work, 56 us (6.3 TB/s).  Without a residual 54, 38 and 29 us (5.1 TB/s), the last with CTAs that go on; the 8-bit form
// alone 34, 26 and 25 us (6.1 TB/s; 29 us where the largest values of one vector wait for those of the vector before).  Rows further ahead, as asynchronous copies into shared memory,
// did not help there: 35 and 27 us with four rows under way, for the instructions that it takes.
// With x in bf16 and no residual a CTA goes on from row to row: its weights stay in shared memory, and a row's loads are under way while the one before it is
// worked on.  (With a residual or in fp32 there is enough under way without that, and no room for it.)  Two CTAs an SM.
template <typename X, typename R, int MOVE> constexpr bool goes_on = sizeof(X) == 2 && __is_same(R, void) && MOVE != MOVE_ELEMENT;

// x_bytes: of an element of x.  In bf16 beside a residual three vectors fit 128 registers, two CTAs (32760 x 1536 with a residual in fp32 82 us; left to itself the compiler takes 130, and one CTA
// 103 us).
__host__ __device__ constexpr int ctas_of_sm(bool goes_on, int move, int nv, int x_bytes) {
  return goes_on ? 2 : move != MOVE_ELEMENT ? (x_bytes == 2 && nv <= 3 ? 2 : 1) : nv == 1 ? 4 : nv == 2 ? 2 : 1;
}

template <typename X, typename R, bool NORM, bool FP8, int MOVE, int NV, int LANES>
__global__ void __launch_bounds__(THREADS, ctas_of_sm(goes_on<X, R, MOVE>, MOVE, NV, (int)sizeof(X))) norm_kernel(const __grid_constant__ NormParams p) {
  griddep_launch();
  __shared__ float part[THREADS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int slot, piece = 0, per;                                   // row of the CTA, warp of the row, rows of the CTA
  if constexpr (LANES < 32) {
    per = THREADS / LANES;
    slot = threadIdx.x / LANES;
  } else {
    per = (THREADS / 32) / p.W;
    slot = warp / p.W;
    piece = warp - slot * p.W;
  }
  constexpr bool GOES_ON = goes_on<X, R, MOVE>;
  const int first = piece * (NV * 512);                       // columns of this warp
  const int c0 = first + (MOVE == MOVE_ELEMENT ? lane : (lane & (LANES - 1)) * 16);
  long long row = (long long)blockIdx.x * per + slot;
  const bool weighs = NORM && p.w != nullptr, early = weighs && !p.w_f32 && MOVE != MOVE_ELEMENT && !GOES_ON;
  Raw<__nv_bfloat16, MOVE> w16[NV];                           // weights in bf16 come beside x: behind it they would cost a row their latency once more
  Raw<X, MOVE> x[NV];
  auto fetch_x = [&](long long at) {                          // of a row that is not there nothing is read or written
    const bool there = slot < per && at < p.rows;
    const long long xr = there ? p.x.row((unsigned)at) : 0;
    fetch_row<X, MOVE, NV>(p.x, xr, c0, there ? p.cols : 0, x);
  };
  // weights in bf16 of a CTA that goes on: the 32 bytes of column vector u of the row as two pieces of 16 bytes, the vectors of a group of four blocks
  // next to each other, so that a warp reads each piece without bank conflicts
  extern __shared__ uint4 kept[];
  griddep_wait();
  Rows weights{};
  weights.data = const_cast<void*>(p.w);
  fetch_x(row);
  if constexpr (GOES_ON) {
    if (weighs && !p.w_f32) {
      const uint4* w = static_cast<const uint4*>(p.w);        // 16-byte aligned, a multiple of 8 columns
      for (int i = threadIdx.x; i < (p.cols + 511) / 512 * 64; i += THREADS) kept[i / 64 * 64 + i % 2 * 32 + i % 64 / 2] = i * 8 < p.cols ? w[i] : uint4{};
    }
    __syncthreads();
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) fetch<__nv_bfloat16, MOVE>(weights, 0, c0 + j * 512, early ? p.cols : 0, w16[j]);
  }
  // (a turn is one for the whole CTA: a warp whose row is not there takes part in its barrier)
  for (long long first_row = (long long)blockIdx.x * per; first_row < p.rows; first_row += (long long)gridDim.x * per, row += (long long)gridDim.x * per) {
  const bool live = slot < per && row < p.rows;
  const unsigned r = live ? (unsigned)row : 0u;
  const int cols = live ? p.cols : 0;
  float2 v[NV][8];
  {
    if constexpr (!__is_same(R, void)) {
      Raw<R, MOVE> t[NV];
      const long long rr = p.r.row(r), wr = p.ro.row(r);
      fetch_row<R, MOVE, NV>(p.r, rr, c0, cols, t);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        values<X, MOVE>(x[j], v[j]);
        add_values<R, MOVE>(t[j], v[j]);
        store16<R, MOVE>(p.ro, wr, c0 + j * 512, cols, v[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) values<X, MOVE>(x[j], v[j]);
    }
    if constexpr (GOES_ON) fetch_x(row + (long long)gridDim.x * per);
  }
  if constexpr (NORM) {
    float2 sum2 = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum2 = fma2(v[j][i], v[j][i], sum2);
    // over the row's lanes and warps
    auto row_sum = [&](float sum) {
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if constexpr (LANES == 32)
        if (p.W > 1) {                                        // the same for every thread of the launch
          if (lane == 0) part[warp] = sum;
          __syncthreads();
          sum = 0.f;
          for (int i = 0; i < p.W; ++i) sum += part[min(slot * p.W + i, THREADS / 32 - 1)];
        }
      return sum;
    };
    const float sum = row_sum(sum2.x + sum2.y);
    const float mean = sum / (float)p.cols + p.eps;
    float scale = rsqrtf(mean);
    // Rows whose squares fp32 does not hold (|t| from 2^64 / sqrt(cols) on), or whose squares vanish with an eps that does as well, are summed again times a power of two.
    const bool over = !(sum <= MOST), under = live && mean < LEAST;
    bool again = over || under;                               // (the sum of all lanes of a row is one value)
    if constexpr (LANES < 32) again = __any_sync(0xffffffffu, again);
    if constexpr (LANES == 32)
      if (p.W > 1) again = __syncthreads_or(again);           // (behind it the sums have been read)
    if (again) {
      const float factor = over ? DOWN : UP;
      float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) { const float2 u = mul2(v[j][i], make_float2(factor, factor)); s2 = fma2(u, u, s2); }
      const float s = row_sum(s2.x + s2.y), once = rsqrtf(s / (float)p.cols + p.eps * factor * factor);
      if constexpr (LANES == 32)
        if (p.W > 1) __syncthreads();
      if (over) scale = once * DOWN;
      if (under) {                                            // the row's scale may lie beyond fp32: t takes the factor first
        scale = once;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) v[j][i] = mul2(v[j][i], make_float2(UP, UP));
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = mul2(v[j][i], make_float2(scale, scale));
    // the weights last, as in the formula: t * w may lie beyond fp32 where the normed value times w does not
    if (early) {
#pragma unroll
      for (int j = 0; j < NV; ++j) scale_values<__nv_bfloat16, MOVE>(w16[j], v[j]);
    } else if (weighs && !p.w_f32) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        Raw<__nv_bfloat16, MOVE> w{};
        if constexpr (GOES_ON) {
          if ((first / 512 + j) * 512 < p.cols) {
            const uint4* at = kept + (first / 512 + j) * 64 + (lane & (LANES - 1));
            reinterpret_cast<uint4*>(w.w)[0] = at[0];
            reinterpret_cast<uint4*>(w.w)[1] = at[32];
          }
        } else {
          fetch<__nv_bfloat16, MOVE, MOVE != MOVE_ELEMENT>(weights, 0, c0 + j * 512, cols, w);
        }
        scale_values<__nv_bfloat16, MOVE>(w, v[j]);
      }
    } else if (weighs) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        Raw<float, MOVE> w;
        fetch<float, MOVE, MOVE != MOVE_ELEMENT>(weights, 0, c0 + j * 512, cols, w);
        scale_values<float, MOVE>(w, v[j]);
      }
    }
  }
  if constexpr (!FP8) {
    const long long wr = p.o.row(r);
#pragma unroll
    for (int j = 0; j < NV; ++j) store16<__nv_bfloat16, MOVE>(p.o, wr, c0 + j * 512, cols, v[j]);
  } else {
    uint8_t* q = p.q + (long long)r * p.pitch;
    constexpr int BLOCKS = MOVE == MOVE_ELEMENT ? 4 : 1;      // of a vector whose largest values a lane has
    uint32_t top[NV][BLOCKS];                                 // of all vectors at once: their turns between the lanes overlap
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if constexpr (MOVE == MOVE_ELEMENT) {
#pragma unroll
        for (int b = 0; b < 4; ++b) top[j][b] = block_max_elements(v[j], b);
      } else {
        top[j][0] = block_max(v[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + j * 512, group = first / 512 + j;
      uint32_t byte[BLOCKS];
      float inv[BLOCKS];
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b) {
        byte[b] = scale_byte(top[j][b]);
        inv[b] = inverse_scale(byte[b]);
      }
      uint32_t word = 0u;                                     // the four blocks' bytes; those behind the last column are 0
      if constexpr (MOVE != MOVE_ELEMENT) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = make_float2(inv[0], inv[0]), y = mul2(v[j][2 * i], f), z = mul2(v[j][2 * i + 1], f);
          w[i] = __byte_perm(pack_e4m3(y.x, y.y), pack_e4m3(z.x, z.y), 0x5410);
        }
        if constexpr (MOVE == MOVE32) {
          if (c < cols) *reinterpret_cast<uint4*>(q + c) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
          if (c < cols) *reinterpret_cast<uint2*>(q + c) = make_uint2(w[0], w[1]);
          if (c + 8 < cols) *reinterpret_cast<uint2*>(q + c + 8) = make_uint2(w[2], w[3]);
        }
        word = (c & ~127) < cols ? byte[0] << (lane / 8 * 8) : 0u;       // (c & ~127: the first column of the lane's block, as vectors begin at multiples of 512)
        if constexpr (LANES >= 16) word |= __shfl_xor_sync(0xffffffffu, word, 8);
        if constexpr (LANES == 32) word |= __shfl_xor_sync(0xffffffffu, word, 16);
        if constexpr (LANES < 32) word >>= (lane & ~(LANES - 1)) / 8 * 8 & 31;
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c + 32 * i < cols) q[c + 32 * i] = (uint8_t)pack_e4m3((i % 2 ? v[j][i / 2].y : v[j][i / 2].x) * inv[i / 4], 0.f);
#pragma unroll
        for (int b = 0; b < 4; ++b)
          if (512 * group + 128 * b < cols) word |= byte[b] << (8 * b);
      }
      if ((lane & (LANES - 1)) == 0 && 512 * group < cols) *reinterpret_cast<uint32_t*>(p.scales + ((long long)group * p.scale_rows + r) * 4) = word;
    }
  }
  if constexpr (!GOES_ON) return;
  }
}

// Four elements of a row, 32 columns apart.
template <typename X>
AS_DEV void fetch_four(const Rows& m, long long row, int c0, int cols, X* e) {
  const X* base = static_cast<const X*>(m.data) + row;
  long long at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) at[i] = c0 + 32 * i;
  if (m.split) {
#pragma unroll
    for (int i = 0; i < 4; ++i) at[i] = m.col(c0 + 32 * i);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) e[i] = c0 + 32 * i < cols ? base[at[i]] : (X)0.f;
}

// A scale for 128 rows and 128 columns: a CTA per block, a thread's 64 elements in registers: 8 lanes a row and 16 columns a lane, or element by
// element 4 columns of each of 16 rows.  The CTA of a group's last block writes the bytes behind it as well.
template <typename X, int MOVE>
__global__ void __launch_bounds__(THREADS) quantize_block_kernel(const __grid_constant__ NormParams p) {
  griddep_launch();
  __shared__ uint32_t part[THREADS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = blockIdx.x * 128, row0 = blockIdx.y * 128;
  float2 v[4][8];
  float most = 0.f;
  griddep_wait();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (MOVE != MOVE_ELEMENT) {
      const int row = row0 + j * 32 + threadIdx.x / 8;
      Raw<X, MOVE> x;
      fetch<X, MOVE>(p.x, row < p.rows ? p.x.row(row) : 0, c0 + lane % 8 * 16, row < p.rows ? p.cols : 0, x);
      values<X, MOVE>(x, v[j]);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = row0 + warp * 16 + j * 4 + r;
        Raw<X, MOVE> x;                       // (its first four: 32 columns apart)
        fetch_four<X>(p.x, row < p.rows ? p.x.row(row) : 0, c0 + lane, row < p.rows ? p.cols : 0, x.e);
        v[j][2 * r] = make_float2((float)x.e[0], (float)x.e[1]);
        v[j][2 * r + 1] = make_float2((float)x.e[2], (float)x.e[3]);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max_abs2(v[j][i], most);
  }
  uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(most));
  if (lane == 0) part[warp] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < THREADS / 32; ++i) top = max(top, part[i]);
  const uint32_t byte = scale_byte(top);
  const float inv = inverse_scale(byte);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (MOVE != MOVE_ELEMENT) {
      const int row = row0 + j * 32 + threadIdx.x / 8, c = c0 + lane % 8 * 16;
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = __byte_perm(pack_e4m3(v[j][2 * i].x * inv, v[j][2 * i].y * inv), pack_e4m3(v[j][2 * i + 1].x * inv, v[j][2 * i + 1].y * inv), 0x5410);
      uint8_t* q = p.q + (long long)row * p.pitch + c;
      if (row < p.rows && c < p.cols) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
      if (row < p.rows && c + 8 < p.cols) *reinterpret_cast<uint2*>(q + 8) = make_uint2(w[2], w[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = row0 + warp * 16 + j * 4 + i / 4, c = c0 + i % 4 * 32 + lane;
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

// Lanes of a row in a warp, warps of a row, vectors of a lane.
struct Split { int lanes, W, NV; };
Split split_of(int cols, int move) {
  if (move != MOVE_ELEMENT && cols <= 256) return {cols <= 128 ? 8 : 16, 1, 1};
  // A fourth vector does not fit the registers of two CTAs beside the next row.  Element by element latency counts, so as many warps as there are take one vector each (32760 x 1537 with a
  // residual in bf16 198 us, by two vectors a warp 230, by four 514; 8000 x 4001 alone to 8 bits 46 and 104).
  const int most = move != MOVE_ELEMENT ? (cols <= 8 * 1536 ? 3 : 4) : cols <= 4096 ? 1 : cols <= 8192 ? 2 : 4;
  const int W = (cols + 512 * most - 1) / (512 * most);
  return {32, W, (cols + 512 * W - 1) / (512 * W)};
}

template <typename X, typename R, bool NORM, bool FP8, int MOVE, int NV, int LANES>
cudaError_t launch(const NormParams& p, cudaStream_t st) {
  const long long per = LANES < 32 ? THREADS / LANES : (THREADS / 32) / p.W;
  long long ctas = (p.rows + per - 1) / per;
  size_t smem = 0;
  if (goes_on<X, R, MOVE>) {
    ctas = std::min(ctas, 2ll * p.sms);
    if (p.w != nullptr && !p.w_f32) smem = (size_t)(p.cols + 511) / 512 * 1024;     // 32 KB at most
  }
  return as_launch_dependent(norm_kernel<X, R, NORM, FP8, MOVE, NV, LANES>, dim3((unsigned)ctas), dim3(THREADS), smem, st, p);
}
template <typename X, typename R, bool NORM, bool FP8, int MOVE>
cudaError_t launch_split(const NormParams& p, const Split& s, cudaStream_t st) {
  if constexpr (MOVE == MOVE_ELEMENT) {       // fewer forms: the columns that are not there cost their comparison only
    return s.NV == 1 ? launch<X, R, NORM, FP8, MOVE, 1, 32>(p, st) : s.NV == 2 ? launch<X, R, NORM, FP8, MOVE, 2, 32>(p, st) : launch<X, R, NORM, FP8, MOVE, 4, 32>(p, st);
  } else {
    if (s.lanes == 8) return launch<X, R, NORM, FP8, MOVE, 1, 8>(p, st);
    if (s.lanes == 16) return launch<X, R, NORM, FP8, MOVE, 1, 16>(p, st);
    switch (s.NV) {
      case 1: return launch<X, R, NORM, FP8, MOVE, 1, 32>(p, st);
      case 2: return launch<X, R, NORM, FP8, MOVE, 2, 32>(p, st);
      case 3: return launch<X, R, NORM, FP8, MOVE, 3, 32>(p, st);
      default: return launch<X, R, NORM, FP8, MOVE, 4, 32>(p, st);
    }
  }
}
template <typename X, typename R, bool NORM, bool FP8>
cudaError_t launch_move(const NormParams& p, int move, const Split& s, cudaStream_t st) {
  switch (move) {
    case MOVE32: return launch_split<X, R, NORM, FP8, MOVE32>(p, s, st);
    case MOVE16: return launch_split<X, R, NORM, FP8, MOVE16>(p, s, st);
    default: return launch_split<X, R, NORM, FP8, MOVE_ELEMENT>(p, s, st);
  }
}
template <typename X, typename R, bool NORM>
cudaError_t launch_out(const NormParams& p, bool fp8, int move, const Split& s, cudaStream_t st) {
  if constexpr (NORM)
    if (!fp8) return launch_move<X, R, NORM, false>(p, move, s, st);
  return launch_move<X, R, NORM, true>(p, move, s, st);
}

// How the rows of a call can move: what all its matrices allow.
int move_of(const as_rows_t& x) { return rows_vec(x, 32) ? MOVE32 : rows_vec(x, 16) ? MOVE16 : MOVE_ELEMENT; }

as_status_t device_ok(int* sms) {
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return failed();
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
  NormParams p{};
  if (const as_status_t s = device_ok(&p.sms); s != AS_OK) return s;
  p.rows = (int)a->rows; p.cols = a->cols; p.eps = a->eps;
  p.x = rows_of(a->x, a->rows, a->cols);
  int move = move_of(a->x);
  if (a->weight != nullptr) move = std::max(move, aligned(a->weight, 32) ? MOVE32 : aligned(a->weight, 16) ? MOVE16 : MOVE_ELEMENT);
  if (res) {
    p.r = rows_of(a->residual, a->rows, a->cols);
    p.ro = rows_of(a->residual_out, a->rows, a->cols);
    move = std::max(move, std::max(move_of(a->residual), move_of(a->residual_out)));
  }
  if (fp8) {
    p.q = static_cast<uint8_t*>(a->out8.data); p.pitch = a->out8.pitch;
    p.scales = static_cast<uint8_t*>(a->out8.scales); p.scale_rows = a->out8.scale_rows;
  } else {
    p.o = rows_of(a->out, a->rows, a->cols);
    move = std::max(move, move_of(a->out));
  }
  p.w = a->weight; p.w_f32 = a->weight_dtype == AS_DTYPE_F32;
  const Split s = split_of(a->cols, move);
  p.W = s.W;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  typedef __nv_bfloat16 bf;
  if (a->x.dtype == AS_DTYPE_F32) e = res ? launch_out<float, float, true>(p, fp8, move, s, st) : launch_out<float, void, true>(p, fp8, move, s, st);
  else if (!res) e = launch_out<bf, void, true>(p, fp8, move, s, st);
  else e = a->residual.dtype == AS_DTYPE_BF16 ? launch_out<bf, bf, true>(p, fp8, move, s, st) : launch_out<bf, float, true>(p, fp8, move, s, st);
  return e == cudaSuccess ? AS_OK : failed();
}

extern "C" as_status_t as_quantize_fp8(const as_quantize_fp8_t* a, void* cuda_stream) {
  if (a == nullptr || a->struct_size != sizeof(as_quantize_fp8_t) || a->reserved != 0) return AS_ERR_INVALID_ARG;
  if (a->cols < 1 || a->rows < 0 || a->rows > 0x7fffffffll || (a->block_rows != 1 && a->block_rows != 128)) return AS_ERR_INVALID_ARG;
  if (!rows_ok(a->x, a->rows, a->cols) || !matrix_ok(a->out, a->rows, a->cols)) return AS_ERR_INVALID_ARG;
  if (a->cols > 16384 || (a->block_rows == 128 && a->rows > 65535ll * 128)) return AS_ERR_UNSUPPORTED;
  if (a->rows == 0) return AS_OK;
  NormParams p{};
  if (const as_status_t s = device_ok(&p.sms); s != AS_OK) return s;
  p.rows = (int)a->rows; p.cols = a->cols;
  p.x = rows_of(a->x, a->rows, a->cols);
  p.q = static_cast<uint8_t*>(a->out.data); p.pitch = a->out.pitch;
  p.scales = static_cast<uint8_t*>(a->out.scales); p.scale_rows = a->out.scale_rows;
  const int move = move_of(a->x);
  const bool f32 = a->x.dtype == AS_DTYPE_F32;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  typedef __nv_bfloat16 bf;
  if (a->block_rows == 1) {
    const Split s = split_of(a->cols, move);
    p.W = s.W;
    e = f32 ? launch_out<float, void, false>(p, true, move, s, st) : launch_out<bf, void, false>(p, true, move, s, st);
  } else {
    const dim3 grid((unsigned)((a->cols + 127) / 128), (unsigned)((a->rows + 127) / 128));
    auto run = [&](auto kernel) { return as_launch_dependent(kernel, grid, dim3(THREADS), 0, st, p); };
    if (f32) e = move == MOVE32 ? run(quantize_block_kernel<float, MOVE32>) : move == MOVE16 ? run(quantize_block_kernel<float, MOVE16>) : run(quantize_block_kernel<float, MOVE_ELEMENT>);
    else e = move == MOVE32 ? run(quantize_block_kernel<bf, MOVE32>) : move == MOVE16 ? run(quantize_block_kernel<bf, MOVE16>) : run(quantize_block_kernel<bf, MOVE_ELEMENT>);
  }
  return e == cudaSuccess ? AS_OK : failed();
}
