// Norms of queries and keys, their rotation by the tokens' positions, and the gradients of both.
//
// All of it reads a tensor once and writes it once: bound by HBM bytes.  A lane holds 16 elements of a head in two pieces of 8, chosen so that both elements of a pair are
// its own: 16 in a run (interleaved pairs, and what is not turned) or 8 of each half (pairs of halves).  The lanes of a head are a power of two, so that a head's sum is a few
// exchanges; a warp holds 32 / lanes heads a vector and NV vectors, and where the norm is over a token's heads up to 8 warps hold a row.  A token's cos and sin are the same for
// every head and for queries and keys: a lane reads those of its 8 pairs once for all of them.  Heads whose sizes, strides or addresses are no multiples of 16 bytes go pair by
// pair (turn_elements_kernel).
#include <algorithm>
#include <cmath>

#include "as_layer.h"
#include "fp8_common.cuh"

namespace {

using namespace as_fp8;
using sm100::griddep_launch;
using sm100::griddep_wait;
typedef __nv_bfloat16 bf;

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr float DOWN = 8.271806126e-25f;       // 2^-80: |x| below 2^128 becomes 2^48 at most, and the sum of 16384 squares 2^110
constexpr float UP = 1.267650600e30f;          // 2^100: fp32's smallest number becomes 2^-49
constexpr float LEAST = 7.888609052e-31f;      // 2^-100: squares that fp32 rounds below its normal numbers are 2^-150 off, 2^-50 of it
constexpr float MOST = 3.402823466e38f;

// ---------------------------------------------------------------- the table
struct TableAxis { double step, amplitude; double base, factor, original; int scaling, pairs, first_row, first_pair; };
struct TableParams {
  float2* out;
  int rows, pairs, axes;
  TableAxis axis[AS_ROTARY_MAX_AXES];
};
constexpr int TABLE_ROWS = 64;                 // of a CTA

// A thread has one pair and walks over rows: its angle a position, in turns, is taken once.  cos and sin of a quarter turn around the next multiple of one, from an angle that 64 bits hold to
// 2^-53 of the position's turns; rounded to fp32 there, it is 2^-24 relative.
__global__ void __launch_bounds__(THREADS) table_kernel(const __grid_constant__ TableParams p) {
  griddep_launch();
  const int pair = blockIdx.y * 64 + threadIdx.x % 64;
  if (pair >= p.pairs) return;
  int a = 0;
#pragma unroll
  for (int i = 1; i < AS_ROTARY_MAX_AXES; ++i)
    if (i < p.axes && pair >= p.axis[i].first_pair) a = i;
  TableAxis x = p.axis[0];
#pragma unroll
  for (int i = 1; i < AS_ROTARY_MAX_AXES; ++i)
    if (a == i) x = p.axis[i];
  const int i = pair - x.first_pair;
  double f, amplitude = 1.;
  if (x.scaling == AS_ROTARY_NTK) f = x.pairs == 1 ? 1. : pow(x.base * pow(x.factor, (double)x.pairs / (x.pairs - 1)), -(double)i / x.pairs);
  else f = pow(x.base, -(double)i / x.pairs);
  if (x.scaling == AS_ROTARY_LINEAR) f /= x.factor;
  const double tau = 6.283185307179586476925;
  if (x.scaling == AS_ROTARY_YARN) {
    const double g = fmin(1., fmax(0., (x.original * f / tau - 1.) / 31.));
    f = f * g + f / x.factor * (1. - g);
    amplitude = 0.1 * log(x.factor) + 1.;
  }
  f /= tau;
  const int end = a + 1 < p.axes ? p.axis[min(a + 1, AS_ROTARY_MAX_AXES - 1)].first_row : p.rows;
  griddep_wait();
  const int row0 = blockIdx.x * TABLE_ROWS;
  for (int r = row0 + threadIdx.x / 64; r < min(row0 + TABLE_ROWS, p.rows); r += THREADS / 64) {
    float2 v = make_float2(0.f, 0.f);
    if (r >= x.first_row && r < end) {
      const double turns = (r - x.first_row) * f, t = 4. * (turns - rint(turns)), q = rint(t);
      float s, c;
      sincospif(0.5f * (float)(t - q), &s, &c);
      const int n = (int)q & 3;
      const float cc = n & 1 ? s : c, ss = n & 1 ? c : s;
      v.x = (float)(amplitude * (n == 1 || n == 2 ? -cc : cc));
      v.y = (float)(amplitude * (n >= 2 ? -ss : ss));
    }
    p.out[(long long)r * p.pairs + pair] = v;
  }
}

// ---------------------------------------------------------------- parameters
struct TurnTensor {
  Rows x, o, dy;                             // (dy: of the backward pass)
  const void* w;
  float* part;                               // backward: partial sums of the weights' gradient, NULL where none is wanted
  void* dw;
  int heads;
};
struct TurnParams {
  TurnTensor t[2];
  const float2* table;
  const void* pos;
  long long pos_stride, first;
  float eps;
  int n_t, rows, tokens, d;
  int pairs, axes, half, pos64;
  int size[AS_ROTARY_MAX_AXES], first_row[AS_ROTARY_MAX_AXES], end[AS_ROTARY_MAX_AXES];      // end: of the axes' pairs
  float sign;                                // of sin
  int w_f32;
  int lanes_log;                             // lanes of a head: 2^lanes_log
  int W;                                     // warps of a row
  int chunks;                                // runs of heads that a warp takes at once, where the norm is not over rows
};

struct Where { int at[AS_ROTARY_MAX_AXES]; };
// Rows of the table for row r; -1: no such position.
AS_DEV Where where_of(const TurnParams& p, unsigned r) {
  Where w{};
  const unsigned b = r / (unsigned)p.tokens, t = r - b * (unsigned)p.tokens;
  if (p.pos != nullptr) {
    const long long at = (long long)b * p.pos_stride + (long long)t * p.axes;
#pragma unroll
    for (int a = 0; a < AS_ROTARY_MAX_AXES; ++a)
      if (a < p.axes) {
        const long long v = p.pos64 ? static_cast<const long long*>(p.pos)[at + a] : static_cast<const int*>(p.pos)[at + a];
        w.at[a] = v >= 0 && v < p.size[a] ? p.first_row[a] + (int)v : -1;
      }
  } else {
    unsigned i = (unsigned)p.first + t;
#pragma unroll
    for (int a = AS_ROTARY_MAX_AXES - 1; a > 0; --a)
      if (a < p.axes) {
        const unsigned q = i / (unsigned)p.size[a];
        w.at[a] = p.first_row[a] + (int)(i - q * (unsigned)p.size[a]);
        i = q;
      }
    w.at[0] = (int)i;
  }
  return w;
}
AS_DEV int axis_of(const TurnParams& p, int pair) { return (pair >= p.end[0]) + (pair >= p.end[1]) + (pair >= p.end[2]); }
AS_DEV int pick(const Where& w, int a) { return a == 0 ? w.at[0] : a == 1 ? w.at[1] : a == 2 ? w.at[2] : w.at[3]; }
AS_DEV float2 factor_of(const TurnParams& p, const Where& w, int pair) {
  const int row = pick(w, axis_of(p, pair));
  if (row < 0) return make_float2(__uint_as_float(0x7fc00000u), __uint_as_float(0x7fc00000u));
  float2 f = __ldg(p.table + (long long)row * p.pairs + pair);
  f.y *= p.sign;
  return f;
}
// Of 8 pairs from a multiple of 8 on.
AS_DEV void factors(const TurnParams& p, const Where& w, int pair, float2 (&f)[8]) {
  const int a = axis_of(p, pair);
  if (a == axis_of(p, pair + 7)) {
    const int row = pick(w, a);
    const float4* at = reinterpret_cast<const float4*>(p.table + (long long)max(row, 0) * p.pairs + pair);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float4 v = __ldg(at + i);
      if (row < 0) v.x = v.y = v.z = v.w = __uint_as_float(0x7fc00000u);
      f[2 * i] = make_float2(v.x, v.y * p.sign);
      f[2 * i + 1] = make_float2(v.z, v.w * p.sign);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = factor_of(p, w, pair + i);
  }
}

// ---------------------------------------------------------------- vectors of a lane
template <typename T> struct Raw { uint4 v[sizeof(T)]; };        // 16 elements: two pieces of 8
template <typename T>
AS_DEV void load(Raw<T>& r, const T* at, int second) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
    r.v[i] = *reinterpret_cast<const uint4*>(at + i * (16 / sizeof(T)));
    r.v[sizeof(T) / 2 + i] = *reinterpret_cast<const uint4*>(at + second + i * (16 / sizeof(T)));
  }
}
template <typename T>
AS_DEV void values(const Raw<T>& r, float (&f)[16]) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(r.v);
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(w[i]);
  }
}
template <typename T>
AS_DEV void store(T* at, int second, const float (&f)[16]) {
  uint4 v[sizeof(T)];
  uint32_t* w = reinterpret_cast<uint32_t*>(v);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if constexpr (sizeof(T) == 2) { if (i % 2 == 0) w[i / 2] = sm100::pack_bf16(f[i], f[i + 1]); }
    else w[i] = __float_as_uint(f[i]);
  }
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
    *reinterpret_cast<uint4*>(at + i * (16 / sizeof(T))) = v[i];
    *reinterpret_cast<uint4*>(at + second + i * (16 / sizeof(T))) = v[sizeof(T) / 2 + i];
  }
}
AS_DEV void load_weights(const TurnParams& p, const void* w, int at, int second, float (&f)[16]) {
  if (p.w_f32) {
    Raw<float> r;
    load(r, static_cast<const float*>(w) + at, second);
    values(r, f);
  } else {
    Raw<bf> r;
    load(r, static_cast<const bf*>(w) + at, second);
    values(r, f);
  }
}
AS_DEV void turn(float (&f)[16], const float2 (&cs)[8], int half) {
  if (half) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = f[i], b = f[8 + i];
      f[i] = a * cs[i].x - b * cs[i].y;
      f[8 + i] = a * cs[i].y + b * cs[i].x;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = f[2 * i], b = f[2 * i + 1];
      f[2 * i] = a * cs[i].x - b * cs[i].y;
      f[2 * i + 1] = a * cs[i].y + b * cs[i].x;
    }
  }
}

// What a lane works on: its head of vector 0, elements of a head, whether they are turned.
struct Lane { int head, heads_a_vector, e0, second, pair; bool in_head, turned; };
AS_DEV Lane lane_of(const TurnParams& p, int lane) {
  Lane l;
  const int slot = lane & ((1 << p.lanes_log) - 1);
  l.head = lane >> p.lanes_log;
  l.heads_a_vector = 32 >> p.lanes_log;
  l.in_head = slot * 16 < p.d;
  l.pair = slot * 8;
  l.turned = p.table != nullptr && l.pair < p.pairs;
  const bool halves = l.turned && p.half;
  l.e0 = halves ? slot * 8 : slot * 16;
  l.second = halves ? p.pairs : 8;
  return l;
}

// Sum over a head's lanes, or over a row's lanes and warps (in the order of the warps).
template <int NORM>
AS_DEV float sum_of(const TurnParams& p, float s, float* part, int slot, int warp, int lane) {
  if constexpr (NORM == AS_NORM_HEAD) {
    for (int o = 1 << p.lanes_log >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  } else {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (p.W > 1) {                             // the same for every thread of the launch
      __syncthreads();                         // the sums before these have been read
      if (lane == 0) part[warp] = s;
      __syncthreads();
      s = 0.f;
      for (int i = 0; i < p.W; ++i) s += part[min(slot * p.W + i, WARPS - 1)];
    }
  }
  return s;
}
// Whether any lane that takes part in the same exchanges asks for it.
template <int NORM>
AS_DEV bool any_of(const TurnParams& p, bool ask) {
  if constexpr (NORM == AS_NORM_ROW)
    if (p.W > 1) return __syncthreads_or(ask);
  return __any_sync(0xffffffffu, ask);
}

// x * factor * scale is the normed value.  `squares(f)`: the lane's sum of (f x)^2.  Rows whose squares fp32 does not hold, or whose squares vanish together with eps, are summed
// again times a power of two.
struct Scale { float factor, scale; };
template <int NORM, typename F>
AS_DEV Scale scale_of(const TurnParams& p, float n, bool live, float* part, int slot, int warp, int lane, F squares) {
  const float sum = sum_of<NORM>(p, squares(1.f), part, slot, warp, lane), mean = sum / n + p.eps;
  Scale s{1.f, rsqrtf(mean)};
  const bool over = !(sum <= MOST), under = live && mean < LEAST;
  if (any_of<NORM>(p, over || under)) {
    const float f = over ? DOWN : under ? UP : 1.f;
    const float again = sum_of<NORM>(p, squares(f), part, slot, warp, lane);
    s = {f, rsqrtf(again / n + p.eps * f * f)};
  }
  return s;
}

// ---------------------------------------------------------------- forward
template <typename T, int NORM, int NV>
__global__ void __launch_bounds__(THREADS, 2) turn_kernel(const __grid_constant__ TurnParams p) {
  griddep_launch();
  __shared__ float part[WARPS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int slot = 0, piece;
  long long row;
  if constexpr (NORM == AS_NORM_ROW) {
    const int per = WARPS / p.W;
    slot = warp / p.W;
    piece = warp - slot * p.W;
    row = slot < per ? (long long)blockIdx.x * per + slot : p.rows;
  } else {
    const long long unit = (long long)blockIdx.x * WARPS + warp;
    row = unit / p.chunks;
    piece = (int)(unit - row * p.chunks);
  }
  const bool live = row < p.rows;
  const unsigned r = live ? (unsigned)row : 0u;
  const Lane l = lane_of(p, lane);
  const int h0 = piece * NV * l.heads_a_vector + l.head;
  griddep_wait();
  constexpr int AHEAD = sizeof(T) == 2 ? 2 : 1;          // tensors whose loads are under way at once
  Raw<T> raw[AHEAD][NV];
  auto fetch = [&](const TurnTensor& t, Raw<T> (&x)[NV]) {
    const T* base = static_cast<const T*>(t.x.data) + t.x.row(r) + l.e0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int h = h0 + j * l.heads_a_vector;
      x[j] = Raw<T>{};
      if (live && l.in_head && h < t.heads) load(x[j], base + h * t.x.sh, l.second);
    }
  };
  fetch(p.t[0], raw[0]);
  if constexpr (AHEAD == 2)
    if (p.n_t == 2) fetch(p.t[1], raw[1]);
  float2 cs[8];
  if (l.turned) factors(p, where_of(p, r), l.pair, cs);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (i >= p.n_t) break;
    const TurnTensor& t = p.t[i];
    Raw<T> (&x)[NV] = raw[AHEAD == 2 ? i : 0];
    if constexpr (AHEAD == 1)
      if (i == 1) fetch(t, x);
    T* out = static_cast<T*>(t.o.data) + t.o.row(r) + l.e0;
    Scale s{1.f, 1.f};
    if constexpr (NORM == AS_NORM_ROW)
      s = scale_of<NORM>(p, (float)t.heads * (float)p.d, live, part, slot, warp, lane, [&](float f) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          float v[16];
          values(x[j], v);
#pragma unroll
          for (int e = 0; e < 16; e += 2) { a = fmaf(v[e] * f, v[e] * f, a); b = fmaf(v[e + 1] * f, v[e + 1] * f, b); }
        }
        return a + b;
      });
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int h = h0 + j * l.heads_a_vector;
      const bool there = live && l.in_head && h < t.heads;
      float v[16];
      values(x[j], v);
      if constexpr (NORM == AS_NORM_HEAD)
        s = scale_of<NORM>(p, (float)p.d, there, part, slot, warp, lane, [&](float f) {
          float a = 0.f, b = 0.f;
#pragma unroll
          for (int e = 0; e < 16; e += 2) { a = fmaf(v[e] * f, v[e] * f, a); b = fmaf(v[e + 1] * f, v[e + 1] * f, b); }
          return a + b;
        });
      if (!there) continue;
      if constexpr (NORM != AS_NORM_NONE) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = v[e] * s.factor * s.scale;
        if (t.w != nullptr) {
          float w[16];
          load_weights(p, t.w, (NORM == AS_NORM_ROW ? h * p.d : 0) + l.e0, l.second, w);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] *= w[e];
        }
      }
      if (l.turned) turn(v, cs, p.half);
      store(out + h * t.o.sh, l.second, v);
    }
  }
}

// ---------------------------------------------------------------- backward
// dx = r (g - n mean(g n)), g = d w, d = R^T dy, n = x r.  A CTA goes on from row to row and keeps its sums of d n in registers: of a head's elements where heads share the weights, else of all
// of a row's.  Both sums of a row, over x^2 and over g x, are taken at once.
template <typename T, int NORM, int NV>
__global__ void __launch_bounds__(THREADS) turn_back_kernel(const __grid_constant__ TurnParams p) {
  griddep_launch();
  __shared__ float part[WARPS], part2[WARPS];
  extern __shared__ float sums[];                        // of the weights' gradient, a row of them
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const TurnTensor& t = p.t[blockIdx.y];
  constexpr bool ROW = NORM == AS_NORM_ROW;
  constexpr int NA = ROW ? NV : 1;
  const int per = ROW ? WARPS / p.W : WARPS;
  const int slot = ROW ? warp / p.W : warp, fixed_piece = ROW ? warp - slot * p.W : 0;
  const Lane l = lane_of(p, lane);
  float acc[NA][16] = {};
  const long long units = ROW ? p.rows : (long long)p.rows * p.chunks;
  griddep_wait();
  for (long long u0 = (long long)blockIdx.x * per; u0 < units; u0 += (long long)gridDim.x * per) {       // a turn is one for the whole CTA
    const long long u = u0 + slot;
    const bool live = slot < per && u < units;
    const unsigned r = live ? (unsigned)(ROW ? u : u / p.chunks) : 0u;
    const int h0 = (ROW ? fixed_piece : live ? (int)(u - (long long)r * p.chunks) : 0) * NV * l.heads_a_vector + l.head;
    Raw<T> x[NV], y[NV];
    const T* bx = static_cast<const T*>(t.x.data) + t.x.row(r) + l.e0;
    const T* by = static_cast<const T*>(t.dy.data) + t.dy.row(r) + l.e0;
    T* out = static_cast<T*>(t.o.data) + t.o.row(r) + l.e0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int h = h0 + j * l.heads_a_vector;
      x[j] = Raw<T>{};
      y[j] = Raw<T>{};
      if (live && l.in_head && h < t.heads) {
        load(x[j], bx + h * t.x.sh, l.second);
        load(y[j], by + h * t.dy.sh, l.second);
      }
    }
    float2 cs[8];
    if (l.turned) factors(p, where_of(p, r), l.pair, cs);
    auto weights = [&](int h, float (&w)[16]) {
      if (t.w != nullptr && l.in_head && h < t.heads) {
        load_weights(p, t.w, (ROW ? h * p.d : 0) + l.e0, l.second, w);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = 1.f;
      }
    };
    auto gradient = [&](int j, float (&d)[16]) {
      values(y[j], d);
      if (l.turned) turn(d, cs, p.half);
    };
    // sums of vectors [j0, j1) -> the lane's parts of sum (f x)^2 and sum g f x
    auto both = [&](int j0, int j1, float f) {
      float a = 0.f, b = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (j < j0 || j >= j1) continue;
        float v[16], d[16], w[16];
        values(x[j], v);
        gradient(j, d);
        weights(h0 + j * l.heads_a_vector, w);
#pragma unroll
        for (int e = 0; e < 16; ++e) { const float xf = v[e] * f; a = fmaf(xf, xf, a); b = fmaf(d[e] * w[e], xf, b); }
      }
      return make_float2(a, b);
    };
    auto reduce = [&](float2 s) { return make_float2(sum_of<NORM>(p, s.x, part, slot, warp, lane), sum_of<NORM>(p, s.y, part2, slot, warp, lane)); };
    Scale s{1.f, 1.f};
    float along = 0.f;
    auto settle = [&](int j0, int j1, float n, bool there) {
      float2 q = reduce(both(j0, j1, 1.f));
      const float mean = q.x / n + p.eps;
      s = {1.f, rsqrtf(mean)};
      const bool over = !(q.x <= MOST), under = there && mean < LEAST;
      if (any_of<NORM>(p, over || under)) {
        const float f = over ? DOWN : under ? UP : 1.f;
        q = reduce(both(j0, j1, f));
        s = {f, rsqrtf(q.x / n + p.eps * f * f)};
      }
      along = q.y * s.scale / n;                         // the mean of g n
    };
    if constexpr (ROW) settle(0, NV, (float)t.heads * (float)p.d, live);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int h = h0 + j * l.heads_a_vector;
      const bool there = live && l.in_head && h < t.heads;
      if constexpr (!ROW) settle(j, j + 1, (float)p.d, there);
      if (!there) continue;
      float v[16], d[16], w[16];
      values(x[j], v);
      gradient(j, d);
      weights(h, w);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float n = v[e] * s.factor * s.scale;
        acc[ROW ? j : 0][e] = fmaf(d[e], n, acc[ROW ? j : 0][e]);
        v[e] = (d[e] * w[e] - n * along) * s.scale * s.factor;
      }
      store(out + h * t.o.sh, l.second, v);
    }
  }
  if (t.part == nullptr) return;
  // rows (and heads) of the CTA in a fixed order, then its row of partial sums
  const int cols = ROW ? t.heads * p.d : p.d;
  if constexpr (!ROW) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      for (int o = 16; o >= 1 << p.lanes_log; o >>= 1) acc[0][e] += __shfl_xor_sync(0xffffffffu, acc[0][e], o);
  }
  for (int i = 0; i < per; ++i) {
    if (slot == i && l.in_head && (ROW || l.head == 0)) {
#pragma unroll
      for (int j = 0; j < NA; ++j) {
        const int h = ROW ? (fixed_piece * NV + j) * l.heads_a_vector + l.head : 0;
        if (ROW && h >= t.heads) continue;
        float* at = sums + (ROW ? h * p.d : 0) + l.e0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float* to = at + (e < 8 ? e : l.second + e - 8);
          *to = i == 0 ? acc[j][e] : *to + acc[j][e];
        }
      }
    }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < cols; c += THREADS) t.part[(long long)blockIdx.x * cols + c] = sums[c];
}

// The weights' gradient from the CTAs' rows of partial sums, in their order: 32 columns a CTA, 8 runs of rows side by side.
struct SumParams { const float* part[2]; void* out[2]; int cols[2]; int rows, f32; };
__global__ void __launch_bounds__(THREADS) turn_sum_kernel(const __grid_constant__ SumParams p) {
  griddep_launch();
  __shared__ float some[WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.y, c = blockIdx.x * 32 + lane, cols = i == 0 ? p.cols[0] : p.cols[1];
  griddep_wait();
  const float* part = i == 0 ? p.part[0] : p.part[1];
  void* out = i == 0 ? p.out[0] : p.out[1];
  if (part == nullptr || blockIdx.x * 32 >= cols) return;
  const int r0 = (int)((long long)p.rows * warp / WARPS), r1 = (int)((long long)p.rows * (warp + 1) / WARPS);
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int r = r0; r < r1; ++r) s += part[(long long)r * cols + c];
  }
  some[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < cols) {
    s = 0.f;
#pragma unroll
    for (int j = 0; j < WARPS; ++j) s += some[j][lane];
    if (p.f32) static_cast<float*>(out)[c] = s;
    else static_cast<bf*>(out)[c] = __float2bfloat16_rn(s);
  }
}

// ---------------------------------------------------------------- pair by pair
// Any size, stride and alignment: a warp takes a head (a CTA takes a row, where the norm is over rows), a lane a pair or an element that is not turned at a time.  The second
// pass reads what the first has brought into the caches.
struct Piece { int a, b; };                              // elements; b < 0: one alone
AS_DEV Piece piece_of(const TurnParams& p, int i) {
  if (i >= p.pairs) return {p.pairs + i, -1};
  return p.half ? Piece{i, i + p.pairs} : Piece{2 * i, 2 * i + 1};
}
AS_DEV float weight_of(const TurnParams& p, const void* w, int at) {
  return w == nullptr ? 1.f : p.w_f32 ? static_cast<const float*>(w)[at] : __bfloat162float(static_cast<const bf*>(w)[at]);
}

template <typename T, int NORM, bool BACK>
__global__ void __launch_bounds__(THREADS) turn_elements_kernel(const __grid_constant__ TurnParams p) {
  griddep_launch();
  __shared__ float part[WARPS], part2[WARPS];
  extern __shared__ float sums[];                        // backward: of the weights' gradient, a row of them for each warp or for the CTA
  constexpr bool ROW = NORM == AS_NORM_ROW;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int which = BACK ? blockIdx.y : 0, np = p.d - p.pairs;           // pieces of a head
  const int cols = ROW ? (which == 0 ? p.t[0] : p.t[1]).heads * p.d : p.d;
  float* mine = sums + (ROW ? 0 : warp * p.d);
  if constexpr (BACK) {
    for (int c = threadIdx.x; c < (ROW ? cols : WARPS * p.d); c += THREADS) sums[c] = 0.f;
    __syncthreads();
  }
  griddep_wait();
  // units: rows of q and of k, or heads of them; backward: of one tensor
  const long long per0 = ROW ? 1 : p.t[0].heads, per1 = ROW ? 1 : p.t[1].heads;
  const long long q_units = BACK ? (which == 0 ? p.rows * per0 : 0) : p.rows * per0;
  const long long units = BACK ? p.rows * (which == 0 ? per0 : per1) : q_units + (p.n_t == 2 ? p.rows * per1 : 0);
  const long long step = ROW ? gridDim.x : (long long)gridDim.x * WARPS;
  for (long long u = ROW ? (long long)blockIdx.x : (long long)blockIdx.x * WARPS + warp; u < units; u += step) {
    const bool first = u < q_units;
    const TurnTensor& t = first ? p.t[0] : p.t[1];
    const long long v = first ? u : u - q_units;
    const unsigned r = (unsigned)(ROW ? v : v / t.heads);
    const int h_of = ROW ? 0 : (int)(v - (long long)r * t.heads);
    const int pieces = ROW ? t.heads * np : np, from = ROW ? threadIdx.x : lane, by = ROW ? THREADS : 32;
    const T* x = static_cast<const T*>(t.x.data) + t.x.row(r);
    const T* y = BACK ? static_cast<const T*>(t.dy.data) + t.dy.row(r) : nullptr;
    T* out = static_cast<T*>(t.o.data) + t.o.row(r);
    const Where at = p.table != nullptr ? where_of(p, r) : Where{};
    auto sum = [&](float s, float* room) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if constexpr (ROW) {
        __syncthreads();
        if (lane == 0) room[warp] = s;
        __syncthreads();
        s = 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) s += room[i];
      }
      return s;
    };
    // d = R^T dy of a piece
    auto gradient = [&](int h, int i, const Piece& e, float& da, float& db) {
      da = (float)y[h * t.dy.sh + e.a];
      db = e.b < 0 ? 0.f : (float)y[h * t.dy.sh + e.b];
      if (e.b >= 0) {
        const float2 cs = factor_of(p, at, i);
        const float a = da;
        da = a * cs.x - db * cs.y;
        db = a * cs.y + db * cs.x;
      }
    };
    auto both = [&](float f) {
      float a = 0.f, b = 0.f;
      for (int i = from; i < pieces; i += by) {
        const int hh = ROW ? i / np : 0, h = h_of + hh, j = i - hh * np;
        const Piece e = piece_of(p, j);
        const float xa = (float)x[h * t.x.sh + e.a] * f, xb = e.b < 0 ? 0.f : (float)x[h * t.x.sh + e.b] * f;
        a = fmaf(xa, xa, fmaf(xb, xb, a));
        if constexpr (BACK) {
          float da, db;
          gradient(h, j, e, da, db);
          b = fmaf(da * weight_of(p, t.w, (ROW ? h * p.d : 0) + e.a), xa, b);
          if (e.b >= 0) b = fmaf(db * weight_of(p, t.w, (ROW ? h * p.d : 0) + e.b), xb, b);
        }
      }
      return make_float2(sum(a, part), BACK ? sum(b, part2) : 0.f);
    };
    Scale s{1.f, 1.f};
    float along = 0.f;
    if constexpr (NORM != AS_NORM_NONE) {
      const float n = ROW ? (float)t.heads * (float)p.d : (float)p.d;
      float2 q = both(1.f);
      const float mean = q.x / n + p.eps;
      s.scale = rsqrtf(mean);
      const bool over = !(q.x <= MOST), under = mean < LEAST;
      if (over || under) {                               // (one value for all that share the sum)
        const float f = over ? DOWN : UP;
        q = both(f);
        s = {f, rsqrtf(q.x / n + p.eps * f * f)};
      }
      along = q.y * s.scale / n;
    }
    for (int i = from; i < pieces; i += by) {
      const int hh = ROW ? i / np : 0, h = h_of + hh, j = i - hh * np;
      const Piece e = piece_of(p, j);
      const int wa = (ROW ? h * p.d : 0) + e.a, wb = (ROW ? h * p.d : 0) + max(e.b, 0);
      float a = (float)x[h * t.x.sh + e.a], b = e.b < 0 ? 0.f : (float)x[h * t.x.sh + e.b];
      if constexpr (NORM != AS_NORM_NONE) { a = a * s.factor * s.scale; b = b * s.factor * s.scale; }
      if constexpr (BACK) {
        float da, db;
        gradient(h, j, e, da, db);
        if (t.part != nullptr) {
          mine[wa] += da * a;                            // (a lane has the same elements in every unit)
          if (e.b >= 0) mine[wb] += db * b;
        }
        a = (da * weight_of(p, t.w, wa) - a * along) * s.scale * s.factor;
        b = (db * (e.b >= 0 ? weight_of(p, t.w, wb) : 0.f) - b * along) * s.scale * s.factor;
      } else {
        if constexpr (NORM != AS_NORM_NONE) {
          a *= weight_of(p, t.w, wa);
          if (e.b >= 0) b *= weight_of(p, t.w, wb);
        }
        if (e.b >= 0) {
          const float2 cs = factor_of(p, at, j);
          const float a0 = a;
          a = a0 * cs.x - b * cs.y;
          b = a0 * cs.y + b * cs.x;
        }
      }
      out[h * t.o.sh + e.a] = (T)a;
      if (e.b >= 0) out[h * t.o.sh + e.b] = (T)b;
    }
  }
  if constexpr (BACK) {
    const TurnTensor& t = which == 0 ? p.t[0] : p.t[1];
    if (t.part == nullptr) return;
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += THREADS) {
      float s = sums[c];
      if constexpr (!ROW)
        for (int w = 1; w < WARPS; ++w) s += sums[w * p.d + c];
      t.part[(long long)blockIdx.x * cols + c] = s;
    }
  }
}

// ---------------------------------------------------------------- host
as_status_t device_ok(int* sms) {
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return failed();
  return major == 10 ? AS_OK : AS_ERR_ARCH;
}

bool heads_ok(const as_rows_t& x, const as_qk_norm_rotary_t& a, int heads, bool out) {
  const long long cols = (long long)heads * a.head_dim;
  return rows_ok(x, a.rows, cols) && x.head_dim == a.head_dim && x.dtype == a.q.dtype && (a.rows == 0 || x.tokens == a.q.tokens) && (!out || apart(x, a.rows, cols));
}

as_status_t rotation_ok(const as_rotation_t& r, long long tokens, int d, int* total) {
  *total = 0;
  if (r.table == nullptr) return AS_OK;
  if (!aligned(r.table, 8) || r.n_axes < 1 || r.n_axes > AS_ROTARY_MAX_AXES || (r.layout != AS_ROTARY_INTERLEAVED && r.layout != AS_ROTARY_HALF) || (r.inverse != 0 && r.inverse != 1))
    return AS_ERR_INVALID_ARG;
  long long pairs = 0, rows = 0;
  __int128 grid = 1;
  for (int i = 0; i < r.n_axes; ++i) {
    if (r.size[i] < 1 || r.pairs[i] < 1) return AS_ERR_INVALID_ARG;
    pairs += r.pairs[i];
    rows += r.size[i];
    grid *= r.size[i];
  }
  if (2 * pairs > d || rows > 0x7fffffffll) return AS_ERR_INVALID_ARG;
  if (r.positions != nullptr) {
    if ((r.position_bytes != 4 && r.position_bytes != 8) || !aligned(r.positions, r.position_bytes) || r.positions_stride < 0) return AS_ERR_INVALID_ARG;
  } else {
    if (r.first < 0 || (__int128)r.first + tokens > grid) return AS_ERR_INVALID_ARG;
    if (r.first + tokens > 0xffffffffll) return AS_ERR_UNSUPPORTED;
  }
  *total = (int)pairs;
  return AS_OK;
}

// Checks of the arguments that both directions share.
as_status_t turn_ok(const as_qk_norm_rotary_t* a, bool back) {
  if (a == nullptr || a->struct_size != sizeof(as_qk_norm_rotary_t) || a->reserved != 0) return AS_ERR_INVALID_ARG;
  if (a->rows < 0 || a->rows > 0x7fffffffll || a->head_dim < 1 || a->head_dim > 1024 || a->norm < AS_NORM_NONE || a->norm > AS_NORM_ROW) return AS_ERR_INVALID_ARG;
  if (a->q_heads < 1 || a->q_heads > (1 << 20) || !heads_ok(a->q, *a, a->q_heads, false)) return AS_ERR_INVALID_ARG;
  const bool two = a->k.data != nullptr;
  if (two && (a->k_heads < 1 || a->k_heads > (1 << 20) || !heads_ok(a->k, *a, a->k_heads, false))) return AS_ERR_INVALID_ARG;
  if (!back && (two != (a->k_out.data != nullptr) || !heads_ok(a->q_out, *a, a->q_heads, true) || (two && !heads_ok(a->k_out, *a, a->k_heads, true)))) return AS_ERR_INVALID_ARG;
  if (a->norm != AS_NORM_NONE) {
    if (!(a->eps >= 0.f) || (a->weight_dtype != AS_DTYPE_BF16 && a->weight_dtype != AS_DTYPE_F32)) return AS_ERR_INVALID_ARG;
    const int size = a->weight_dtype == AS_DTYPE_BF16 ? 2 : 4;
    if (!aligned(a->q_weight, size) || !aligned(a->k_weight, size)) return AS_ERR_INVALID_ARG;
  }
  int pairs;
  if (const as_status_t s = rotation_ok(a->rotation, a->rows > 0 ? a->q.tokens : 0, a->head_dim, &pairs); s != AS_OK) return s;
  if (a->norm == AS_NORM_ROW && (long long)std::max(a->q_heads, two ? a->k_heads : 0) * a->head_dim > 16384) return AS_ERR_UNSUPPORTED;
  return AS_OK;
}

// Whether pieces of 8 elements move 16 bytes at a time.
bool heads_vec(const as_rows_t& x) { return aligned(x.data, 16) && ((x.stride_batch | x.stride_head | x.stride_token) & (x.dtype == AS_DTYPE_BF16 ? 7 : 3)) == 0; }

struct Shape { bool vec; int NV, chunks; long long ctas; };
// Fills in what the kernels share; `most`: vectors that a lane's registers hold.
Shape turn_params(const as_qk_norm_rotary_t& a, const as_rotation_t& r, int sms, bool back, const as_rows_t* more, int n_more, TurnParams& p) {
  const bool two = a.k.data != nullptr;
  int pairs;
  rotation_ok(r, 0, a.head_dim, &pairs);
  p.n_t = two ? 2 : 1;
  p.rows = (int)a.rows; p.tokens = (int)a.q.tokens; p.d = a.head_dim;
  p.eps = a.eps;
  p.w_f32 = a.weight_dtype == AS_DTYPE_F32;
  p.t[0].heads = a.q_heads;
  p.t[1].heads = two ? a.k_heads : 0;
  p.t[0].x = rows_of(a.q, a.rows, (long long)a.q_heads * a.head_dim);
  if (two) p.t[1].x = rows_of(a.k, a.rows, (long long)a.k_heads * a.head_dim);
  if (a.norm != AS_NORM_NONE) { p.t[0].w = a.q_weight; p.t[1].w = two ? a.k_weight : nullptr; }
  p.table = reinterpret_cast<const float2*>(r.table);
  p.pairs = pairs;
  if (p.table != nullptr) {
    p.axes = r.n_axes;
    p.half = r.layout == AS_ROTARY_HALF;
    p.sign = (r.inverse != 0) != back ? -1.f : 1.f;
    p.pos = r.positions; p.pos64 = r.position_bytes == 8; p.pos_stride = r.positions_stride; p.first = r.first;
    int rows = 0, end = 0;
    for (int i = 0; i < AS_ROTARY_MAX_AXES; ++i) {
      p.first_row[i] = rows;
      if (i < r.n_axes) { p.size[i] = r.size[i]; rows += r.size[i]; end += r.pairs[i]; }
      p.end[i] = end;
    }
  }
  Shape s{};
  s.vec = a.head_dim % 16 == 0 && a.head_dim <= 512 && pairs % 8 == 0 && aligned(r.table, 16) && heads_vec(a.q) && (!two || heads_vec(a.k));
  for (int i = 0; i < n_more; ++i) s.vec = s.vec && (more[i].data == nullptr || heads_vec(more[i]));
  if (a.norm != AS_NORM_NONE) s.vec = s.vec && aligned(a.q_weight, 16) && (!two || aligned(a.k_weight, 16));
  p.lanes_log = 0;
  while ((16 << p.lanes_log) < a.head_dim) ++p.lanes_log;
  const int heads = std::max(p.t[0].heads, p.t[1].heads), of_vector = std::max(1, 32 >> p.lanes_log), vectors = (heads + of_vector - 1) / of_vector;
  const int most = back ? (a.q.dtype == AS_DTYPE_BF16 ? 3 : 2) : 3;
  p.W = 1; p.chunks = 1;
  if (a.norm == AS_NORM_ROW) {
    p.W = (vectors + most - 1) / most;
    if (p.W > WARPS) s.vec = false;
    else s.NV = (vectors + p.W - 1) / p.W;
    s.ctas = s.vec ? (a.rows + WARPS / p.W - 1) / (WARPS / p.W) : a.rows * (back ? 1 : p.n_t);
  } else {
    // few rows: a vector a warp, so that all of them are under way at once
    s.NV = a.rows * ((vectors + most - 1) / most) <= 4ll * sms ? 1 : std::min(vectors, most);
    p.chunks = (vectors + s.NV - 1) / s.NV;
    const long long units = s.vec ? a.rows * p.chunks : a.rows * (back ? heads : (long long)p.t[0].heads + p.t[1].heads);
    s.ctas = (units + WARPS - 1) / WARPS;
  }
  return s;
}

template <typename T, int NORM>
cudaError_t launch_turn(const TurnParams& p, const Shape& s, int sms, cudaStream_t st) {
  if (!s.vec) return as_launch_dependent(turn_elements_kernel<T, NORM, false>, dim3((unsigned)std::min<long long>(s.ctas, 8ll * sms)), dim3(THREADS), 0, st, p);
  const dim3 grid((unsigned)s.ctas), block(THREADS);
  switch (s.NV) {
    case 1: return as_launch_dependent(turn_kernel<T, NORM, 1>, grid, block, 0, st, p);
    case 2: return as_launch_dependent(turn_kernel<T, NORM, 2>, grid, block, 0, st, p);
    default: return as_launch_dependent(turn_kernel<T, NORM, 3>, grid, block, 0, st, p);
  }
}
template <typename T>
cudaError_t launch_norm(const TurnParams& p, const Shape& s, int norm, int sms, cudaStream_t st) {
  return norm == AS_NORM_NONE ? launch_turn<T, AS_NORM_NONE>(p, s, sms, st) : norm == AS_NORM_HEAD ? launch_turn<T, AS_NORM_HEAD>(p, s, sms, st) : launch_turn<T, AS_NORM_ROW>(p, s, sms, st);
}

template <typename T, int NORM>
cudaError_t launch_back(const TurnParams& p, const Shape& s, unsigned ctas, size_t smem, cudaStream_t st) {
  const dim3 grid(ctas, (unsigned)p.n_t), block(THREADS);
  auto run = [&](auto kernel) {
    if (smem > 48 * 1024)
      if (const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); e != cudaSuccess) return e;
    return as_launch_dependent(kernel, grid, block, smem, st, p);
  };
  if (!s.vec) return run(turn_elements_kernel<T, NORM, true>);
  if constexpr (sizeof(T) == 2)
    if (s.NV == 3) return run(turn_back_kernel<T, NORM, 3>);
  return s.NV == 2 ? run(turn_back_kernel<T, NORM, 2>) : run(turn_back_kernel<T, NORM, 1>);
}

// CTAs of the backward pass, for each tensor: as many as the device holds at once.
unsigned back_ctas(const Shape& s, int sms) { return (unsigned)std::min<long long>(s.ctas, 2ll * sms); }

// The rows of the backward call that the shape looks at beside the inputs.
int back_rows(const as_qk_norm_rotary_backward_t& b, as_rows_t (&more)[4]) {
  more[0] = b.dq; more[1] = b.dq_out; more[2] = b.dk; more[3] = b.dk_out;
  return 4;
}
as_status_t back_ok(const as_qk_norm_rotary_backward_t* b) {
  if (b == nullptr || b->struct_size != sizeof(as_qk_norm_rotary_backward_t) || b->reserved != 0) return AS_ERR_INVALID_ARG;
  if (const as_status_t s = turn_ok(b->fwd, true); s != AS_OK) return s;
  const as_qk_norm_rotary_t& a = *b->fwd;
  if (a.norm == AS_NORM_NONE) return AS_ERR_INVALID_ARG;
  const bool two = a.k.data != nullptr;
  if (!heads_ok(b->dq, a, a.q_heads, false) || !heads_ok(b->dq_out, a, a.q_heads, true)) return AS_ERR_INVALID_ARG;
  if (two != (b->dk.data != nullptr) || two != (b->dk_out.data != nullptr) || (two && (!heads_ok(b->dk, a, a.k_heads, false) || !heads_ok(b->dk_out, a, a.k_heads, true)))) return AS_ERR_INVALID_ARG;
  const int size = a.weight_dtype == AS_DTYPE_BF16 ? 2 : 4;
  if ((b->dq_weight != nullptr && (a.q_weight == nullptr || !aligned(b->dq_weight, size))) || (b->dk_weight != nullptr && (!two || a.k_weight == nullptr || !aligned(b->dk_weight, size))))
    return AS_ERR_INVALID_ARG;
  return AS_OK;
}
uint64_t back_bytes(const as_qk_norm_rotary_backward_t& b, unsigned ctas, long long (&cols)[2]) {
  const as_qk_norm_rotary_t& a = *b.fwd;
  cols[0] = b.dq_weight == nullptr ? 0 : a.norm == AS_NORM_ROW ? (long long)a.q_heads * a.head_dim : a.head_dim;
  cols[1] = b.dk_weight == nullptr ? 0 : a.norm == AS_NORM_ROW ? (long long)a.k_heads * a.head_dim : a.head_dim;
  return (uint64_t)ctas * (uint64_t)(cols[0] + cols[1]) * 4;
}

}  // namespace

extern "C" as_status_t as_rotary_table(const as_rotary_axis_t* axes, int32_t n_axes, float* table, void* cuda_stream) {
  if (axes == nullptr || n_axes < 1 || n_axes > AS_ROTARY_MAX_AXES || table == nullptr || !aligned(table, 16)) return AS_ERR_INVALID_ARG;
  TableParams p{};
  long long rows = 0, pairs = 0;
  for (int i = 0; i < n_axes; ++i) {
    const as_rotary_axis_t& x = axes[i];
    if (x.size < 1 || x.pairs < 1 || x.reserved != 0 || x.scaling < AS_ROTARY_PLAIN || x.scaling > AS_ROTARY_YARN || !(x.base > 0.) || !std::isfinite(x.base)) return AS_ERR_INVALID_ARG;
    if (x.scaling != AS_ROTARY_PLAIN && (!(x.factor >= 1.) || !std::isfinite(x.factor))) return AS_ERR_INVALID_ARG;
    if (x.scaling == AS_ROTARY_YARN && (!(x.original > 0.) || !std::isfinite(x.original))) return AS_ERR_INVALID_ARG;
    p.axis[i] = TableAxis{0., 1., x.base, x.factor, x.original, x.scaling, x.pairs, (int)rows, (int)pairs};
    rows += x.size;
    pairs += x.pairs;
    if (rows > 0x7fffffffll || pairs > 8192) return AS_ERR_UNSUPPORTED;
  }
  int sms;
  if (const as_status_t s = device_ok(&sms); s != AS_OK) return s;
  p.out = reinterpret_cast<float2*>(table);
  p.rows = (int)rows; p.pairs = (int)pairs; p.axes = n_axes;
  const dim3 grid((unsigned)((rows + TABLE_ROWS - 1) / TABLE_ROWS), (unsigned)((pairs + 63) / 64));
  return as_launch_dependent(table_kernel, grid, dim3(THREADS), 0, static_cast<cudaStream_t>(cuda_stream), p) == cudaSuccess ? AS_OK : failed();
}

extern "C" as_status_t as_qk_norm_rotary(const as_qk_norm_rotary_t* a, void* cuda_stream) {
  if (const as_status_t s = turn_ok(a, false); s != AS_OK) return s;
  if (a->rows == 0) return AS_OK;
  int sms;
  if (const as_status_t s = device_ok(&sms); s != AS_OK) return s;
  TurnParams p{};
  const as_rows_t more[2] = {a->q_out, a->k_out};
  const Shape s = turn_params(*a, a->rotation, sms, false, more, 2, p);
  p.t[0].o = rows_of(a->q_out, a->rows, (long long)a->q_heads * a->head_dim);
  if (p.n_t == 2) p.t[1].o = rows_of(a->k_out, a->rows, (long long)a->k_heads * a->head_dim);
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (s.ctas > 0x7fffffffll) return AS_ERR_UNSUPPORTED;
  const cudaError_t e = a->q.dtype == AS_DTYPE_BF16 ? launch_norm<bf>(p, s, a->norm, sms, st) : launch_norm<float>(p, s, a->norm, sms, st);
  return e == cudaSuccess ? AS_OK : failed();
}

extern "C" as_status_t as_qk_norm_rotary_backward_workspace_bytes(const as_qk_norm_rotary_backward_t* b, uint64_t* bytes) {
  if (bytes == nullptr) return AS_ERR_INVALID_ARG;
  if (const as_status_t s = back_ok(b); s != AS_OK) return s;
  *bytes = 0;
  if (b->fwd->rows == 0) return AS_OK;
  int sms;
  if (const as_status_t s = device_ok(&sms); s != AS_OK) return s;
  TurnParams p{};
  as_rows_t more[4];
  long long cols[2];
  const Shape s = turn_params(*b->fwd, b->fwd->rotation, sms, true, more, back_rows(*b, more), p);
  *bytes = back_bytes(*b, back_ctas(s, sms), cols);
  return AS_OK;
}

extern "C" as_status_t as_qk_norm_rotary_backward(const as_qk_norm_rotary_backward_t* b, void* cuda_stream) {
  if (const as_status_t s = back_ok(b); s != AS_OK) return s;
  const as_qk_norm_rotary_t& a = *b->fwd;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int size = a.weight_dtype == AS_DTYPE_BF16 ? 2 : 4;
  long long cols[2];
  int sms;
  if (const as_status_t s = device_ok(&sms); s != AS_OK) return s;
  if (a.rows == 0) {                                     // sums over nothing
    back_bytes(*b, 0, cols);
    if (cols[0] > 0 && cudaMemsetAsync(b->dq_weight, 0, (size_t)(cols[0] * size), st) != cudaSuccess) return failed();
    if (cols[1] > 0 && cudaMemsetAsync(b->dk_weight, 0, (size_t)(cols[1] * size), st) != cudaSuccess) return failed();
    return AS_OK;
  }
  TurnParams p{};
  as_rows_t more[4];
  const Shape s = turn_params(a, a.rotation, sms, true, more, back_rows(*b, more), p);
  const unsigned ctas = back_ctas(s, sms);
  const uint64_t need = back_bytes(*b, ctas, cols);
  if (need > 0 && (b->workspace == nullptr || !aligned(b->workspace, 16) || b->workspace_bytes < need)) return AS_ERR_WORKSPACE;
  float* part = static_cast<float*>(b->workspace);
  const as_rows_t* dy[2] = {&b->dq, &b->dk};
  const as_rows_t* out[2] = {&b->dq_out, &b->dk_out};
  void* dw[2] = {b->dq_weight, b->dk_weight};
  SumParams sum{};
  size_t smem = 0;
  for (int i = 0; i < p.n_t; ++i) {
    const long long wide = (long long)p.t[i].heads * a.head_dim;
    p.t[i].dy = rows_of(*dy[i], a.rows, wide);
    p.t[i].o = rows_of(*out[i], a.rows, wide);
    if (cols[i] > 0) { p.t[i].part = part; sum.part[i] = part; sum.out[i] = dw[i]; sum.cols[i] = (int)cols[i]; part += ctas * cols[i]; }
    smem = std::max(smem, (size_t)(a.norm == AS_NORM_ROW ? wide : s.vec ? a.head_dim : WARPS * a.head_dim) * 4);
  }
  cudaError_t e;
  if (a.q.dtype == AS_DTYPE_BF16) e = a.norm == AS_NORM_HEAD ? launch_back<bf, AS_NORM_HEAD>(p, s, ctas, smem, st) : launch_back<bf, AS_NORM_ROW>(p, s, ctas, smem, st);
  else e = a.norm == AS_NORM_HEAD ? launch_back<float, AS_NORM_HEAD>(p, s, ctas, smem, st) : launch_back<float, AS_NORM_ROW>(p, s, ctas, smem, st);
  if (e == cudaSuccess && cols[0] + cols[1] > 0) {
    sum.rows = (int)ctas;
    sum.f32 = a.weight_dtype == AS_DTYPE_F32;
    e = as_launch_dependent(turn_sum_kernel, dim3((unsigned)((std::max(cols[0], cols[1]) + 31) / 32), 2), dim3(THREADS), 0, st, sum);
  }
  return e == cudaSuccess ? AS_OK : failed();
}
