// Norms of queries and keys, their rotation by the tokens' positions, and the gradients of both.
//
// All of it reads a tensor once and writes it once: bound by HBM bytes.  A lane holds 16 elements of a head (8, where 16 do not fit) in two pieces, one of each half of what is turned or of
// what is not: both elements of a pair are its own in either layout, and the lanes of a head move runs of 128 bytes.  The lanes of a head are a power of two, so that a head's sum is a few exchanges; a warp
// holds 32 / lanes heads a vector and NV vectors, and where the norm is over a token's heads up to 8 warps hold a row.  Rows come to shared memory by asynchronous copies, a row ahead of the one that is
// worked on, and so do a token's cos and sin, which are the same for every head and for queries and keys.  Three vectors a lane: what a row costs once (positions, addresses, factors) is a third of the whole
// with one (81 frames by heads: 106 us with one, 104 with two, 74 with three).  Heads whose sizes, strides or addresses do not allow it go pair by pair (turn_elements_kernel).
//
// The kernels alone: 32760 tokens of 2 x 12 heads of 128 in bf16, from the fused projection's rows into heads, norm by heads: 74 us, 5.4 TB/s; its gradient 111 us, 5.4 TB/s (calls one after another 78 and
// 121).  In fp32 235 us, 3.4 TB/s, and 354 (one CTA an SM).  7800 tokens, norm over rows: 24 us, 3.9 TB/s (3.3 rows a warp, each of which is a chain of latencies), its gradient 55 us (issue slots
// used 38 % with 14 warps an SM; of 7.8 cycles between a warp's instructions 2.2 wait for memory, 1.3 for an instruction before, 1.0 for shared memory, which the rows are read from twice).
#include <algorithm>
#include <atomic>
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
struct TableAxis { double base, factor, original; int scaling, pairs, first_row, first_pair; };
struct TableParams {
  float2* out;
  int rows, pairs, axes;
  TableAxis axis[AS_ROTARY_MAX_AXES];
};
constexpr int TABLE_ROWS = 64;                 // of a CTA

// A thread has one pair and walks over rows: its angle a position is taken once, in 64 bits.  cos and sin are those of what is left behind the next multiple of a quarter turn, whose
// rounding to fp32 is relative to it.  (With turns in fp64, whose conversions are slow, 65536 positions of 32 pairs took 14 us.)
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
  // a position's angle in turns, as a fraction of 2^64: positions times it, and the turns that are dropped, are exact
  f /= tau;
  const unsigned long long step = (unsigned long long)((f - floor(f)) * 18446744073709551616.);
  const int end = a + 1 < p.axes ? p.axis[min(a + 1, AS_ROTARY_MAX_AXES - 1)].first_row : p.rows;
  griddep_wait();
  const int row0 = blockIdx.x * TABLE_ROWS, n = min(TABLE_ROWS, p.rows - row0);       // (row0 + TABLE_ROWS may lie past 2^31)
  for (int j = threadIdx.x / 64; j < n; j += THREADS / 64) {
    const int r = row0 + j;
    float2 v = make_float2(0.f, 0.f);
    if (r >= x.first_row && r < end) {
      const unsigned long long turns = (unsigned long long)(r - x.first_row) * step, q = (turns + (1ull << 61)) >> 62;       // the next multiple of a quarter turn
      float s, c;
      sincospif(ldexpf((float)(long long)(turns - (q << 62)), -63), &s, &c);
      const float cc = q & 1 ? s : c, ss = q & 1 ? c : s;
      v.x = (q == 1 || q == 2 ? -cc : cc) * (float)amplitude;
      v.y = (q >= 2 ? -ss : ss) * (float)amplitude;
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
  unsigned long long by_size[AS_ROTARY_MAX_AXES], by_tokens;       // 2^64 / n, rounded up (0: n is 1): a quotient is the upper half of a product, exact below 2^32
  float sign;                                // of sin
  float over_n[2];                           // 1 / elements that a sum of squares goes over, of either tensor
  int w_f32;
  int lanes_log;                             // lanes of a head: 2^lanes_log
  int W;                                     // warps of a row
  int chunks;                                // runs of heads that a warp takes at once, where the norm is not over rows
  int room;                                  // bytes of a warp's factors: chunks of two pairs, in whole groups of eight
  int kept;                                  // rows' weights are kept in shared memory: bytes of the first tensor's (0: they are not)
};
AS_DEV unsigned quotient(unsigned i, unsigned long long by) { return by == 0ull ? i : (unsigned)__umul64hi(by, i); }
struct Token { unsigned b, t; };
AS_DEV Token token_of(const TurnParams& p, unsigned r) {
  const unsigned b = p.tokens == p.rows ? 0u : quotient(r, p.by_tokens);
  return {b, r - b * (unsigned)p.tokens};
}
AS_DEV long long address(const Rows& m, const Token& k) { return (long long)k.b * m.sb + (long long)k.t * m.st; }

struct Where { int at[AS_ROTARY_MAX_AXES]; };
// Rows of the table for row r; -1: no such position.
AS_DEV Where where_of(const TurnParams& p, const Token& k) {
  Where w{};
  const unsigned b = k.b, t = k.t;
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
        const unsigned q = quotient(i, p.by_size[a]);
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
// A token's cos and sin in its warp's shared memory, two pairs (16 bytes) a lane, asked for a row ahead: read by every lane from the table they were 100 instructions and two waits a row.
// Chunks of two pairs lie so that the lanes of a head, which read one of every two or four, meet no bank twice (within their group of eight).
AS_DEV uint32_t chunk_at(uint32_t room, int c) { return room + (uint32_t)((c ^ (c >> 3 & 7)) << 4); }
AS_DEV void ask_factors(const TurnParams& p, const Where& w, uint32_t room, int lane) {
  for (int pair = 2 * lane; pair < p.pairs; pair += 64) {
    const int a = pick(w, axis_of(p, pair)), b = pick(w, axis_of(p, pair + 1));
    const uint32_t to = chunk_at(room, pair / 2);
    if (a == b && a >= 0) {
      asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(to), "l"(p.table + (long long)a * p.pairs + pair) : "memory");
    } else {
      auto one = [&](uint32_t at, int row, int i) {
        if (row >= 0) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(at), "l"(p.table + (long long)row * p.pairs + i) : "memory");
        else asm volatile("st.shared.v2.u32 [%0], {%1, %1};" ::"r"(at), "r"(0x7fc00000u) : "memory");
      };
      one(to, a, pair);
      one(to + 8, b, pair + 1);
    }
  }
}

// ---------------------------------------------------------------- vectors of a lane
// E elements of a head (16, or 8) as the first and the second elements of E / 2 pairs, two pairs a register pair: arithmetic goes two values at a time.
template <int E> struct PairsOf { float2 a[E / 4], b[E / 4]; };
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
AS_DEV float2 both(float x) { return make_float2(x, x); }
AS_DEV float2 sub2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tsub.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
template <int E>
AS_DEV void scale(PairsOf<E>& v, float2 f) {
#pragma unroll
  for (int i = 0; i < E / 4; ++i) { v.a[i] = mul2(v.a[i], f); v.b[i] = mul2(v.b[i], f); }
}
template <int E>
AS_DEV void scale(PairsOf<E>& v, const PairsOf<E>& w) {
#pragma unroll
  for (int i = 0; i < E / 4; ++i) { v.a[i] = mul2(v.a[i], w.a[i]); v.b[i] = mul2(v.b[i], w.b[i]); }
}
template <int E>
AS_DEV float2 dot(const PairsOf<E>& v, const PairsOf<E>& w, float2 s) {
#pragma unroll
  for (int i = 0; i < E / 4; ++i) { s = fma2(v.a[i], w.a[i], s); s = fma2(v.b[i], w.b[i], s); }
  return s;
}

// A lane's E elements as they lie: two pieces of E / 2, in words, and in what moves at once: 16 bytes, or 8 (8 elements in bf16).
template <typename T, int E> struct Raw { uint32_t w[E * sizeof(T) / 4]; };
template <typename T, int E> constexpr int PIECE = E / 2 * (int)sizeof(T);          // bytes of a piece
template <typename T, int E> constexpr int MOVE = PIECE<T, E> < 16 ? 8 : 16;         // bytes that move at once
template <typename T, int E> constexpr int MOVES = E * (int)sizeof(T) / MOVE<T, E>;  // of a lane's elements
// Where move i begins: elements behind the first piece's first one.
template <typename T, int E>
AS_DEV int element_of(int i, int second) { return (i < MOVES<T, E> / 2 ? 0 : second) + i % (MOVES<T, E> / 2) * (MOVE<T, E> / (int)sizeof(T)); }
template <int BYTES>
AS_DEV void read_shared(uint32_t at, uint32_t* w) {
  if constexpr (BYTES == 16) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
  else asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
}
template <int BYTES>
AS_DEV void copy_shared(uint32_t to, const void* from) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
template <int BYTES>
AS_DEV void clear_shared(uint32_t to) {
  if constexpr (BYTES == 16) asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0) : "memory");
  else asm volatile("st.shared.v2.u32 [%0], {%1, %1};" ::"r"(to), "r"(0) : "memory");
}
// HALF: the pieces are the first and the second elements of E / 2 pairs; else each is E / 4 pairs.  (What is not turned may be called either.)
template <bool HALF, typename T, int E>
AS_DEV void values(const Raw<T, E>& r, PairsOf<E>& f) {
  const uint32_t* w = r.w;
  auto lo = [](uint32_t x) { return __uint_as_float(x << 16); };
  auto hi = [](uint32_t x) { return __uint_as_float(x & 0xffff0000u); };
#pragma unroll
  for (int i = 0; i < E / 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      if constexpr (HALF) { f.a[i] = make_float2(lo(w[i]), hi(w[i])); f.b[i] = make_float2(lo(w[E / 4 + i]), hi(w[E / 4 + i])); }
      else { f.a[i] = make_float2(lo(w[2 * i]), lo(w[2 * i + 1])); f.b[i] = make_float2(hi(w[2 * i]), hi(w[2 * i + 1])); }
    } else {
      auto at = [&](int j) { return __uint_as_float(w[j]); };
      if constexpr (HALF) { f.a[i] = make_float2(at(2 * i), at(2 * i + 1)); f.b[i] = make_float2(at(E / 2 + 2 * i), at(E / 2 + 1 + 2 * i)); }
      else { f.a[i] = make_float2(at(4 * i), at(4 * i + 2)); f.b[i] = make_float2(at(4 * i + 1), at(4 * i + 3)); }
    }
  }
}
template <bool HALF, typename T, int E>
AS_DEV void store(T* at, int second, const PairsOf<E>& f) {
  uint32_t w[E * sizeof(T) / 4];
#pragma unroll
  for (int i = 0; i < E / 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      if constexpr (HALF) { w[i] = sm100::pack_bf16(f.a[i].x, f.a[i].y); w[E / 4 + i] = sm100::pack_bf16(f.b[i].x, f.b[i].y); }
      else { w[2 * i] = sm100::pack_bf16(f.a[i].x, f.b[i].x); w[2 * i + 1] = sm100::pack_bf16(f.a[i].y, f.b[i].y); }
    } else {
      auto put = [&](int j, float x) { w[j] = __float_as_uint(x); };
      if constexpr (HALF) { put(2 * i, f.a[i].x); put(2 * i + 1, f.a[i].y); put(E / 2 + 2 * i, f.b[i].x); put(E / 2 + 1 + 2 * i, f.b[i].y); }
      else { put(4 * i, f.a[i].x); put(4 * i + 1, f.b[i].x); put(4 * i + 2, f.a[i].y); put(4 * i + 3, f.b[i].y); }
    }
  }
#pragma unroll
  for (int i = 0; i < MOVES<T, E>; ++i) {
    T* to = at + element_of<T, E>(i, second);
    const uint32_t* x = w + i * (MOVE<T, E> / 4);
    if constexpr (MOVE<T, E> == 16) *reinterpret_cast<uint4*>(to) = make_uint4(x[0], x[1], x[2], x[3]);
    else *reinterpret_cast<uint2*>(to) = make_uint2(x[0], x[1]);
  }
}
// KEPT: from shared memory, at the address `kept`.
template <bool HALF, bool KEPT, typename W, int E>
AS_DEV void load_weights_of(const W* w, uint32_t kept, int at, int second, PairsOf<E>& f) {
  Raw<W, E> r;
#pragma unroll
  for (int i = 0; i < MOVES<W, E>; ++i) {
    const int e = at + element_of<W, E>(i, second);
    uint32_t* to = r.w + i * (MOVE<W, E> / 4);
    if constexpr (KEPT) read_shared<MOVE<W, E>>(kept + (uint32_t)e * (uint32_t)sizeof(W), to);
    else if constexpr (MOVE<W, E> == 16) *reinterpret_cast<uint4*>(to) = __ldg(reinterpret_cast<const uint4*>(w + e));
    else *reinterpret_cast<uint2*>(to) = __ldg(reinterpret_cast<const uint2*>(w + e));
  }
  values<HALF>(r, f);
}
template <bool HALF, bool KEPT, int E>
AS_DEV void load_weights(const TurnParams& p, const void* w, uint32_t kept, int at, int second, PairsOf<E>& f) {
  if (p.w_f32) load_weights_of<HALF, KEPT>(static_cast<const float*>(w), kept, at, second, f);
  else load_weights_of<HALF, KEPT>(static_cast<const bf*>(w), kept, at, second, f);
}
// A row's weights to shared memory, by the whole CTA, which meets behind it.
AS_DEV void keep_weights(const TurnParams& p, const TurnTensor& t, uint8_t* to) {
  if (t.w == nullptr) return;
  const int n = t.heads * p.d * (p.w_f32 ? 4 : 2) / 16;
  for (int i = threadIdx.x; i < n; i += THREADS) reinterpret_cast<uint4*>(to)[i] = __ldg(static_cast<const uint4*>(t.w) + i);
}
// cos and sin of a lane's E / 2 pairs.
template <int E> struct FactorsOf { float2 c[E / 4], s[E / 4]; };
template <bool HALF, int E>
AS_DEV FactorsOf<E> factors_of(const TurnParams& p, uint32_t room, int slot) {
  FactorsOf<E> t;
#pragma unroll
  for (int i = 0; i < E / 4; ++i) {                      // chunks of two pairs
    const int c = HALF ? slot * (E / 4) + i : i < E / 8 ? slot * (E / 8) + i : p.pairs / 4 + slot * (E / 8) + i - E / 8;
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(chunk_at(room, c)) : "memory");
    t.c[i] = make_float2(v.x, v.z);
    t.s[i] = mul2(make_float2(v.y, v.w), both(p.sign));
  }
  return t;
}
// Behind the copies that this thread has asked for, and, where the factors are among them, those of its warp.
AS_DEV void wait_copies() { asm volatile("cp.async.wait_all;" ::: "memory"); }
template <int E>
AS_DEV void turn(PairsOf<E>& v, const FactorsOf<E>& f) {
#pragma unroll
  for (int i = 0; i < E / 4; ++i) {
    const float2 a = v.a[i], b = v.b[i];
    v.a[i] = sub2(mul2(a, f.c[i]), mul2(b, f.s[i]));
    v.b[i] = fma2(a, f.s[i], mul2(b, f.c[i]));
  }
}

// What a lane works on: its head of vector 0, elements of a head, whether they are turned.
struct Lane { int head, heads_a_vector, slot, e0, second; bool in_head, turned; };
template <int E>
AS_DEV Lane lane_of(const TurnParams& p, int lane) {
  Lane l;
  l.slot = lane & ((1 << p.lanes_log) - 1);
  l.head = lane >> p.lanes_log;
  l.heads_a_vector = 32 >> p.lanes_log;
  l.in_head = l.slot * E < p.d;
  l.turned = l.slot * (E / 2) < p.pairs;
  l.e0 = l.turned ? l.slot * (E / 2) : p.pairs + l.slot * (E / 2);       // what is not turned begins at 2 P, its slots at 2 P / E
  l.second = l.turned ? p.pairs : (p.d - 2 * p.pairs) / 2;
  return l;
}

// Sums over a head's lanes, or over a row's lanes and warps (in the order of the warps), N at once.
template <int NORM, int N>
AS_DEV void sums_of(const TurnParams& p, float (&s)[N], float (&part)[N][WARPS], int slot, int warp, int lane) {
#pragma unroll
  for (int k = 4; k >= 0; --k) {
    if (NORM == AS_NORM_HEAD && k >= p.lanes_log) continue;
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], 1 << k);
  }
  if constexpr (NORM == AS_NORM_ROW)
    if (p.W > 1) {                             // the same for every thread of the launch
      __syncthreads();                         // the sums before these have been read
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (lane == 0) part[i][warp] = s[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s[i] = 0.f;
        for (int w = 0; w < p.W; ++w) s[i] += part[i][min(slot * p.W + w, WARPS - 1)];
      }
    }
}
// Whether any lane that takes part in the same exchanges asks for it.
template <int NORM>
AS_DEV bool any_of(const TurnParams& p, bool ask) {
  if constexpr (NORM == AS_NORM_ROW)
    if (p.W > 1) return __syncthreads_or(ask);
  return __any_sync(0xffffffffu, ask);
}
// The normed value is x * factor * scale; factor is 1 but for rows whose squares fp32 does not hold, or whose squares vanish together with eps: those are summed again times a power
// of two.
AS_DEV bool over(float sum) { return !(sum <= MOST); }
AS_DEV float factor_for(float sum, float over_n, float eps, bool there) { return over(sum) ? DOWN : there && fmaf(sum, over_n, eps) < LEAST ? UP : 1.f; }

// ---------------------------------------------------------------- forward
// A warp holds a row of queries and one of keys (or pieces of them) at once.  What counts beside the bytes is the number of instructions: one value at a time, each vector of 16 elements a
// lane took 340 of them, and 32760 tokens of 2 x 12 heads 106 us.
template <typename T, int NORM, int NV, bool HALF, int E>
__global__ void __launch_bounds__(THREADS, 2) turn_kernel(const __grid_constant__ TurnParams p) {
  typedef PairsOf<E> Pairs;
  typedef FactorsOf<E> Factors;
  griddep_launch();
  __shared__ float part[1][WARPS];
  extern __shared__ uint4 dynamic[];                     // factors of each warp's row; weights of both tensors
  constexpr bool ROW = NORM == AS_NORM_ROW;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = ROW ? WARPS / p.W : WARPS, slot = ROW ? warp / p.W : warp, piece = ROW ? warp - slot * p.W : (int)blockIdx.y;
  const Lane l = lane_of<E>(p, lane);
  const int h0 = piece * NV * l.heads_a_vector + l.head;
  long long row = (long long)blockIdx.x * per + slot;
  bool live = slot < per && row < p.rows;
  Token k = token_of(p, live ? (unsigned)row : 0u);
  // rows of both tensors, in this lane's own pieces of 16 bytes: the next row's are asked for as soon as this one's have been read for the last time
  constexpr int PIECES = MOVES<T, E>, STEP = 32 * MOVE<T, E>;            // moves of a vector, bytes of one by a warp
  const uint32_t rows_at = sm100::smem_u32(dynamic) + (uint32_t)(warp * (NV * 2 * PIECES * STEP) + lane * MOVE<T, E>);
  const uint32_t room = sm100::smem_u32(dynamic) + (uint32_t)(WARPS * (NV * 2 * PIECES * STEP) + warp * p.room);
  uint8_t* kept = reinterpret_cast<uint8_t*>(dynamic) + WARPS * (NV * 2 * PIECES * STEP + p.room);
  auto place = [&](int i, int j, int piece) { return rows_at + (uint32_t)(((i * NV + j) * PIECES + piece) * STEP); };
  auto ask = [&](const TurnTensor& t, int i, int j, const T* base) {
    const int h = h0 + j * l.heads_a_vector;
    if (!l.in_head || h >= t.heads) return;
#pragma unroll
    for (int q = 0; q < PIECES; ++q) copy_shared<MOVE<T, E>>(place(i, j, q), base + h * t.x.sh + element_of<T, E>(q, l.second));
  };
  auto take = [&](int i, int j, Pairs& v) {
    Raw<T, E> r;
#pragma unroll
    for (int q = 0; q < PIECES; ++q) read_shared<MOVE<T, E>>(place(i, j, q), r.w + q * (MOVE<T, E> / 4));
    values<HALF>(r, v);
  };
  auto base_of = [&](const TurnTensor& t, const Token& k) { return static_cast<const T*>(t.x.data) + address(t.x, k) + l.e0; };
  griddep_wait();
  if (p.table != nullptr && live) ask_factors(p, where_of(p, k), room, lane);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (i < p.n_t) {
      const TurnTensor& t = p.t[i];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (!l.in_head || h0 + j * l.heads_a_vector >= t.heads)              // heads that are not there are 0
#pragma unroll
          for (int q = 0; q < PIECES; ++q) clear_shared<MOVE<T, E>>(place(i, j, q));
        if (live) ask(t, i, j, base_of(t, k));
      }
    }
  if constexpr (ROW)
    if (p.kept > 0) {
      keep_weights(p, p.t[0], kept);
      if (p.n_t == 2) keep_weights(p, p.t[1], kept + p.kept);
      __syncthreads();
    }
  for (long long first = (long long)blockIdx.x * per; first < p.rows; first += (long long)gridDim.x * per) {        // a turn is one for the whole CTA
  row += (long long)gridDim.x * per;
  const bool more = slot < per && row < p.rows;
  const Token next = token_of(p, more ? (unsigned)row : 0u);
  Factors cs;
  wait_copies();
  if (p.table != nullptr) {
    __syncwarp();
    if (l.turned) cs = factors_of<HALF, E>(p, room, l.slot);
    __syncwarp();
    if (more) ask_factors(p, where_of(p, next), room, lane);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (i >= p.n_t) break;
    const TurnTensor& t = p.t[i];
    const T* ahead = base_of(t, next);
    T* out = static_cast<T*>(t.o.data) + address(t.o, k) + l.e0;
    Pairs w;
    if constexpr (NORM == AS_NORM_HEAD)
      if (t.w != nullptr && l.in_head) load_weights<HALF, false>(p, t.w, 0u, l.e0, l.second, w);
    const uint32_t kept_at = sm100::smem_u32(kept) + (i == 0 ? 0u : (uint32_t)p.kept);
    float factor = 1.f, sum[1];                          // (the sum, and then the scale)
    auto settle = [&](bool there, auto squares) {
      auto sum_up = [&] {
        const float2 s = squares();
        sum[0] = s.x + s.y;
        sums_of<NORM>(p, sum, part, slot, warp, lane);
      };
      sum_up();
      factor = factor_for(sum[0], p.over_n[i], p.eps, there);
      if (any_of<NORM>(p, factor != 1.f)) sum_up();
      sum[0] = rsqrtf(fmaf(sum[0], p.over_n[i], p.eps * factor * factor));
    };
    Pairs v;
    if constexpr (ROW) {
      settle(live, [&] {
        float2 s = both(0.f);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          take(i, j, v);
          if (factor != 1.f) scale(v, both(factor));
          s = dot(v, v, s);
        }
        return s;
      });
    }
#pragma unroll
    for (int jj = 0; jj < NV; ++jj) {
      const int j = ROW ? NV - 1 - jj : jj, h = h0 + j * l.heads_a_vector;             // (over rows: the last one is still at hand, times its factor)
      const bool there = live && l.in_head && h < t.heads;
      if (!ROW || jj > 0) take(i, j, v);
      if (more) ask(t, i, j, ahead);
      if constexpr (NORM == AS_NORM_HEAD) {
        factor = 1.f;
        settle(there, [&] {
          if (factor != 1.f) scale(v, both(factor));
          return dot(v, v, both(0.f));
        });
      }
      if (!there) continue;
      if constexpr (NORM != AS_NORM_NONE) {
        if (ROW && jj > 0 && factor != 1.f) scale(v, both(factor));
        scale(v, both(sum[0]));
        if (t.w != nullptr) {
          if constexpr (ROW) {
            if (p.kept > 0) load_weights<HALF, true>(p, t.w, kept_at, h * p.d + l.e0, l.second, w);
            else load_weights<HALF, false>(p, t.w, 0u, h * p.d + l.e0, l.second, w);
          }
          scale(v, w);
        }
      }
      if (l.turned) turn(v, cs);
      store<HALF>(out + h * t.o.sh, l.second, v);
    }
  }
  live = more;
  k = next;
  }
}

// ---------------------------------------------------------------- backward
// dx = r (g - n mean(g n)), g = d w, d = R^T dy, n = x r.  A CTA goes on from row to row of one tensor.  Each warp has its sums of d n in shared
// memory (in registers, up to 48 of them, they left room for one CTA an SM), and the rows that it works on come there by asynchronous copies.  Both sums of a row, over x^2 and over g x, are taken at once.
template <typename T, int NORM, int NV, bool HALF, int E>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 2 ? 2 : 1) turn_back_kernel(const __grid_constant__ TurnParams p) {
  typedef PairsOf<E> Pairs;
  typedef FactorsOf<E> Factors;
  griddep_launch();
  __shared__ float part[2][WARPS];
  extern __shared__ float4 sums[];                       // of d n, of each warp: [vectors][4][32 lanes]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const TurnTensor& t = p.t[blockIdx.y];
  constexpr bool ROW = NORM == AS_NORM_ROW;
  const int per = ROW ? WARPS / p.W : WARPS;
  const int slot = ROW ? warp / p.W : warp, fixed_piece = ROW ? warp - slot * p.W : 0;
  const Lane l = lane_of<E>(p, lane);
  const bool sums_wanted = t.part != nullptr;
  constexpr int NA = ROW ? NV : 1;                       // vectors of sums: heads share them, or each has its own
  constexpr int G = E / 4;                                // groups of two pairs, four sums each
  float4* mine = sums + warp * (NA * G * 32) + lane;
  if (sums_wanted) {
#pragma unroll
    for (int i = 0; i < NA * G; ++i) mine[i * 32] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const int chunk = ROW ? 0 : (int)(blockIdx.x % (unsigned)p.chunks);
  const unsigned first_cta = ROW ? blockIdx.x : blockIdx.x / (unsigned)p.chunks, ctas = ROW ? gridDim.x : gridDim.x / (unsigned)p.chunks;      // (gridDim.x is a multiple of chunks)
  const int h0 = (ROW ? fixed_piece : chunk) * NV * l.heads_a_vector + l.head;
  const float over_n = p.over_n[blockIdx.y];
  griddep_wait();
  Pairs w;
#pragma unroll
  for (int i = 0; i < G; ++i) w.a[i] = w.b[i] = both(1.f);
  if (!ROW && t.w != nullptr && l.in_head) load_weights<HALF, false>(p, t.w, 0u, l.e0, l.second, w);
  // x and dy of a row, in this lane's own pieces of 16 bytes: the next row's are asked for as soon as this one's have been read for the last time
  constexpr int PIECES = MOVES<T, E>, STEP = 32 * MOVE<T, E>;            // moves of a vector, bytes of one by a warp
  float4* behind = sums + WARPS * (NA * G * 32);
  const uint32_t room = sm100::smem_u32(behind) + (uint32_t)(warp * (NV * 2 * PIECES * STEP) + lane * MOVE<T, E>);
  behind += WARPS * (NV * 2 * PIECES * STEP / 16);
  const uint32_t factors = sm100::smem_u32(behind) + (uint32_t)(warp * p.room), kept = sm100::smem_u32(behind) + (uint32_t)(WARPS * p.room);
  if constexpr (ROW)
    if (p.kept > 0) {
      keep_weights(p, t, reinterpret_cast<uint8_t*>(behind) + WARPS * p.room);
      __syncthreads();
    }
  auto place = [&](int j, int tensor, int piece) { return room + (uint32_t)(((j * 2 + tensor) * PIECES + piece) * STEP); };
  auto ask = [&](const T* bx, const T* by, bool live, int j) {
    const int h = h0 + j * l.heads_a_vector;
    if (!(live && l.in_head && h < t.heads)) return;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = element_of<T, E>(i, l.second);
      copy_shared<MOVE<T, E>>(place(j, 0, i), bx + h * t.x.sh + e);
      copy_shared<MOVE<T, E>>(place(j, 1, i), by + h * t.dy.sh + e);
    }
  };
  auto take_raw = [&](int j, int tensor, Raw<T, E>& r) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) read_shared<MOVE<T, E>>(place(j, tensor, i), r.w + i * (MOVE<T, E> / 4));
  };
  auto x_of = [&](const Token& k) { return static_cast<const T*>(t.x.data) + address(t.x, k) + l.e0; };
  auto y_of = [&](const Token& k) { return static_cast<const T*>(t.dy.data) + address(t.dy, k) + l.e0; };
  long long row = (long long)first_cta * per + slot;
  bool live = slot < per && row < p.rows;
  Token tk = token_of(p, live ? (unsigned)row : 0u);
  if (p.table != nullptr && live) ask_factors(p, where_of(p, tk), factors, lane);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (!l.in_head || h0 + j * l.heads_a_vector >= t.heads)                  // heads that are not there are 0
#pragma unroll
      for (int i = 0; i < 2 * PIECES; ++i) clear_shared<MOVE<T, E>>(place(j, 0, i));
    ask(x_of(tk), y_of(tk), live, j);
  }
  for (long long u0 = (long long)first_cta * per; u0 < p.rows; u0 += (long long)ctas * per) {       // a turn is one for the whole CTA
    row += (long long)ctas * per;
    const bool more = slot < per && row < p.rows;
    const Token next = token_of(p, more ? (unsigned)row : 0u);
    T* out = static_cast<T*>(t.o.data) + address(t.o, tk) + l.e0;
    wait_copies();
    Factors cs;
    if (p.table != nullptr) {
      __syncwarp();
      if (l.turned) cs = factors_of<HALF, E>(p, factors, l.slot);
      __syncwarp();
      if (more) ask_factors(p, where_of(p, next), factors, lane);
    }
    // x and d of vector j, and its weights
    auto operands = [&](int j, Pairs& v, Pairs& d) {
      Raw<T, E> r;
      take_raw(j, 0, r);
      values<HALF>(r, v);
      take_raw(j, 1, r);
      values<HALF>(r, d);
      if (l.turned) turn(d, cs);
      if constexpr (ROW) {
        const int h = h0 + j * l.heads_a_vector;
        if (t.w != nullptr && live && l.in_head && h < t.heads) {
          if (p.kept > 0) load_weights<HALF, true>(p, t.w, kept, h * p.d + l.e0, l.second, w);
          else load_weights<HALF, false>(p, t.w, 0u, h * p.d + l.e0, l.second, w);
        }
      }
    };
    float factor = 1.f, sum[2];                          // of (f x)^2 and of g f x; then the scale, and the mean of g n
    auto settle = [&](bool there, auto sums_now) {
      auto take = [&] {
        float2 s[2] = {both(0.f), both(0.f)};
        sums_now(s);
        sum[0] = s[0].x + s[0].y;
        sum[1] = s[1].x + s[1].y;
        sums_of<NORM>(p, sum, part, slot, warp, lane);
      };
      take();
      factor = factor_for(sum[0], over_n, p.eps, there);
      if (any_of<NORM>(p, factor != 1.f)) take();
      sum[0] = rsqrtf(fmaf(sum[0], over_n, p.eps * factor * factor));
      sum[1] = sum[1] * sum[0] * over_n;
    };
    auto add = [&](const Pairs& v, Pairs d, float2 (&s)[2]) {
      s[0] = dot(v, v, s[0]);
      scale(d, w);
      s[1] = dot(d, v, s[1]);
    };
    Pairs v, d;
    if constexpr (ROW)
      settle(live, [&](float2 (&s)[2]) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          operands(j, v, d);
          if (factor != 1.f) scale(v, both(factor));
          add(v, d, s);
        }
      });
#pragma unroll
    for (int jj = 0; jj < NV; ++jj) {
      const int j = ROW ? NV - 1 - jj : jj, h = h0 + j * l.heads_a_vector;             // (over rows: the last one is still at hand, times its factor)
      const bool there = live && l.in_head && h < t.heads;
      if (!ROW || jj > 0) operands(j, v, d);
      if (more) ask(x_of(next), y_of(next), true, j);
      if constexpr (!ROW) {
        factor = 1.f;
        settle(there, [&](float2 (&s)[2]) {
          if (factor != 1.f) scale(v, both(factor));
          add(v, d, s);
        });
      }
      if (!there) continue;
      if (ROW && jj > 0 && factor != 1.f) scale(v, both(factor));
      scale(v, both(sum[0]));
      if (sums_wanted) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
          const float4 q = mine[((ROW ? j : 0) * G + i) * 32];
          const float2 qa = fma2(d.a[i], v.a[i], make_float2(q.x, q.y)), qb = fma2(d.b[i], v.b[i], make_float2(q.z, q.w));
          mine[((ROW ? j : 0) * G + i) * 32] = make_float4(qa.x, qa.y, qb.x, qb.y);
        }
      }
      scale(d, w);
      const float2 along = both(-sum[1]), r2 = both(sum[0]);
#pragma unroll
      for (int i = 0; i < G; ++i) { d.a[i] = mul2(fma2(v.a[i], along, d.a[i]), r2); d.b[i] = mul2(fma2(v.b[i], along, d.b[i]), r2); }
      if (factor != 1.f) scale(d, both(factor));
      store<HALF>(out + h * t.o.sh, l.second, d);
    }
    live = more;
    tk = next;
  }
  if (!sums_wanted) return;
  // the warps' sums in their order: the CTA's row of partial sums.  A group is the first elements of pairs 2 i and 2 i + 1, and then their second ones
  auto element = [&](int i, int e) {                     // word e of group i
    const int pair = 2 * i + (e & 1), second = e >> 1;
    return HALF ? (second ? l.second + pair : pair) : (2 * pair + second < E / 2 ? 2 * pair + second : l.second + 2 * pair + second - E / 2);
  };
  if constexpr (ROW) {
    __syncthreads();
    if (slot == 0) {                                     // of the rows that the CTA had at once, those of slot 0 add the others' up
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int h = (fixed_piece * NV + j) * l.heads_a_vector + l.head;
        if (!l.in_head || h >= t.heads) continue;
        float* to = t.part + ((long long)blockIdx.x * t.heads + h) * p.d + l.e0;
#pragma unroll
        for (int i = 0; i < G; ++i) {
          float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int k = 0; k < per; ++k) {
            const float4 x = sums[(k * p.W + fixed_piece) * (NV * G * 32) + (j * G + i) * 32 + lane];
            q.x += x.x; q.y += x.y; q.z += x.z; q.w += x.w;
          }
          to[element(i, 0)] = q.x; to[element(i, 1)] = q.y; to[element(i, 2)] = q.z; to[element(i, 3)] = q.w;
        }
      }
    }
  } else {
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < G; ++i) {
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {
          const float4 x = sums[k * (G * 32) + i * 32 + lane];
          f.x += x.x; f.y += x.y; f.z += x.z; f.w += x.w;
        }
        float q[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          for (int o = 16; o >= 1 << p.lanes_log; o >>= 1) q[e] += __shfl_xor_sync(0xffffffffu, q[e], o);
          if (l.in_head && l.head == 0) t.part[(long long)blockIdx.x * p.d + l.e0 + element(i, e)] = q[e];
        }
      }
    }
  }
}

// The weights' gradient from the CTAs' rows of partial sums, in their order: 32 columns a CTA, 32 runs of rows side by side (8 runs: 10 us for 296 rows, all of it latency).
struct SumParams { const float* part[2]; void* out[2]; int cols[2]; int rows, f32; };
constexpr int SUM_RUNS = 32;
__global__ void __launch_bounds__(SUM_RUNS * 32) turn_sum_kernel(const __grid_constant__ SumParams p) {
  griddep_launch();
  __shared__ float some[SUM_RUNS][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.y, c = blockIdx.x * 32 + lane, cols = i == 0 ? p.cols[0] : p.cols[1];
  griddep_wait();
  const float* part = i == 0 ? p.part[0] : p.part[1];
  void* out = i == 0 ? p.out[0] : p.out[1];
  if (part == nullptr || blockIdx.x * 32 >= cols) return;
  const int r0 = p.rows * warp / SUM_RUNS, r1 = p.rows * (warp + 1) / SUM_RUNS;
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
    for (int j = 0; j < SUM_RUNS; ++j) s += some[j][lane];
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
  extern __shared__ float room[];                        // backward: of the weights' gradient, a row of them for each warp or for the CTA
  constexpr bool ROW = NORM == AS_NORM_ROW;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int which = BACK ? blockIdx.y : 0, np = p.d - p.pairs;           // pieces of a head
  const int cols = ROW ? (which == 0 ? p.t[0] : p.t[1]).heads * p.d : p.d;
  float* mine = room + (ROW ? 0 : warp * p.d);
  if constexpr (BACK) {
    for (int c = threadIdx.x; c < (ROW ? cols : WARPS * p.d); c += THREADS) room[c] = 0.f;
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
    const Token k = token_of(p, r);
    const T* x = static_cast<const T*>(t.x.data) + address(t.x, k);
    const T* y = BACK ? static_cast<const T*>(t.dy.data) + address(t.dy, k) : nullptr;
    T* out = static_cast<T*>(t.o.data) + address(t.o, k);
    const Where at = p.table != nullptr ? where_of(p, k) : Where{};
    auto sum = [&](float s, float* of) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if constexpr (ROW) {
        __syncthreads();
        if (lane == 0) of[warp] = s;
        __syncthreads();
        s = 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) s += of[i];
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
    auto sums_of_both = [&](float f) {
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
    struct { float factor, scale; } s{1.f, 1.f};
    float along = 0.f;
    if constexpr (NORM != AS_NORM_NONE) {
      const float n = ROW ? (float)t.heads * (float)p.d : (float)p.d;
      float2 q = sums_of_both(1.f);
      const float mean = q.x / n + p.eps;
      s.scale = rsqrtf(mean);
      if (over(q.x) || mean < LEAST) {                   // (one value for all that share the sum)
        const float f = over(q.x) ? DOWN : UP;
        q = sums_of_both(f);
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
      float s = room[c];
      if constexpr (!ROW)
        for (int w = 1; w < WARPS; ++w) s += room[w * p.d + c];
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
  if (!back && a->rows > 0) {                // results over their own inputs only
    if (!in_place_ok(a->q_out, a->q, a->rows, (long long)a->q_heads * a->head_dim) || (two && !in_place_ok(a->k_out, a->k, a->rows, (long long)a->k_heads * a->head_dim))) return AS_ERR_INVALID_ARG;
    if (two && (a->q_out.data == a->k.data || a->k_out.data == a->q.data || a->q_out.data == a->k_out.data)) return AS_ERR_INVALID_ARG;
  }
  int pairs;
  if (const as_status_t s = rotation_ok(a->rotation, a->rows > 0 ? a->q.tokens : 0, a->head_dim, &pairs); s != AS_OK) return s;
  if (a->norm == AS_NORM_ROW && (long long)std::max(a->q_heads, two ? a->k_heads : 0) * a->head_dim > 16384) return AS_ERR_UNSUPPORTED;
  return AS_OK;
}

// Whether pieces of 4 or 8 elements move at once.
bool heads_vec(const as_rows_t& x, int elements) {
  const int bytes = elements * (x.dtype == AS_DTYPE_BF16 ? 2 : 4) < 16 ? 8 : 16;
  return aligned(x.data, bytes) && ((x.stride_batch | x.stride_head | x.stride_token) & (bytes / (x.dtype == AS_DTYPE_BF16 ? 2 : 4) - 1)) == 0;
}

constexpr size_t KEPT_MOST = 12 * 1024;      // of rows' weights
// Shared memory of a kernel's calls: more than 48 KB has to be asked for.  It is, once for a kernel and a device, for the most that any call of it takes: a limit that each call set to its own size
// would be lowered by one thread between another one's setting and its launch.
template <auto KERNEL>
cudaError_t allow_smem(size_t smem, size_t most) {
  if (smem <= 40 * 1024) return cudaSuccess;
  static std::atomic<uint64_t> done{0};                  // a bit for each device
  int dev = 0;
  if (const cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0ull;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}
// A warp's factors at the most: of heads of 32 lanes, all of them turned.
constexpr size_t room_most(int E) { return (size_t)(16 * E / 2 + 7) / 8 * 128; }

struct Shape { bool vec; int E, NV, chunks; long long ctas; size_t kept; };       // kept: bytes of both tensors' weights
// Fills in what the kernels share; `most`: vectors that a lane's registers hold.
Shape turn_params(const as_qk_norm_rotary_t& a, const as_rotation_t& r, int sms, bool back, const as_rows_t* more, int n_more, TurnParams& p) {
  const bool two = a.k.data != nullptr;
  int pairs;
  rotation_ok(r, 0, a.head_dim, &pairs);
  p.n_t = two ? 2 : 1;
  p.rows = (int)a.rows; p.tokens = (int)a.q.tokens; p.d = a.head_dim;
  auto by = [](unsigned n) { return n == 1u ? 0ull : ~0ull / n + 1ull; };
  p.by_tokens = by((unsigned)std::max(p.tokens, 1));
  for (int i = 0; i < 2; ++i) p.over_n[i] = 1.f / ((float)a.head_dim * (a.norm == AS_NORM_ROW ? (float)std::max(i == 0 ? a.q_heads : a.k_heads, 1) : 1.f));
  p.eps = a.eps;
  p.w_f32 = a.weight_dtype == AS_DTYPE_F32;
  p.t[0].heads = a.q_heads;
  p.t[1].heads = two ? a.k_heads : 0;
  p.t[0].x = rows_of(a.q, a.rows, (long long)a.q_heads * a.head_dim);
  if (two) p.t[1].x = rows_of(a.k, a.rows, (long long)a.k_heads * a.head_dim);
  if (a.norm != AS_NORM_NONE) { p.t[0].w = a.q_weight; p.t[1].w = two ? a.k_weight : nullptr; }
  p.table = reinterpret_cast<const float2*>(r.table);
  p.pairs = pairs;                           // (0 without a table)
  p.room = (pairs / 2 + 7) / 8 * 128;
  if (p.table != nullptr) {
    p.axes = r.n_axes;
    p.half = r.layout == AS_ROTARY_HALF;
    p.sign = (r.inverse != 0) != back ? -1.f : 1.f;
    p.pos = r.positions; p.pos64 = r.position_bytes == 8; p.pos_stride = r.positions_stride; p.first = r.first;
    int rows = 0, end = 0;
    for (int i = 0; i < AS_ROTARY_MAX_AXES; ++i) {
      p.first_row[i] = rows;
      if (i < r.n_axes) { p.size[i] = r.size[i]; p.by_size[i] = by((unsigned)r.size[i]); rows += r.size[i]; end += r.pairs[i]; }
      p.end[i] = end;
    }
  }
  Shape s{};
  // 16 elements a lane, or 8, where sizes, pairs, strides and addresses allow it
  auto fits = [&](int E) {
    const int piece = E / 2, of_weights = piece * (p.w_f32 ? 4 : 2) < 16 ? 8 : 16;
    if (a.head_dim % E != 0 || a.head_dim > 32 * E || pairs % piece != 0 || !aligned(r.table, 16) || !heads_vec(a.q, piece) || (two && !heads_vec(a.k, piece))) return false;
    for (int i = 0; i < n_more; ++i)
      if (more[i].data != nullptr && !heads_vec(more[i], piece)) return false;
    return a.norm == AS_NORM_NONE || (aligned(a.q_weight, of_weights) && (!two || aligned(a.k_weight, of_weights)));
  };
  s.E = fits(16) ? 16 : 8;
  s.vec = s.E == 16 || fits(8);
  p.lanes_log = 0;
  while ((s.E << p.lanes_log) < a.head_dim) ++p.lanes_log;
  const int heads = std::max(p.t[0].heads, p.t[1].heads), of_vector = std::max(1, 32 >> p.lanes_log), vectors = (heads + of_vector - 1) / of_vector;
  const int most = a.q.dtype == AS_DTYPE_BF16 ? 3 : 2;
  p.W = 1; p.chunks = 1;
  if (a.norm == AS_NORM_ROW) {
    p.W = (vectors + most - 1) / most;
    if (p.W > WARPS) s.vec = false;
    else s.NV = (vectors + p.W - 1) / p.W;
    s.ctas = s.vec ? (a.rows + WARPS / p.W - 1) / (WARPS / p.W) : a.rows * (back ? 1 : p.n_t);
    // weights in shared memory, up to what has been measured: two vectors of 1536 in fp32 (two CTAs an SM would have the room for more)
    const size_t size = p.w_f32 ? 4 : 2, of_q = (size_t)p.t[0].heads * a.head_dim * size, of_k = (size_t)p.t[1].heads * a.head_dim * size;
    s.kept = back ? std::max(of_q, of_k) : of_q + of_k;
    if (s.vec && s.kept <= KEPT_MOST && of_q % 16 == 0 && of_k % 16 == 0 && aligned(a.q_weight, 16) && (!two || aligned(a.k_weight, 16))) p.kept = (int)of_q;
    else s.kept = 0;
  } else {
    // few rows: a vector a warp, so that all of them are under way at once
    s.NV = a.rows * ((vectors + most - 1) / most) <= 4ll * sms ? 1 : std::min(vectors, most);
    p.chunks = (vectors + s.NV - 1) / s.NV;
    if (p.chunks > 65535) s.vec = false;
    s.ctas = s.vec ? (a.rows + WARPS - 1) / WARPS : (a.rows * (back ? heads : (long long)p.t[0].heads + p.t[1].heads) + WARPS - 1) / WARPS;
  }
  return s;
}

template <typename T, int NORM, int E>
cudaError_t launch_lanes(const TurnParams& p, const Shape& s, int sms, cudaStream_t st) {
  const dim3 grid((unsigned)std::min<long long>(s.ctas, std::max(1, 2 * sms / p.chunks)), (unsigned)p.chunks), block(THREADS);        // CTAs go on from row to row
  const size_t smem = WARPS * (s.NV * (E * 64) * sizeof(T) + (size_t)p.room) + s.kept;
  auto launch = [&](auto nv, auto half) {
    constexpr int NV = decltype(nv)::value;
    constexpr auto kernel = turn_kernel<T, NORM, NV, decltype(half)::value, E>;
    if (const cudaError_t e = allow_smem<kernel>(smem, WARPS * (NV * (E * 64) * sizeof(T) + room_most(E)) + KEPT_MOST); e != cudaSuccess) return e;
    return as_launch_dependent(kernel, grid, block, smem, st, p);
  };
  auto run = [&](auto nv) { return p.half ? launch(nv, std::true_type{}) : launch(nv, std::false_type{}); };
  switch (s.NV) {
    case 1: return run(std::integral_constant<int, 1>{});
    case 2: return run(std::integral_constant<int, 2>{});
    default: return run(std::integral_constant<int, 3>{});
  }
}
template <typename T, int NORM>
cudaError_t launch_turn(const TurnParams& p, const Shape& s, int sms, cudaStream_t st) {
  if (!s.vec) return as_launch_dependent(turn_elements_kernel<T, NORM, false>, dim3((unsigned)std::min<long long>(s.ctas, 8ll * sms)), dim3(THREADS), 0, st, p);
  return s.E == 16 ? launch_lanes<T, NORM, 16>(p, s, sms, st) : launch_lanes<T, NORM, 8>(p, s, sms, st);
}
template <typename T>
cudaError_t launch_norm(const TurnParams& p, const Shape& s, int norm, int sms, cudaStream_t st) {
  return norm == AS_NORM_NONE ? launch_turn<T, AS_NORM_NONE>(p, s, sms, st) : norm == AS_NORM_HEAD ? launch_turn<T, AS_NORM_HEAD>(p, s, sms, st) : launch_turn<T, AS_NORM_ROW>(p, s, sms, st);
}

template <typename T, int NORM, int E>
cudaError_t launch_back_lanes(const TurnParams& p, const Shape& s, unsigned ctas, cudaStream_t st) {
  const size_t smem = WARPS * ((NORM == AS_NORM_ROW ? s.NV : 1) * (E * 128) + s.NV * (E * 64) * sizeof(T) + (size_t)p.room) + s.kept;
  auto launch = [&](auto nv, auto half) {
    constexpr int NV = decltype(nv)::value;
    constexpr auto kernel = turn_back_kernel<T, NORM, NV, decltype(half)::value, E>;
    if (const cudaError_t e = allow_smem<kernel>(smem, WARPS * ((NORM == AS_NORM_ROW ? NV : 1) * (E * 128) + NV * (E * 64) * sizeof(T) + room_most(E)) + KEPT_MOST); e != cudaSuccess) return e;
    return as_launch_dependent(kernel, dim3(ctas, (unsigned)p.n_t), dim3(THREADS), smem, st, p);
  };
  auto run = [&](auto nv) { return p.half ? launch(nv, std::true_type{}) : launch(nv, std::false_type{}); };
  if constexpr (sizeof(T) == 2)
    if (s.NV == 3) return run(std::integral_constant<int, 3>{});
  return s.NV == 2 ? run(std::integral_constant<int, 2>{}) : run(std::integral_constant<int, 1>{});
}
template <typename T, int NORM>
cudaError_t launch_back(const TurnParams& p, const Shape& s, unsigned ctas, cudaStream_t st) {
  if (s.vec) return s.E == 16 ? launch_back_lanes<T, NORM, 16>(p, s, ctas, st) : launch_back_lanes<T, NORM, 8>(p, s, ctas, st);
  const size_t smem = (size_t)(NORM == AS_NORM_ROW ? std::max(p.t[0].heads, p.t[1].heads) : WARPS) * p.d * 4;
  constexpr auto kernel = turn_elements_kernel<T, NORM, true>;
  if (const cudaError_t e = allow_smem<kernel>(smem, 16384 * 4); e != cudaSuccess) return e;             // (over rows: of 16384 columns; by heads: 8 x 1024)
  return as_launch_dependent(kernel, dim3(ctas, (unsigned)p.n_t), dim3(THREADS), smem, st, p);
}

// CTAs of the backward pass, for each tensor: as many as the device holds at once (of vectors: a multiple of the chunks, which they take in turn).
unsigned back_ctas(const TurnParams& p, const Shape& s, bool f32, int sms) {
  const int most = std::max(1, (s.vec ? f32 ? 1 : 2 : 4) * sms / p.n_t);
  if (!s.vec) return (unsigned)std::min<long long>(s.ctas, most);
  return (unsigned)(std::min<long long>(s.ctas, std::max(1, most / p.chunks)) * p.chunks);
}

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
  if (a.rows > 0) {
    const long long cols[2] = {(long long)a.q_heads * a.head_dim, (long long)a.k_heads * a.head_dim};
    if (!in_place_ok(b->dq_out, b->dq, a.rows, cols[0]) || !in_place_ok(b->dq_out, a.q, a.rows, cols[0])) return AS_ERR_INVALID_ARG;
    if (two && (!in_place_ok(b->dk_out, b->dk, a.rows, cols[1]) || !in_place_ok(b->dk_out, a.k, a.rows, cols[1]))) return AS_ERR_INVALID_ARG;
    const void *q_out = b->dq_out.data, *k_out = b->dk_out.data;
    if (two && (q_out == k_out || q_out == b->dk.data || q_out == a.k.data || k_out == b->dq.data || k_out == a.q.data)) return AS_ERR_INVALID_ARG;
  }
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
    p.axis[i] = TableAxis{x.base, x.factor, x.original, x.scaling, x.pairs, (int)rows, (int)pairs};
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
  *bytes = back_bytes(*b, back_ctas(p, s, b->fwd->q.dtype == AS_DTYPE_F32, sms), cols);
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
  const unsigned ctas = back_ctas(p, s, a.q.dtype == AS_DTYPE_F32, sms);
  const uint64_t need = back_bytes(*b, ctas, cols);
  if (need > 0 && (b->workspace == nullptr || !aligned(b->workspace, 16) || b->workspace_bytes < need)) return AS_ERR_WORKSPACE;
  float* part = static_cast<float*>(b->workspace);
  const as_rows_t* dy[2] = {&b->dq, &b->dk};
  const as_rows_t* out[2] = {&b->dq_out, &b->dk_out};
  void* dw[2] = {b->dq_weight, b->dk_weight};
  SumParams sum{};
  for (int i = 0; i < p.n_t; ++i) {
    const long long wide = (long long)p.t[i].heads * a.head_dim;
    p.t[i].dy = rows_of(*dy[i], a.rows, wide);
    p.t[i].o = rows_of(*out[i], a.rows, wide);
    if (cols[i] > 0) { p.t[i].part = part; sum.part[i] = part; sum.out[i] = dw[i]; sum.cols[i] = (int)cols[i]; part += ctas * cols[i]; }
  }
  cudaError_t e;
  if (a.q.dtype == AS_DTYPE_BF16) e = a.norm == AS_NORM_HEAD ? launch_back<bf, AS_NORM_HEAD>(p, s, ctas, st) : launch_back<bf, AS_NORM_ROW>(p, s, ctas, st);
  else e = a.norm == AS_NORM_HEAD ? launch_back<float, AS_NORM_HEAD>(p, s, ctas, st) : launch_back<float, AS_NORM_ROW>(p, s, ctas, st);
  if (e == cudaSuccess && cols[0] + cols[1] > 0) {
    sum.rows = (int)ctas;
    sum.f32 = a.weight_dtype == AS_DTYPE_F32;
    e = as_launch_dependent(turn_sum_kernel, dim3((unsigned)((std::max(cols[0], cols[1]) + 31) / 32), 2), dim3(SUM_RUNS * 32), 0, st, sum);
  }
  return e == cudaSuccess ? AS_OK : failed();
}
