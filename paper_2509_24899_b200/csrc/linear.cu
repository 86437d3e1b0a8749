// Linear layers in bf16: out = residual + gate * act(x w^T + bias), and the gradients dx = dz w, dw = dz^T x, on the tensor cores.
//
// One kernel does the three products; they differ in which of an operand's two indices lies in a run in memory, which the copies (boxes of 64 elements by rows) and the operand
// descriptors say.  A pair of CTAs (cta_group::2) computes a tile of 256 rows by up to 256 columns: each holds 128 rows of the first operand, half of the tile's columns of the second
// and 128 rows of results.  The grid is persistent, one CTA an SM; a tile's results are read out while the next one is computed, from the other of two accumulators.
// The kernel alone: 32760 x 1536 by 6144 x 1536 with a bias and gelu_tanh 427 us, 1.45 PFLOP/s, the tensor pipe active 92 % of the time at the 1.44 GHz that the power limit leaves; 32760 x 6144 by
// 1536 x 6144 onto a residual in fp32 477 us, 1.30 PFLOP/s (with nothing behind the products 412 and 439; the library's bf16 products of these sizes 420 and 462); the gradients' products of 7800 x 1536 by
// 6144 x 1536 113 us (dx) and 97 us (dw).  In calls one after another, of which the power limit leaves a lower clock, 497, 573 and, the whole gradient, 320.
//
//   warp 0       copies (TMA, 64 steps of the summed index a stage, 128-byte swizzle), told by the leading CTA's barrier
//   warp 1       the MMAs (leading CTA only)
//   warp 2       allocates tensor memory
//   warps 3-18   results, 32 rows x 32 columns at a time: tensor memory -> registers, a lane a row: bias, activation, gate, bf16, a strip of shared memory, from where TMA takes
//                them; with a residual, in fp32 or in layouts without boxes 16 columns at a time through the strip, from where 4 lanes move a row
//
// What bounds it is the tensor pipe and the operands' bytes into an SM, which for 256 x 256 are level: 64 bytes a clock beside 8192 operations.
//
// Where the tiles are too few for the SMs, a cluster of CTAs shares the summed index of a tile (SHARED), or it is cut into parts whose sums go to the workspace in fp32 and finish_kernel adds them
// up in order.  Few rows of x: linear_few_kernel, further down.
#include <algorithm>
#include <type_traits>

#include "as_layer.h"
#include "fp8_common.cuh"
#include "fp8_context.h"
#include "fp8_maps.h"
#include "linear_plan.h"
#include "sm100_pairs.cuh"
#include "tensor_common.cuh"

namespace {

using namespace as_fp8;
using namespace sm100;
typedef __nv_bfloat16 bf;

constexpr int RESULT_WARPS = 16, FIRST_RESULT = 3, LIN_THREADS = (FIRST_RESULT + RESULT_WARPS) * 32;
constexpr int BM = LIN_BM, BK = LIN_BK;
constexpr int MAX_STAGES = 10;
constexpr int SMEM_MAX = 227 * 1024;
constexpr uint32_t BOX = 64 * 128;          // bytes of a box of 64 x 64

enum { B_FULL = 0, B_EMPTY = B_FULL + MAX_STAGES, B_AFULL = B_EMPTY + MAX_STAGES, B_AEMPTY = B_AFULL + 2, B_RES = B_AEMPTY + 2, B_COUNT = B_RES + 2 * RESULT_WARPS };
// shared memory: barriers, tensor-memory address, abort flag; for each result warp two strips of 32 rows x 64 bytes, which results leave from and residuals come to; then the stages
constexpr int STRIP = 32 * 64;
constexpr int STRIPS_OFF = 1024;
constexpr int STAGES_OFF = STRIPS_OFF + RESULT_WARPS * 2 * STRIP;
// Byte of 16-byte chunk `ch` of a strip's row: the 64-byte swizzle.
AS_DEV uint32_t swz64(int row, int ch) { return (uint32_t)(row * 64 + ((ch ^ (row >> 1 & 3)) << 4)); }
static_assert(B_COUNT * 8 + 8 <= STRIPS_OFF && STAGES_OFF % 1024 == 0, "");

// ---------------------------------------------------------------- what follows a sum
struct Epilogue {
  Rows out, res, pre;                        // data == nullptr: not there
  const void *bias, *gate;
  long long gate_stride;
  unsigned gate_rows;                        // rows that share a gate
  int N, act;
  bool out_f32, res_f32, bias_f32, gate_f32;
  bool vec;                                  // four columns move at once
  bool boxes, pre_boxes, res_boxes;          // out and pre leave, and the residual comes, in boxes of 32 rows x 64 bytes by TMA
};

AS_DEV float ld1(const void* p, bool f32, long long i) { return f32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const bf*>(p)[i]); }
AS_DEV float4 ld4(const void* p, bool f32, long long i) {
  if (f32) return *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
  const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const bf*>(p) + i);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
}
AS_DEV void st4(void* p, bool f32, long long i, float4 v) {
  if (f32) *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = v;
  else *reinterpret_cast<uint2*>(static_cast<bf*>(p) + i) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}
AS_DEV void st1(void* p, bool f32, long long i, float v) {
  if (f32) static_cast<float*>(p)[i] = v;
  else static_cast<bf*>(p)[i] = __float2bfloat16_rn(v);
}

// 1 / (1 + e^-x): e^-x is 2^(-x log2 e), infinite for what is far below 0, where the quotient is 0.
AS_DEV float sigmoid(float x) { return __fdividef(1.f, 1.f + ex2(-1.442695041f * x)); }
constexpr float GELU_A = 1.5957691216f, GELU_B = 0.044715f;      // 2 sqrt(2 / pi): gelu_tanh(z) = z sigmoid(A (z + B z^3)), as 1 + tanh(u) = 2 sigmoid(2 u)
// The normal distribution's function, with e = e^(-z^2 / 2): erfc(a) = e^(-a^2) f(a), a = |z| / sqrt 2, f a polynomial of t = 1 / (1 + 0.35 a), fitted to the least relative error over a up to 9.6 (7e-9;
// in fp32 4e-7 of 1, and 8e-6 of itself far below 0, where the rounding of z^2 counts).
AS_DEV float normal_cdf(float z, float& e) {
  const float t = __fdividef(1.f, fmaf(fabsf(z), 0.35f * 0.7071067812f, 1.f));
  e = ex2(-0.7213475204f * z * z);
  float f = 0.0377782903f;
  f = fmaf(f, t, -0.155430015f); f = fmaf(f, t, 0.172923096f); f = fmaf(f, t, -0.015841502f); f = fmaf(f, t, 0.076692656f); f = fmaf(f, t, 0.151870132f);
  f = fmaf(f, t, 0.1490568f); f = fmaf(f, t, 0.188387351f); f = fmaf(f, t, 0.197075969f); f = fmaf(f, t, 0.197487229f);
  const float half = 0.5f * f * t * e;
  return z < 0.f ? half : 1.f - half;
}
// z times what is 0 far below 0 (there z may be minus infinity).
AS_DEV float times(float z, float f) { return f == 0.f ? 0.f : z * f; }
template <int ACT>
AS_DEV float activated(float z) {
  if constexpr (ACT == AS_ACT_RELU) return z < 0.f ? 0.f : z;     // (NaN stays)
  else if constexpr (ACT == AS_ACT_SILU) return times(z, sigmoid(z));
  else if constexpr (ACT == AS_ACT_GELU) { float e; return times(z, normal_cdf(z, e)); }
  else if constexpr (ACT == AS_ACT_GELU_TANH) return times(z, sigmoid(GELU_A * z * fmaf(GELU_B * z, z, 1.f)));
  else return z;
}
// f with the activation as a constant.
template <typename F>
AS_DEV void with_activation(int act, F f) {
  switch (act) {
    case AS_ACT_RELU: f(std::integral_constant<int, AS_ACT_RELU>{}); break;
    case AS_ACT_SILU: f(std::integral_constant<int, AS_ACT_SILU>{}); break;
    case AS_ACT_GELU: f(std::integral_constant<int, AS_ACT_GELU>{}); break;
    case AS_ACT_GELU_TANH: f(std::integral_constant<int, AS_ACT_GELU_TANH>{}); break;
    default: break;
  }
}
AS_DEV float activated(float z, int act) {
  with_activation(act, [&](auto a) { z = activated<decltype(a)::value>(z); });
  return z;
}
// (act(z), act'(z)).  sigmoid(-x) is e^-x sigmoid(x); arguments below -80 count as that, where both are 0 to fp32 beside anything that they are added to.
template <int ACT>
AS_DEV float2 activated2(float z) {
  if constexpr (ACT == AS_ACT_RELU) {
    return make_float2(z < 0.f ? 0.f : z, z > 0.f ? 1.f : z != z ? z : 0.f);
  } else if constexpr (ACT == AS_ACT_SILU) {
    const float e = ex2(-1.442695041f * (z < -80.f ? -80.f : z)), s = __fdividef(1.f, 1.f + e), t = e * s;
    return make_float2(z < -80.f ? 0.f : z * s, z < -80.f ? 0.f : t == 0.f ? s : s * fmaf(z, t, 1.f));
  } else if constexpr (ACT == AS_ACT_GELU) {
    float e;
    const float c = normal_cdf(z, e);
    return make_float2(times(z, c), e == 0.f ? c : fmaf(z * 0.3989422804f, e, c));
  } else if constexpr (ACT == AS_ACT_GELU_TANH) {
    const float q = GELU_B * z * z, u = GELU_A * z * (1.f + q), e = ex2(-1.442695041f * (u < -80.f ? -80.f : u)), s = __fdividef(1.f, 1.f + e), t = e * s;
    return make_float2(u < -80.f ? 0.f : z * s, u < -80.f ? 0.f : t == 0.f ? s : fmaf(z * s, t * GELU_A * fmaf(3.f, q, 1.f), s));
  } else {
    return make_float2(z, 1.f);
  }
}

// Sums of columns n .. n + 3 of row m, on to out and pre.
struct Column4 { float4 bias; bool gates_alike; float4 gate; };
AS_DEV Column4 columns_of(const Epilogue& e, int n) {
  Column4 c{make_float4(0.f, 0.f, 0.f, 0.f), e.gate != nullptr && e.gate_rows == 0u, make_float4(1.f, 1.f, 1.f, 1.f)};
  float *b = &c.bias.x, *g = &c.gate.x;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < e.N) {
      if (e.bias != nullptr) b[i] = ld1(e.bias, e.bias_f32, n + i);
      if (c.gates_alike) g[i] = ld1(e.gate, e.gate_f32, n + i);
    }
  return c;
}
AS_DEV void finish4(const Epilogue& e, const Column4& c, int m, int n, float4 v) {
  v.x += c.bias.x; v.y += c.bias.y; v.z += c.bias.z; v.w += c.bias.w;
  float* f = &v.x;
  if (e.vec) {
    if (e.pre.data != nullptr) st4(e.pre.data, false, e.pre.row((unsigned)m) + e.pre.col((unsigned)n), v);
    if (e.act != AS_ACT_NONE) {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = activated(f[i], e.act);
    }
    if (e.gate != nullptr) {
      const float4 g = c.gates_alike ? c.gate : ld4(e.gate, e.gate_f32, (long long)((unsigned)m / e.gate_rows) * e.gate_stride + n);
      v.x *= g.x; v.y *= g.y; v.z *= g.z; v.w *= g.w;
    }
    if (e.res.data != nullptr) {
      const float4 r = ld4(e.res.data, e.res_f32, e.res.row((unsigned)m) + e.res.col((unsigned)n));
      v.x += r.x; v.y += r.y; v.z += r.z; v.w += r.w;
    }
    st4(e.out.data, e.out_f32, e.out.row((unsigned)m) + e.out.col((unsigned)n), v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (n + i >= e.N) continue;
      float x = f[i];
      if (e.pre.data != nullptr) st1(e.pre.data, false, e.pre.row((unsigned)m) + e.pre.col((unsigned)(n + i)), x);
      x = activated(x, e.act);
      if (e.gate != nullptr) x *= c.gates_alike ? (&c.gate.x)[i] : ld1(e.gate, e.gate_f32, (long long)((unsigned)m / e.gate_rows) * e.gate_stride + n + i);
      if (e.res.data != nullptr) x += ld1(e.res.data, e.res_f32, e.res.row((unsigned)m) + e.res.col((unsigned)(n + i)));
      st1(e.out.data, e.out_f32, e.out.row((unsigned)m) + e.out.col((unsigned)(n + i)), x);
    }
  }
}

// ---------------------------------------------------------------- the products
struct GemmParams {
  Epilogue e;
  float* part;                              // sums of parts [parts][M][pitch], or nullptr
  uint32_t* status;
  long long part_pitch, units;              // units: tiles x parts
  int M, T, mt_entry;                       // rows of results in entries of T, of mt_entry tiles each
  int bn, nt, stages, parts;
  int ksteps, ks_entry;                     // steps of BK of the summed index, where it is rows: of an entry
  int run;                                  // LONG: steps of a run of sums
  unsigned long long by_nt, by_mt;          // 2^64 / nt and 2^64 / mt_entry, rounded up (0: 1): a quotient is the upper half of a product, exact below 2^32
  int a_hd, b_hd;                           // columns of a head of the operands, multiples of 64 (INT32_MAX: there are no heads)
};

template <int CG>
AS_DEV void load_box4(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int t, int h, int b) {
  if constexpr (CG == 1)
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(t), "r"(h), "r"(b) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(t), "r"(h), "r"(b) : "memory");
}
template <int CG>
AS_DEV void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CG == 1) mma_ss(d, a, b, idesc, accumulate);
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// 8 columns of a lane's row, waited for; and back.
AS_DEV void tmem_ld8(uint32_t at, float (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]) : "r"(at) : "memory");
}
AS_DEV void tmem_st8(uint32_t at, const float (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(at), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]) : "memory");
}

template <int CG>
struct Ctx {
  uint32_t sbase, tmem;
  WaitCtx wc;
  uint32_t rank;                             // of the CTA in its pair
  long long unit, step;                      // this pair's units: unit, unit + step, ...
  AS_DEV uint32_t bar(int i) const { return sbase + 8 * i; }
  AS_DEV bool wait(int i, uint32_t parity) const { return mbar_wait(bar(i), parity, wc); }
};
// A unit of work: a tile and a part of the summed index.
struct Unit { int entry, t0, n0, k0, k1, part; };
// (With 64-bit divisions here, in every warp and for every unit, tiles of one step took a tenth longer.)
AS_DEV unsigned quotient(unsigned i, unsigned long long by) { return by == 0ull ? i : (unsigned)__umul64hi(by, i); }
template <int CG>
AS_DEV Unit unit_of(const GemmParams& p, long long u) {
  Unit w{};
  unsigned tile = (unsigned)u;
  w.k1 = p.ksteps;
  if (p.parts > 1) {
    tile = (unsigned)u / (unsigned)p.parts;
    w.part = (int)((unsigned)u - tile * (unsigned)p.parts);
    w.k0 = (int)((long long)p.ksteps * w.part / p.parts);
    w.k1 = (int)((long long)p.ksteps * (w.part + 1) / p.parts);
  }
  const unsigned mt = quotient(tile, p.by_nt);
  w.n0 = (int)(tile - mt * (unsigned)p.nt) * p.bn;
  w.entry = (int)quotient(mt, p.by_mt);
  w.t0 = (int)(mt - (unsigned)w.entry * (unsigned)p.mt_entry) * (BM * CG);
  return w;
}

// A_MN, B_MN: the operand's rows or columns of the result lie in a run in memory (else the summed index does).
template <int CG, bool A_MN, bool B_MN>
AS_DEV void lin_copies(const GemmParams& p, const Ctx<CG>& c, const CUtensorMap* ma, const CUtensorMap* mb) {
  const int rows_b = p.bn / CG;
  const uint32_t stage_bytes = (uint32_t)(BM + rows_b) * BK * 2;
  constexpr int A_BOXES = A_MN ? BM / 64 : 1, B_BOXES = B_MN ? 256 / CG / 64 : 1;
  Ring r;
  for (long long u = c.unit; u < p.units; u += c.step) {
    const Unit w = unit_of<CG>(p, u);
    const int m0 = w.t0 + (int)c.rank * BM, n0 = w.n0 + (int)c.rank * rows_b;
    // Where boxes begin.  What does not change from step to step is divided here: with the heads of every box looked for at every step this thread was what the products waited for (32760 x 6144 by
    // 1536, columns of w in a run: 571 us, 423 us where a step has two boxes).
    int ax[A_BOXES], ah[A_BOXES], bx[B_BOXES], bh[B_BOXES];
    if constexpr (A_MN) {
#pragma unroll
      for (int i = 0; i < A_BOXES; ++i) { ah[i] = p.a_hd == INT32_MAX ? 0 : (m0 + 64 * i) / p.a_hd; ax[i] = m0 + 64 * i - ah[i] * p.a_hd; }
    } else {
      ah[0] = w.k0 == 0 ? 0 : w.k0 * BK / p.a_hd;
      ax[0] = w.k0 * BK - ah[0] * p.a_hd;
    }
    if constexpr (B_MN) {
#pragma unroll
      for (int i = 0; i < B_BOXES; ++i) { bh[i] = p.b_hd == INT32_MAX ? 0 : (n0 + 64 * i) / p.b_hd; bx[i] = n0 + 64 * i - bh[i] * p.b_hd; }
    }
    int ke = A_MN && w.k0 != 0 ? w.k0 / p.ks_entry : 0, kt = A_MN ? w.k0 - ke * p.ks_entry : w.k0;      // entry and step of the summed index
    for (int k = w.k0; k < w.k1; ++k) {
      if (!c.wait(B_EMPTY + r.slot, r.turn ^ 1u)) goto out;
      const uint32_t at = c.sbase + STAGES_OFF + (uint32_t)r.slot * stage_bytes, bt = at + BM * BK * 2;
      if (c.rank == 0) mbar_expect_tx(c.bar(B_FULL + r.slot), stage_bytes * CG);
      const uint32_t bar = CG == 1 ? c.bar(B_FULL + r.slot) : leaders(c.bar(B_FULL + r.slot));
      if constexpr (A_MN) {
#pragma unroll
        for (int i = 0; i < A_BOXES; ++i) load_box4<CG>(at + i * BOX, ma, bar, ax[i], kt * BK, ah[i], ke);
      } else {
        load_box4<CG>(at, ma, bar, ax[0], m0, ah[0], w.entry);
        ax[0] += BK;
        if (ax[0] >= p.a_hd) { ax[0] = 0; ++ah[0]; }
      }
      if constexpr (B_MN) {
#pragma unroll
        for (int i = 0; i < B_BOXES; ++i)
          if (64 * i < rows_b) load_box4<CG>(bt + i * BOX, mb, bar, bx[i], kt * BK, bh[i], ke);
      } else {
        load_box4<CG>(bt, mb, bar, k * BK, n0, 0, 0);
      }
      if (++kt == p.ks_entry && A_MN) { kt = 0; ++ke; }
      r.next(p.stages);
    }
  }
out:
  // every copy has landed, and every MMA has read its operands, before the CTA may end
  for (int s = 0; s < p.stages; ++s) {
    if (!c.wait(B_EMPTY + r.slot, r.turn ^ 1u)) break;
    r.next(p.stages);
  }
}

// LONG: long sums go to the result warps in runs of about most_steps steps, which add them up in fp32 rounded to nearest.  The tensor cores truncate, in one direction: over 384 instructions (6144
// columns) that left 7e-6 of a product, which a result in fp32 shows.  One in bf16, whose rounding is 2^-8 at most, does not; but what is left grows with the sum, and a weight's gradient would carry it in
// every element: of products of one sign 8e-5 over 16384 elements, 1.9e-4 over 32768, 3.9e-4 over 65536, 3.5e-3 over 524288, in runs of 256 steps 1e-4 at any length (65536 x 2048 by 2048 in one run 412 us,
// in runs 421).  A tile's first run is the longest: the tile before it is read out meanwhile.
constexpr int most_steps(bool f32) { return f32 ? 18 : 256; }
struct Runs {
  int first, rest;
  AS_DEV Runs(int steps, int most) {
    const int n = (steps + most - 1) / most;
    first = n == 1 ? steps : (4 * steps + 3 * n - 1) / (3 * n);
    rest = n == 1 ? 1 : (steps - first + n - 2) / (n - 1);
  }
};
template <int CG, bool A_MN, bool B_MN, bool LONG>
AS_DEV void lin_issue(const GemmParams& p, const Ctx<CG>& c) {
  const uint32_t stage_bytes = (uint32_t)(BM + p.bn / CG) * BK * 2;
  const uint32_t idesc = make_idesc(BM * CG, 0, A_MN, B_MN) | (uint32_t)(p.bn >> 3) << 17;
  Ring r;
  uint32_t buf = 0, turn = 0;
  for (long long u = c.unit; u < p.units; u += c.step) {
    const Unit w = unit_of<CG>(p, u);
    const Runs runs(w.k1 - w.k0, p.run);
    int k = w.k0;
    do {
    const int first = k, end = LONG ? min(w.k1, k + (k == w.k0 ? runs.first : runs.rest)) : w.k1;
    if (!c.wait(B_AEMPTY + buf, turn ^ 1u)) return;
    const uint32_t d = c.tmem + buf * 256u;
    for (; k < end; ++k) {
      if (!c.wait(B_FULL + r.slot, r.turn)) return;
      tc_fence_after();
      const uint32_t at = c.sbase + STAGES_OFF + (uint32_t)r.slot * stage_bytes;
      const uint64_t da = make_sdesc(at, A_MN ? BOX : 16, 1024), db = make_sdesc(at + BM * BK * 2, B_MN ? BOX : 16, 1024);
#pragma unroll
      for (int i = 0; i < BK / 16; ++i) mma<CG>(d, da + (A_MN ? 128 : 2) * i, db + (B_MN ? 128 : 2) * i, idesc, k > first || i > 0 ? 1u : 0u);
      commit<CG>(c.bar(B_EMPTY + r.slot));
      r.next(p.stages);
    }
    commit<CG>(c.bar(B_AFULL + buf));
    buf ^= 1u;
    if (buf == 0) turn ^= 1u;
    } while (LONG && k < w.k1);
  }
}

// A box's rows in a matrix: they are of one entry, and fewer than 32 only at its end, where a copy is cut off; else there is none.
struct Box { unsigned batch, token; bool whole; };
AS_DEV Box box_of(const Rows& m, bool boxes, int m0, int rows) {
  if (!boxes) return {0u, 0u, false};
  const unsigned b = m.batched ? (unsigned)m0 / m.tokens : 0u, t = (unsigned)m0 - b * m.tokens, end = t + (unsigned)max(rows, 0);
  return {b, t, rows == 32 ? end <= m.tokens : end == m.tokens};
}
struct At { int x, t, h, b; };
AS_DEV At at_of(const Rows& m, const Box& box, int n, int N) {
  const unsigned head = m.hd == N ? 0u : (unsigned)n / (unsigned)m.hd;
  return {n - (int)head * m.hd, (int)box.token, (int)head, (int)box.batch};
}
// A warp's two strips, used in turn.
struct Strips {
  uint32_t at, bar;                           // the first one; its barrier, told when a residual has come
  uint32_t slot, turns;                       // the one that is used next; parities of both barriers
  AS_DEV uint32_t strip() const { return at + slot * STRIP; }
};
// 16 bytes of this lane's row of the strip.
AS_DEV void put16(uint32_t strip, int lane, int i, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(strip + swz64(lane, i)), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
AS_DEV void get16(uint32_t strip, int lane, int i, uint32_t (&w)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(strip + swz64(lane, i)) : "memory");
}
// The strip, as it has been written by its warp, to columns n ... of a matrix.
AS_DEV void send_box(const CUtensorMap* map, const Rows& m, const Box& box, Strips& s, int lane, int rows, int n, int N) {
  fence_proxy_async();
  __syncwarp();
  if (lane == 0 && rows > 0 && n < N) {
    const At a = at_of(m, box, n, N);
    store_box(map, s.strip(), a.x, a.t, a.h, a.b);
  }
  if (lane == 0) tma_store_commit();          // (one group for every use of a strip, whether there is something to store or not)
  s.slot ^= 1u;
}
// The strip that is used next has been read by the copy out of it, the last but one.
AS_DEV void wait_strip(int lane) {
  if (lane == 0) tma_store_wait_read_but_last();
  __syncwarp();
}
// This lane's row of 32 values as bf16 through a strip.
AS_DEV void leave_bf16(const CUtensorMap* map, const Rows& m, const Box& box, Strips& s, int lane, int rows, int n, int N, const float (&x)[32]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    put16(s.strip(), lane, i, pack_bf16(x[8 * i], x[8 * i + 1]), pack_bf16(x[8 * i + 2], x[8 * i + 3]), pack_bf16(x[8 * i + 4], x[8 * i + 5]), pack_bf16(x[8 * i + 6], x[8 * i + 7]));
  send_box(map, m, box, s, lane, rows, n, N);
}
AS_DEV void leave_f32(const CUtensorMap* map, const Rows& m, const Box& box, Strips& s, int lane, int rows, int n, int N, const float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) put16(s.strip(), lane, i, __float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
  send_box(map, m, box, s, lane, rows, n, N);
}
// The residual's box of columns n ... on its way to the strip that is used next, which is free.
AS_DEV void fetch_box(const CUtensorMap* map, const Rows& m, const Box& box, const Strips& s, int lane, int n, int N) {
  if (lane == 0) {
    const uint32_t bar = s.bar + 8 * s.slot;
    const At a = at_of(m, box, n, N);
    mbar_expect_tx(bar, STRIP);
    load_box4<1>(s.strip(), map, bar, a.x, a.t, a.h, a.b);
  }
}
AS_DEV bool wait_box(Strips& s, const WaitCtx& wc) {
  const bool ok = mbar_wait_warp(s.bar + 8 * s.slot, s.turns >> s.slot & 1u, wc);
  s.turns ^= 1u << s.slot;
  return ok;
}

// 16 columns of 32 rows through a strip, plus a residual, four lanes a row: layouts, alignments and mixtures of types that have no boxes, and sums of parts.
struct Target { Rows m; bool f32; };
AS_DEV void leave_rows(const Target& to, const Target& res, bool vec, uint32_t strip, int lane, int m0, int rows, int n0, int N, const float* x) {
  const int n = n0 + 4 * (lane & 3), row = lane / 4;
  const bool adds = res.m.data != nullptr;
  if (lane == 0) tma_store_wait_read();
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) put16(strip, lane, i, __float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
  __syncwarp();
  if (vec && n < N) {
    auto value = [&](int i) {
      uint32_t w[4];
      get16(strip, i * 8 + row, lane & 3, w);
      return make_float4(__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3]));
    };
    {
      const long long oc = to.m.col((unsigned)n), rc = adds ? res.m.col((unsigned)n) : 0;
      float4 r[4];
      if (adds) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = i * 8 + row < rows ? ld4(res.m.data, res.f32, res.m.row((unsigned)(m0 + i * 8 + row)) + rc) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float4 v = value(i);
        if (adds) { v.x += r[i].x; v.y += r[i].y; v.z += r[i].z; v.w += r[i].w; }
        if (i * 8 + row < rows) st4(to.m.data, to.f32, to.m.row((unsigned)(m0 + i * 8 + row)) + oc, v);
      }
    }
  }
  if (!vec) {                                 // element by element, so that 16 lanes move a row's run
    const int c = lane & 15, col = n0 + c;
    const bool in = col < N;
    const long long oc = in ? to.m.col((unsigned)col) : 0, rc = in && adds ? res.m.col((unsigned)col) : 0;
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
      const int r = 2 * i + lane / 16;
      float v;
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(strip + swz64(r, c / 4) + (uint32_t)(c % 4) * 4u) : "memory");
      if (!in || r >= rows) continue;
      const unsigned m = (unsigned)(m0 + r);
      if (adds) v += ld1(res.m.data, res.f32, res.m.row(m) + rc);
      st1(to.m.data, to.f32, to.m.row(m) + oc, v);
    }
  }
  __syncwarp();
}

// A vector's values of this strip, a column a lane: x = f(x, value).  (Exchanged between the lanes: there is no room beside the stages to read them from, and from global memory, the same
// 16 bytes for all lanes at a time, they made a tile's results a quarter longer.)
template <typename F>
AS_DEV void with_vector(float mine, float (&x)[32], F f) {
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = f(x[i], __shfl_sync(0xffffffffu, mine, i));
}
AS_DEV float add_(float a, float b) { return a + b; }
AS_DEV float mul_(float a, float b) { return a * b; }

// Results of a tile: this warp's 32 rows, 32 of every 128 columns.  LONG: of sums that come in runs.
struct ResultMaps { const CUtensorMap *out, *pre, *res; };
template <int CG, bool LONG>
AS_DEV void lin_results(const GemmParams& p, const Ctx<CG>& c, const ResultMaps& maps, int lane, int warp) {
  const Epilogue& e = p.e;
  const int quarter = (warp + FIRST_RESULT) & 3, group = warp >> 2;         // (a warp reaches the quarter of tensor memory that its number in the CTA says)
  const uint32_t lanes = (uint32_t)quarter * 32u << 16;
  Strips strips{c.sbase + STRIPS_OFF + (uint32_t)warp * (2 * STRIP), c.bar(B_RES + 2 * warp), 0u, 0u};
  uint32_t buf = 0, turn = 0;
  auto give_back = [&] {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) arrive_leader<CG>(c.bar(B_AEMPTY + buf));
  };
  auto next_buffer = [&] {
    buf ^= 1u;
    if (buf == 0) turn ^= 1u;
  };
  for (long long u = c.unit; u < p.units; u += c.step) {
    const Unit w = unit_of<CG>(p, u);
    const int t0 = w.t0 + (int)c.rank * BM + quarter * 32, m0 = w.entry * p.T + t0, rows = min(32, p.T - t0);
    // The residual comes a box ahead of its sums, the first one while the products run.  (From the warps' own loads, four lanes a row, 32760 x 6144 by 1536 onto fp32 took 543 us.)
    const bool boxed = [&] { return e.res_boxes && box_of(e.out, e.boxes, m0, rows).whole && box_of(e.res, true, m0, rows).whole; }();
    const int wide = e.out_f32 ? 16 : 32, boxes = 32 / wide;                  // columns of a box, boxes of a strip's width
    auto fetch = [&](int n) { fetch_box(maps.res, e.res, box_of(e.res, true, m0, rows), strips, lane, n, e.N); };
    // biases and gates, a column a lane; gates of rows that do not share them are read row by row
    const unsigned gate_row = e.gate_rows == 0u || rows <= 0 ? 0u : (unsigned)m0 / e.gate_rows;
    const bool gates_alike = e.gate_rows == 0u || rows <= 0 || gate_row == (unsigned)(m0 + rows - 1) / e.gate_rows;
    auto mine = [&](const void* v, bool f32, long long at, int j) {
      const int n = w.n0 + 32 * group + 128 * j + lane;
      return v != nullptr && n < e.N ? ld1(v, f32, at + n) : 0.f;
    };
    bool fetched = boxed && rows > 0 && 32 * group < p.bn;
    if (fetched) {
      fence_proxy_async();                    // the tile before this one may have left its rows through the strip without a copy: its reads come ahead of the copy's writes
      wait_strip(lane);
      fetch(w.n0 + 32 * group);
    }
    float bias[2], gate[2];
    auto vectors = [&] {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        bias[j] = mine(e.bias, e.bias_f32, 0, j);
        gate[j] = mine(e.gate, e.gate_f32, gate_row * e.gate_stride, j);
      }
    };
    if constexpr (!LONG) vectors();
    if constexpr (LONG) {
      // the runs' sums, in registers; with the last run's they go back to where that one lies
      const Runs runs(w.k1 - w.k0, p.run);
      if (runs.first < w.k1 - w.k0) {
        float x[8][8];                        // columns 32 group + 128 (i / 4) + 8 (i % 4)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k) x[i][k] = 0.f;
        bool ok = true;
        for (int k = w.k0 + runs.first;; k += runs.rest) {               // where the run ends
          ok = mbar_wait_warp(c.bar(B_AFULL + buf), turn, c.wc);
          if (!ok) break;
          tc_fence_after();
          const bool last = k >= w.k1;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int c0 = 32 * group + 128 * (i / 4) + 8 * (i % 4);
            if (c0 < p.bn) {
              float y[8];
              tmem_ld8(c.tmem + lanes + buf * 256u + c0, y);
#pragma unroll
              for (int q = 0; q < 8; ++q) x[i][q] += y[q];
              if (last) tmem_st8(c.tmem + lanes + buf * 256u + c0, x[i]);
            }
          }
          if (last) break;
          give_back();
          next_buffer();
        }
        if (!ok) break;
        tmem_st_wait();
      } else {
        if (!mbar_wait_warp(c.bar(B_AFULL + buf), turn, c.wc)) break;
        tc_fence_after();
      }
    } else {
      if (!mbar_wait_warp(c.bar(B_AFULL + buf), turn, c.wc)) break;
      tc_fence_after();
    }
    if constexpr (LONG) vectors();
    if (32 * group >= p.bn) give_back();
    bool ok = true;
#pragma unroll 1
    for (int j = 0; j < 2; ++j) {
      const int c0 = 32 * group + 128 * j, n0 = w.n0 + c0;
      if (c0 >= p.bn) break;
      uint32_t raw[32];
      tmem_ld32(c.tmem + lanes + buf * 256u + c0, raw);
      tmem_ld_wait(raw);
      if (c0 + 128 >= p.bn) give_back();      // this warp has read its part of the accumulator
      float(&x)[32] = reinterpret_cast<float(&)[32]>(raw);
      if (p.part != nullptr) {
        const Target to{Rows{p.part + (long long)w.part * p.M * p.part_pitch, 0, 0, p.part_pitch, 1u, 1, 0ull, false, false}, true};
#pragma unroll
        for (int h = 0; h < 2; ++h) leave_rows(to, {}, true, strips.at, lane, m0, rows, n0 + 16 * h, e.N, x + 16 * h);
        continue;
      }
      if (e.bias != nullptr) with_vector(j == 0 ? bias[0] : bias[1], x, add_);
      if (e.pre.data != nullptr) {
        const Box box = box_of(e.pre, e.pre_boxes, m0, rows);
        if (box.whole) {
          wait_strip(lane);
          leave_bf16(maps.pre, e.pre, box, strips, lane, rows, n0, e.N, x);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) leave_rows({e.pre, false}, {}, e.vec, strips.at, lane, m0, rows, n0 + 16 * h, e.N, x + 16 * h);
        }
      }
      with_activation(e.act, [&](auto a) {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = activated<decltype(a)::value>(x[i]);
      });
      if (e.gate != nullptr && gates_alike) {
        with_vector(j == 0 ? gate[0] : gate[1], x, mul_);
      } else if (e.gate != nullptr) {
        const long long at = (long long)((unsigned)(m0 + min(lane, rows - 1)) / e.gate_rows) * e.gate_stride;
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] *= n0 + i < e.N ? ld1(e.gate, e.gate_f32, at + n0 + i) : 0.f;
      }
      const Box box = box_of(e.out, e.boxes, m0, rows);
      if (box.whole && (boxed || e.res.data == nullptr)) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          if (q >= boxes) break;
          const int n = n0 + 16 * q;
          if (fetched) {
            ok = wait_box(strips, c.wc);
            if (!ok) break;
            uint32_t r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              get16(strips.strip(), lane, i, r);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if (wide == 16) {
                  x[16 * q + 4 * i + k] += __uint_as_float(r[k]);
                } else if (q == 0) {
                  x[8 * i + 2 * k] += __uint_as_float(r[k] << 16);
                  x[8 * i + 2 * k + 1] += __uint_as_float(r[k] & 0xffff0000u);
                }
              }
            }
          } else {
            wait_strip(lane);
          }
          if (wide == 16) leave_f32(maps.out, e.out, box, strips, lane, rows, n, e.N, x + 16 * q);
          else if (q == 0) leave_bf16(maps.out, e.out, box, strips, lane, rows, n, e.N, x);
          if (fetched && (q + 1 < boxes || c0 + 128 < p.bn && j == 0)) {
            wait_strip(lane);
            fetch(q + 1 < boxes ? n + 16 : n0 + 128);
          }
        }
        if (!ok) break;
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) leave_rows({e.out, e.out_f32}, {e.res, e.res_f32}, e.vec, strips.at, lane, m0, rows, n0 + 16 * h, e.N, x + 16 * h);
      }
    }
    if (!ok) break;
    next_buffer();
  }
  if (lane == 0) tma_store_wait_read();       // (the writes land by the end of the kernel)
}

// A tile whose summed index is shared by a cluster of CTAs: each leaves its sums in its shared memory, in fp32 and where the stages were, and adds up a part of the tile's 4-column pieces over all of
// them, in the order of their ranks, and does what follows.
constexpr int PART_PAD = 16;                  // bytes behind a row of sums, so that rows begin in other banks
AS_DEV void part_leave(const GemmParams& p, const Ctx<1>& c, int lane, int warp) {
  const int quarter = (warp + FIRST_RESULT) & 3, group = warp >> 2;
  if (!mbar_wait_warp(c.bar(B_AFULL), 0, c.wc)) return;
  tc_fence_after();
  const uint32_t row = c.sbase + STAGES_OFF + (uint32_t)(quarter * 32 + lane) * (uint32_t)(p.bn * 4 + PART_PAD);
  for (int c0 = 32 * group; c0 < p.bn; c0 += 128) {
    uint32_t x[32];
    tmem_ld32(c.tmem + ((uint32_t)quarter * 32u << 16) + c0, x);
    tmem_ld_wait(x);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row + c0 * 4 + i * 16), "r"(x[4 * i]), "r"(x[4 * i + 1]), "r"(x[4 * i + 2]), "r"(x[4 * i + 3]) : "memory");
  }
}
// A thread keeps to its columns, whose vectors it fetches ahead of the meeting, and takes two rows at once: what this step costs is latency, of the cluster's shared memory and of what follows.
AS_DEV void part_add(const GemmParams& p, const Ctx<1>& c, const Unit& w, const Column4& cols, int rank) {
  const int across = p.bn / 4, rows = LIN_THREADS / across, piece = threadIdx.x % across, n = w.n0 + 4 * piece;
  const int first = BM * rank / p.parts + threadIdx.x / across, end = min(BM * (rank + 1) / p.parts, p.T - w.t0);
  if (threadIdx.x >= rows * across || n >= p.e.N) return;
  const uint32_t at = c.sbase + STAGES_OFF + (uint32_t)piece * 16u, pitch = (uint32_t)(p.bn * 4 + PART_PAD);
  for (int r = first; r < end; r += 2 * rows) {
    float4 f[2];
    for (int q0 = 0; q0 < p.parts; q0 += 4) {
      float4 v[4][2];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q0 + q >= p.parts) continue;
        uint32_t from;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(at), "r"(q0 + q));
#pragma unroll
        for (int i = 0; i < 2; ++i)           // (a row behind the last one is read where it would be, in the same tile or its stages, and not used)
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(v[q][i].x), "=f"(v[q][i].y), "=f"(v[q][i].z), "=f"(v[q][i].w) : "r"(from + (uint32_t)min(r + i * rows, BM - 1) * pitch) : "memory");
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q0 + q >= p.parts) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (q0 + q == 0) f[i] = v[0][i];
          else { f[i].x += v[q][i].x; f[i].y += v[q][i].y; f[i].z += v[q][i].z; f[i].w += v[q][i].w; }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (r + i * rows < end) finish4(p.e, cols, w.entry * p.T + w.t0 + r + i * rows, n, f[i]);
  }
}

enum { PLAIN = 0, LONG_SUMS = 1, SHARED = 2 };  // SHARED: p.parts CTAs of a cluster share a tile, one tile each cluster (CG == 1)
// A CTA's (or a pair's) units: `first`, first + step, ...
template <int CG, bool A_MN, bool B_MN, int MODE>
AS_DEV void lin_run(const CUtensorMap* ma, const CUtensorMap* mb, const ResultMaps& results, const GemmParams& p, unsigned first, unsigned step) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);      // the same in both CTAs of a pair
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + 8 * B_COUNT);
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + 8 * B_COUNT + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr bool LONG = MODE == LONG_SUMS;
  Ctx<CG> c{smem_u32(smem), 0u, WaitCtx{p.status, abort_flag}, CG == 1 ? 0u : cta_rank(), first, step};
  if (threadIdx.x < B_COUNT) {                 // a barrier a thread
    const bool given_back = threadIdx.x == B_AEMPTY || threadIdx.x == B_AEMPTY + 1;
    mbar_init(c.bar((int)threadIdx.x), given_back ? RESULT_WARPS * CG : 1);
    fence_barrier_init();
    fence_proxy_async();
  }
  if (threadIdx.x == LIN_THREADS - 1) {
    *abort_flag = 0u;
    tma_prefetch_desc(ma); tma_prefetch_desc(mb);
  }
  if (warp == 2) { alloc_tmem<CG>(smem_u32(tmem_slot)); griddep_launch(); }
  tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2) cluster_sync();       // the peer's barriers stand before anything arrives there
  tc_fence_after();
  c.tmem = *tmem_slot;
  griddep_wait();
  if (warp == 0) {
    if (elect_one()) lin_copies<CG, A_MN, B_MN>(p, c, ma, mb);
    __syncwarp();
  } else if (warp == 1) {
    if (c.rank == 0 && elect_one()) lin_issue<CG, A_MN, B_MN, LONG>(p, c);
    __syncwarp();
  } else if (warp >= FIRST_RESULT) {
    if constexpr (MODE == SHARED) part_leave(p, c, lane, warp - FIRST_RESULT);
    else lin_results<CG, LONG>(p, c, results, lane, warp - FIRST_RESULT);
  }
  if constexpr (MODE == SHARED) {
    const Unit w = unit_of<1>(p, c.unit);
    const Column4 cols = columns_of(p.e, w.n0 + 4 * (threadIdx.x % (p.bn / 4)));
    cluster_sync();                            // all sums of the tile stand
    part_add(p, c, w, cols, (int)cta_rank());
  }
  if (*abort_flag != 0u) {                     // a wait ran out: copies and MMAs under way get 20 us (they take two) before memory is given back
    const long long t0 = clock64();
    while (clock64() - t0 < 40000) {}
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2 || MODE == SHARED) cluster_sync();       // nothing of this CTA is reached from the others any more
  if (warp == 2) {
    tc_fence_after();
    free_tmem<CG>(c.tmem);
  }
}
template <int CG, bool A_MN, bool B_MN, int MODE>
__global__ void __launch_bounds__(LIN_THREADS, 1)
linear_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb, const __grid_constant__ CUtensorMap mo, const __grid_constant__ CUtensorMap mp,
              const __grid_constant__ CUtensorMap mr, const __grid_constant__ GemmParams p) {
  lin_run<CG, A_MN, B_MN, MODE>(&ma, &mb, ResultMaps{&mo, &mp, &mr}, p, blockIdx.x / CG, gridDim.x / CG);
}
// Both products of a backward pass at once, dx by the first CTAs and dw by the others: small ones, each of which is mostly its launch, set-up, first copies and read-out (300 x 512 by 256, dx and dw one
// after the other 13.8 us, at once 7.0; 1000 x 1536 by 1536 23 and 14; 7800 rows 72 and 62; 16 x 4096 by 4096, a stream of w that half of the SMs ask for, 28 and 30).
struct Two { CUtensorMap a[2], b[2], out[2]; GemmParams p[2]; int first; };
__global__ void __launch_bounds__(LIN_THREADS, 1) linear_two_kernel(const __grid_constant__ Two t) {
  const unsigned first = (unsigned)t.first;
  if (blockIdx.x < first) lin_run<1, false, true, PLAIN>(&t.a[0], &t.b[0], ResultMaps{&t.out[0], &t.out[0], &t.out[0]}, t.p[0], blockIdx.x, first);
  else lin_run<1, true, true, PLAIN>(&t.a[1], &t.b[1], ResultMaps{&t.out[1], &t.out[1], &t.out[1]}, t.p[1], blockIdx.x - first, gridDim.x - first);
}

// Sums of parts, in their order, and what follows them: four columns a thread.
struct FinishParams { Epilogue e; const float* part; long long pitch; int M, parts; unsigned pieces; };
__global__ void __launch_bounds__(256) finish_kernel(const __grid_constant__ FinishParams p) {
  griddep_launch();
  const int across = (int)(p.pitch / 4);
  griddep_wait();
  for (unsigned i = blockIdx.x * 256u + threadIdx.x; i < (unsigned)p.pieces; i += gridDim.x * 256u) {
    const int m = (int)(i / (unsigned)across), n = (int)(i - (unsigned)m * (unsigned)across) * 4;
    if (n >= p.e.N) continue;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const Column4 cols = columns_of(p.e, n);
    for (int q0 = 0; q0 < p.parts; q0 += 8) {
      float4 x[8];
#pragma unroll
      for (int q = 0; q < 8; ++q)
        x[q] = q0 + q < p.parts ? *reinterpret_cast<const float4*>(p.part + ((long long)(q0 + q) * p.M + m) * p.pitch + n) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int q = 0; q < 8; ++q) { v.x += x[q].x; v.y += x[q].y; v.z += x[q].z; v.w += x[q].w; }
    }
    finish4(p.e, cols, m, n, v);
  }
}

// ---------------------------------------------------------------- few rows
// Few rows of x: w is read by all SMs, into the operands of the warps' own matrix instructions (16 rows of w, 8 of x, 16 columns), as a tile of the pair would be empty but for some rows
// and few CTAs would walk all columns.  `split` warps share 16 rows of w (of 8 NT of x), every split-th block of 64 columns each, a CTA has 16 / split such tiles at once.  Which columns an instruction
// calls its k-th does not matter as long as both operands agree: a lane holds columns 8 q .. 8 q + 7 of each half of its rows' block, so that four
// lanes copy 64 bytes in a run.  The warps' sums meet in shared memory, in the order of the warps.
// Bound by the bytes of w and the latency of memory: operands come by asynchronous copies into slots that a warp alone reads, blocks ahead and on into the next unit.
constexpr int FEW_WARPS = 16, FEW_ROWS_W = 16;
__host__ __device__ constexpr int few_ahead(int nt) { return nt == 1 ? 4 : 3; }
__host__ __device__ constexpr int few_slot(int nt) { return (4 + 2 * nt) * 512; }
constexpr int few_smem(int nt) { return FEW_WARPS * few_ahead(nt) * few_slot(nt); }

struct FewParams {
  Epilogue e;
  Rows x;
  const bf* w;
  long long w_pitch;
  int M, K, units, split;                   // units: a CTA's tiles of 16 rows of w
};
AS_DEV void few_copy_w(uint32_t dst, const void* src, int bytes) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory"); }
AS_DEV void few_copy_x(uint32_t dst, const void* src, int bytes) { asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory"); }
AS_DEV void few_read(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

template <int NT>
__global__ void __launch_bounds__(FEW_WARPS * 32, 1) linear_few_kernel(const __grid_constant__ FewParams p) {
  constexpr int AHEAD = few_ahead(NT), SLOT = few_slot(NT);
  griddep_launch();
  extern __shared__ __align__(16) uint8_t slots[];
  __shared__ float sums[2][FEW_WARPS][8 * NT][FEW_ROWS_W + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane / 4, q = lane % 4;
  const int kb = (p.K + BK - 1) / BK;
  const uint32_t mine = smem_u32(slots) + (uint32_t)warp * (AHEAD * SLOT);
  const int part = warp & (p.split - 1), tile = warp / p.split, tiles = FEW_WARPS / p.split, m0 = blockIdx.y * (8 * NT);
  griddep_wait();
  int unit = blockIdx.x, block = part, slot = 0;                      // what is asked for next
  auto ask = [&] {
    if (block < kb && unit < p.units) {
      const uint32_t own = mine + slot * SLOT + lane * 16;
      const int c = block * BK + q * 8, n = (unit * tiles + tile) * FEW_ROWS_W + g;
#pragma unroll
      for (int i = 0; i < 2; ++i) {                                   // 8 columns each
        const int bytes = 2 * max(0, min(8, p.K - c - 32 * i)), c1 = bytes > 0 ? c + 32 * i : 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) few_copy_w(own + (2 * h + i) * 512, p.w + (long long)min(n + 8 * h, p.e.N - 1) * p.w_pitch + c1, bytes);
        const long long col = p.x.col((unsigned)c1);
#pragma unroll
        for (int t = 0; t < NT; ++t)        // (a row that is not there leaves its results, which are not written, to chance)
          if (m0 + 8 * t + g < p.M) few_copy_x(own + (4 + 2 * t + i) * 512, static_cast<const bf*>(p.x.data) + p.x.row((unsigned)(m0 + 8 * t + g)) + col, bytes);
      }
      if (++slot == AHEAD) slot = 0;
      if ((block += p.split) >= kb) {
        block = part;
        unit += gridDim.x;
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");              // (an empty group where there is nothing left: the waits below count groups)
  };
#pragma unroll
  for (int i = 0; i < AHEAD - 1; ++i) ask();
  int take = 0, turn = 0;
  for (int u = blockIdx.x; u < p.units; u += gridDim.x, turn ^= 1) {
    float acc[NT][4] = {}, run[NT][4] = {};                           // (matrix instructions truncate their sums: runs of 32 of them are added up rounded to nearest)
    int in_run = 0;
    for (int k = part; k < kb; k += p.split) {
      ask();                                                          // (a lane fills and reads its own 16 bytes of each piece: nothing to wait for in the other lanes)
      asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
      const uint32_t own = mine + take * SLOT + lane * 16;
      if (++take == AHEAD) take = 0;
      uint32_t w[2][2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        few_read(own + i * 512, w[0][i]);
        few_read(own + (2 + i) * 512, w[1][i]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        uint32_t x[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) few_read(own + (4 + 2 * t + i) * 512, x[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                       : "+f"(run[t][0]), "+f"(run[t][1]), "+f"(run[t][2]), "+f"(run[t][3])
                       : "r"(w[0][i / 2][2 * (i % 2)]), "r"(w[1][i / 2][2 * (i % 2)]), "r"(w[0][i / 2][2 * (i % 2) + 1]), "r"(w[1][i / 2][2 * (i % 2) + 1]),
                         "r"(x[i / 2][2 * (i % 2)]), "r"(x[i / 2][2 * (i % 2) + 1]));
      }
      if (++in_run == 8 || k + p.split >= kb) {
        in_run = 0;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) { acc[t][j] += run[t][j]; run[t][j] = 0.f; }
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) sums[turn][warp][8 * t + 2 * q + j % 2][g + 8 * (j / 2)] = acc[t][j];
    __syncthreads();                                                  // (one for a unit: the next one's sums go to the other half)
    for (int i = threadIdx.x; i < tiles * 8 * NT * FEW_ROWS_W; i += FEW_WARPS * 32) {
      const int ti = i / (8 * NT * FEW_ROWS_W), mi = i / FEW_ROWS_W % (8 * NT), j = i % FEW_ROWS_W, m = m0 + mi, n = (u * tiles + ti) * FEW_ROWS_W + j;
      if (m < p.M && n < p.e.N) {
        float f = 0.f;
        for (int k = 0; k < p.split; ++k) f += sums[turn][ti * p.split + k][mi][j];
        const Epilogue& e = p.e;
        if (e.bias != nullptr) f += ld1(e.bias, e.bias_f32, n);
        if (e.pre.data != nullptr) st1(e.pre.data, false, e.pre.row((unsigned)m) + e.pre.col((unsigned)n), f);
        f = activated(f, e.act);
        if (e.gate != nullptr) f *= ld1(e.gate, e.gate_f32, (e.gate_rows == 0u ? 0ll : (long long)((unsigned)m / e.gate_rows) * e.gate_stride) + n);
        if (e.res.data != nullptr) f += ld1(e.res.data, e.res_f32, e.res.row((unsigned)m) + e.res.col((unsigned)n));
        st1(e.out.data, e.out_f32, e.out.row((unsigned)m) + e.out.col((unsigned)n), f);
      }
    }
  }
}

// ---------------------------------------------------------------- dz, and sums over rows
// dz = dy * gate * act'(pre) in bf16, as the other operand of both products is (the tensor cores take two of one type; in tf32, or as the sum of two bf16 values, the products would take twice as long):
// beside the results' own rounding, 1.66e-3 in the mean square, that is another of the same size, 2.34e-3 in all.  With it the sums of dz and
// of dy * act(pre), from the unrounded values, over runs of rows, which do not cross from one gate's rows to another's.  A lane has 8 columns, a warp every eighth row of the run, the next one under way; the warps' sums meet in shared memory in their order.  One pass over dy and pre: HBM bytes (32760 x 6144 from fp32 with silu and a gate's
// gradient 261 us, 6.2 TB/s), in bf16 with an activation the instructions beside them (7800 x 6144 with gelu_tanh 70 us, 4.1 TB/s; with the activation chosen at every value, and both its sigmoids from
// exponentials of their own, 254; with runs for 2.7 turns of the SMs instead of one 76).
struct DzParams {
  Rows dy, pre;
  const void* gate;
  bf* dz;                                    // [M][pitch], or nullptr
  float *part_b, *part_g;                    // [gates * runs][N], or nullptr
  void *dbias, *dgate;                       // where there is one run in all: the sums themselves (bias_f32: dbias's type)
  long long gate_stride, pitch;
  int N, act, rows_gate, runs;               // rows that share a gate; runs of them
  bool gate_f32, bias_f32, vec;
};
constexpr int DZ_COLS = 256;
AS_DEV void unpack8(const uint4& w, float (&f)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(u[i] << 16); f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}

template <int ACT, typename Y, bool OF_GATE>
__global__ void __launch_bounds__(256, 3) dz_kernel(const __grid_constant__ DzParams p) {
  griddep_launch();
  __shared__ float room[8][DZ_COLS + 8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n = blockIdx.x * DZ_COLS + lane * 8, gate = blockIdx.y / p.runs, run = blockIdx.y - gate * p.runs;
  const int r0 = (int)((long long)p.rows_gate * run / p.runs), r1 = (int)((long long)p.rows_gate * (run + 1) / p.runs);
  const unsigned first = (unsigned)(gate * (long long)p.rows_gate);
  griddep_wait();
  const bool keeps = p.pre.data != nullptr, gated = p.gate != nullptr;
  float g[8], sb[8] = {}, sg[8] = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = gated && n + i < p.N ? ld1(p.gate, p.gate_f32, (long long)gate * p.gate_stride + n + i) : 1.f;
  const Y* dy = static_cast<const Y*>(p.dy.data);
  const bf* pre = static_cast<const bf*>(p.pre.data);
  // one row's values on to dz and the sums
  auto take = [&](unsigned m, float (&d)[8], const float (&z)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 a = activated2<ACT>(z[i]);
      if constexpr (OF_GATE) sg[i] = fmaf(d[i], a.x, sg[i]);
      d[i] = d[i] * g[i] * a.y;
      sb[i] += d[i];
    }
    if (p.dz == nullptr) return;
    bf* at = p.dz + (long long)m * p.pitch + n;
    if (n + 8 <= p.N) {
      *reinterpret_cast<uint4*>(at) = make_uint4(pack_bf16(d[0], d[1]), pack_bf16(d[2], d[3]), pack_bf16(d[4], d[5]), pack_bf16(d[6], d[7]));
    } else {
      for (int i = 0; i < 8; ++i)
        if (n + i < p.N) at[i] = __float2bfloat16_rn(d[i]);
    }
  };
  if (n < p.N && p.vec) {
    const long long dc = p.dy.col((unsigned)n), pc = keeps ? p.pre.col((unsigned)n) : 0;
    struct Row { uint4 d[sizeof(Y) / 2], z; };
    auto fetch = [&](unsigned m, Row& v) {
      const uint4* at = reinterpret_cast<const uint4*>(dy + p.dy.row(m) + dc);
#pragma unroll
      for (int i = 0; i < (int)sizeof(Y) / 2; ++i) v.d[i] = at[i];
      v.z = keeps ? *reinterpret_cast<const uint4*>(pre + p.pre.row(m) + pc) : make_uint4(0u, 0u, 0u, 0u);
    };
    auto use = [&](unsigned m, const Row& v) {
      float d[8], z[8];
      if constexpr (sizeof(Y) == 2) unpack8(v.d[0], d);
      else {
        *reinterpret_cast<uint4*>(d) = v.d[0];
        *reinterpret_cast<uint4*>(d + 4) = v.d[1];
      }
      unpack8(v.z, z);
      take(m, d, z);
    };
    Row now, next;
    int r = r0 + warp;
    if (r < r1) fetch(first + (unsigned)r, now);
    for (; r < r1; r += 8) {
      if (r + 8 < r1) fetch(first + (unsigned)(r + 8), next);
      use(first + (unsigned)r, now);
      now = next;
    }
  } else if (n < p.N) {
    for (int r = r0 + warp; r < r1; r += 8) {
      const unsigned m = first + (unsigned)r;
      const long long dr = p.dy.row(m), pr = keeps ? p.pre.row(m) : 0;
      float d[8], z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        d[i] = n + i < p.N ? (float)dy[dr + p.dy.col((unsigned)(n + i))] : 0.f;
        z[i] = keeps && n + i < p.N ? __bfloat162float(pre[pr + p.pre.col((unsigned)(n + i))]) : 0.f;
      }
      take(m, d, z);
    }
  }
  auto leave = [&](const float (&s)[8], float* part, void* sum, bool f32) {
    if (part == nullptr && sum == nullptr) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) room[warp][lane * 8 + i] = s[i];
    __syncthreads();
    const int c = blockIdx.x * DZ_COLS + threadIdx.x;
    if (c < p.N) {
      float f = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) f += room[w][threadIdx.x];
      if (sum != nullptr) st1(sum, f32, c, f);
      else part[(long long)blockIdx.y * p.N + c] = f;
    }
  };
  leave(sb, p.part_b, p.dbias, p.bias_f32);
  if constexpr (OF_GATE) leave(sg, p.part_g, p.dgate, p.gate_f32);
}
template <typename Y>
cudaError_t launch_dz(const DzParams& p, dim3 grid, cudaStream_t st) {
  auto run = [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    return p.part_g != nullptr || p.dgate != nullptr ? as_launch_dependent(dz_kernel<ACT, Y, true>, grid, dim3(256), 0, st, p) : as_launch_dependent(dz_kernel<ACT, Y, false>, grid, dim3(256), 0, st, p);
  };
  switch (p.act) {
    case AS_ACT_RELU: return run(std::integral_constant<int, AS_ACT_RELU>{});
    case AS_ACT_SILU: return run(std::integral_constant<int, AS_ACT_SILU>{});
    case AS_ACT_GELU: return run(std::integral_constant<int, AS_ACT_GELU>{});
    case AS_ACT_GELU_TANH: return run(std::integral_constant<int, AS_ACT_GELU_TANH>{});
    default: return run(std::integral_constant<int, AS_ACT_NONE>{});
  }
}

// Columns' sums over runs of rows, in order: block row 0 all of them (the bias), 1 + i those of gate i.
struct ColumnSumParams { const float *part_b, *part_g; void *dbias, *dgate; int N, runs, gates; bool b_f32, g_f32; };
__global__ void __launch_bounds__(256) column_sum_kernel(const __grid_constant__ ColumnSumParams p) {
  griddep_launch();
  __shared__ float some[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  const bool of_bias = blockIdx.y == 0;
  griddep_wait();
  const float* part = of_bias ? p.part_b : p.part_g;
  if (part == nullptr) return;
  const long long first = of_bias ? 0 : (long long)(blockIdx.y - 1) * p.runs, rows = of_bias ? (long long)p.gates * p.runs : p.runs;
  const long long r0 = first + rows * warp / 8, r1 = first + rows * (warp + 1) / 8;
  float s = 0.f;
  if (c < p.N) {
#pragma unroll 8
    for (long long r = r0; r < r1; ++r) s += part[r * p.N + c];
  }
  some[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < p.N) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += some[i][lane];
    if (of_bias) st1(p.dbias, p.b_f32, c, s);
    else st1(p.dgate, p.g_f32, (long long)(blockIdx.y - 1) * p.N + c, s);
  }
}

// A matrix into rows a multiple of 16 bytes apart, for operands that the copies cannot read as they lie: 8 elements a thread, from two aligned pieces of 16 bytes where both lie within the row, else
// element by element.  (Element by element throughout 2000 x 1535 took 8 us.)
struct GatherParams { Rows x; bf* out; long long pitch; unsigned rows, across; int cols, run; };       // across: pieces of 8 columns; run: columns that lie in a run
struct Gathers { GatherParams of[2]; };      // of one operand or two, at once
__global__ void __launch_bounds__(256) gather_kernel(const __grid_constant__ Gathers g) {
  griddep_launch();
  const GatherParams& p = blockIdx.y == 0 ? g.of[0] : g.of[1];
  griddep_wait();
  const long long pieces = (long long)p.rows * p.across;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (long long)gridDim.x * 256) {
    const unsigned r = (unsigned)(i / p.across);
    const int c = (int)(i - (long long)r * p.across) * 8, first = c / p.run * p.run, last = min(first + p.run, p.cols);      // the run that column c lies in
    const bf* row = static_cast<const bf*>(p.x.data) + p.x.row(r);
    bf* to = p.out + (long long)r * p.pitch + c;
    const bf* at = row + p.x.col((unsigned)c);
    const uintptr_t down = reinterpret_cast<uintptr_t>(at) & ~(uintptr_t)15;
    const int off = (int)(reinterpret_cast<uintptr_t>(at) - down);                       // bytes, even
    if (c + 8 <= last && down >= reinterpret_cast<uintptr_t>(at - (c - first)) && down + (off ? 32 : 16) <= reinterpret_cast<uintptr_t>(at + (last - c))) {
      const uint4 x = *reinterpret_cast<const uint4*>(down), y = off ? *reinterpret_cast<const uint4*>(down + 16) : make_uint4(0u, 0u, 0u, 0u);
      uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
      if (off & 8) { w[0] = w[2]; w[1] = w[3]; w[2] = w[4]; w[3] = w[5]; w[4] = w[6]; w[5] = w[7]; }
      if (off & 4) { w[0] = w[1]; w[1] = w[2]; w[2] = w[3]; w[3] = w[4]; w[4] = w[5]; }
      const uint32_t by = off & 2 ? 16u : 0u;
      *reinterpret_cast<uint4*>(to) = make_uint4(__funnelshift_r(w[0], w[1], by), __funnelshift_r(w[1], w[2], by), __funnelshift_r(w[2], w[3], by), __funnelshift_r(w[3], w[4], by));
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k < p.cols) to[k] = row[p.x.col((unsigned)(c + k))];
    }
  }
}

// ---------------------------------------------------------------- host
using as_lin::Plan;
using as_lin::plan_of;

struct Maps { CUtensorMap a, b, out, pre, res; };
template <int CG, bool A_MN, bool B_MN, int MODE>
cudaError_t launch(const Maps& m, const GemmParams& p, int units, size_t smem, cudaStream_t st) {
  const int together = MODE == SHARED ? p.parts : CG;        // (SHARED: units are CTAs)
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = together; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(units * CG)); cfg.blockDim = dim3(LIN_THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cfg.attrs = attr; cfg.numAttrs = together == 1 ? 1 : 2;
  return cudaLaunchKernelEx(&cfg, linear_kernel<CG, A_MN, B_MN, MODE>, m.a, m.b, m.out, m.pre, m.res, p);
}

// Whether four columns of a matrix move at once.
bool vec4(const as_rows_t& x) {
  return x.data == nullptr || (aligned(x.data, x.dtype == AS_DTYPE_BF16 ? 8 : 16) && ((x.head_dim | x.stride_batch | x.stride_head | x.stride_token) & 3) == 0);
}

// Whether 16 bytes of a matrix move at once.
bool rows_vec16(const as_rows_t& x) { return aligned(x.data, 16) && ((x.stride_batch | x.stride_head | x.stride_token) & (x.dtype == AS_DTYPE_BF16 ? 7 : 3)) == 0; }

// An operand as the copies read it: rows in entries of T.
as_rows_t in_entries(as_rows_t x, long long rows, long long T) {
  if (x.tokens == rows && T != rows) { x.stride_batch = T * x.stride_token; x.tokens = T; }
  return x;
}
as_rows_t plain_rows(const void* data, long long rows, long long cols, long long pitch) {
  as_rows_t x{};
  x.data = const_cast<void*>(data); x.dtype = AS_DTYPE_BF16; x.head_dim = (int32_t)cols; x.tokens = rows; x.stride_token = pitch;
  return x;
}
long long pitch_of(long long cols) { return (cols + 7) / 8 * 8; }
uint64_t up256(uint64_t n) { return (n + 255) & ~255ull; }

// Whether the copies can read a matrix as it lies: strides that are multiples of 16 bytes, heads that boxes of 64 columns do not cross.
bool box_ok(const as_rows_t& x, long long rows, long long cols) {
  if (x.dtype != AS_DTYPE_BF16 || !aligned(x.data, 16)) return false;
  const long long heads = cols / x.head_dim, entries = rows / x.tokens;
  if (heads > 1 && (x.head_dim % 64 != 0 || x.stride_head <= 0 || x.stride_head % 8 != 0)) return false;
  if (x.tokens > 1 && (x.stride_token <= 0 || x.stride_token % 8 != 0)) return false;
  return entries <= 1 || (x.stride_batch > 0 && x.stride_batch % 8 == 0);
}
// The same matrix without entries where their rows go on from one to the next.
as_rows_t joined(as_rows_t x, long long rows) {
  if (x.tokens != rows && (x.tokens == 1 || x.stride_batch == x.tokens * x.stride_token)) {
    if (x.tokens == 1) x.stride_token = x.stride_batch;
    x.tokens = rows;
    x.stride_batch = 0;
  }
  return x;
}
// Entries of few rows leave the tiles of 256 (or steps of 64) that hold them empty: above 1.25 times the rows a copy is shorter.
bool entries_ok(const as_rows_t& x, long long rows) {
  if (x.tokens == rows) return true;
  return (rows / x.tokens) * ((x.tokens + 255) / 256 * 256) * 4 <= std::max<long long>(rows, 256) * 5;
}

// What one product needs and where.
struct Operand { as_rows_t rows; bool copy; as_rows_t from; };       // copy: `from` is brought into a dense form in the workspace first
Operand operand_of(const as_rows_t& x, long long rows, long long cols) {
  Operand o{joined(x, rows), false, x};
  if (!box_ok(o.rows, rows, cols) || !entries_ok(o.rows, rows)) {
    o.copy = true;
    o.rows = plain_rows(nullptr, rows, cols, pitch_of(cols));
  }
  return o;
}
uint64_t copy_bytes(const Operand& o, long long rows) { return o.copy ? up256((uint64_t)rows * (uint64_t)o.rows.stride_token * 2) : 0; }

// Brings operands that need it into the workspace, in one launch.
struct Copy { Operand* o; long long rows, cols; };
cudaError_t run_copies(const Copy (&c)[2], uint8_t*& room, int sms, cudaStream_t st) {
  Gathers g{};
  int n = 0;
  long long ctas = 0;
  for (const Copy& i : c) {
    if (!i.o->copy) continue;
    GatherParams& p = g.of[n++];
    i.o->rows.data = room;
    p.x = rows_of(i.o->from, i.rows, i.cols);
    p.out = reinterpret_cast<bf*>(room); p.pitch = i.o->rows.stride_token;
    p.rows = (unsigned)i.rows; p.across = (unsigned)((i.cols + 7) / 8); p.cols = (int)i.cols;
    p.run = p.x.split ? i.o->from.head_dim : (int)i.cols;
    room += copy_bytes(*i.o, i.rows);
    ctas = std::max(ctas, (i.rows * (long long)p.across + 255) / 256);
  }
  return n == 0 ? cudaSuccess : as_launch_dependent(gather_kernel, dim3((unsigned)std::min<long long>(ctas, 16ll * sms), (unsigned)n), dim3(256), 0, st, g);
}

// One product on the tensor cores.  a [M, K] and b [N, K] by their meaning; A_MN, B_MN: they lie with M (N) in a run, as [K rows, M columns].
struct Product {
  as_rows_t a, b;
  bool a_mn, b_mn;
  long long M, N, K;                         // K: the summed index
  long long T;                               // entries of the rows of results, or of the summed index where a_mn
  Plan plan;
};
uint64_t part_bytes(const Product& q) { return q.plan.parts == 1 || q.plan.shared ? 0 : up256((uint64_t)q.plan.parts * (uint64_t)q.M * (uint64_t)((q.N + 3) / 4 * 4) * 4); }
// Steps of the summed index, which end with its entries.
long long ksteps_of(const Product& q) { return q.a_mn ? (q.K / q.T) * ((q.T + BK - 1) / BK) : (q.K + BK - 1) / BK; }
// Whether a unit's sum is longer than one run.
bool long_sums(const Product& q, const Plan& plan, bool f32) { return (ksteps_of(q) + plan.parts - 1) / plan.parts > most_steps(f32); }
// sms: that it has to itself; alone: beside another product of the same launch, by single CTAs.
Plan plan_for(const Product& q, bool f32, as_fp8_context_t h, int sms, bool alone = true) {
  const long long entries = q.a_mn ? 1 : q.M / q.T;
  return plan_of(entries, q.a_mn ? q.M : q.T, q.M, q.N, ksteps_of(q), q.b_mn, most_steps(f32), sms, alone ? h->clusters : nullptr);
}

struct Prepared { Maps m; GemmParams p; size_t smem; };
// out, pre, res: what the epilogue's matrices are.
cudaError_t prepare(as_fp8_context_t h, const Product& q, const Epilogue& e, const as_rows_t& out, const as_rows_t& pre, const as_rows_t& res, void* part, Prepared& r) {
  const Plan& plan = q.plan;
  GemmParams& p = r.p;
  p.e = e;
  p.status = h->status;
  p.M = (int)q.M;
  p.T = (int)(q.a_mn ? q.M : q.T);
  p.mt_entry = (p.T + BM * plan.cg - 1) / (BM * plan.cg);
  p.bn = plan.bn; p.parts = plan.parts;
  p.nt = (int)((q.N + plan.bn - 1) / plan.bn);
  auto reciprocal = [](unsigned n) { return n == 1u ? 0ull : ~0ull / n + 1ull; };
  p.by_nt = reciprocal((unsigned)p.nt);
  p.by_mt = reciprocal((unsigned)p.mt_entry);
  p.ks_entry = (int)(q.a_mn ? (q.T + BK - 1) / BK : 1);
  p.ksteps = (int)ksteps_of(q);
  p.run = most_steps(e.out_f32);
  p.units = (q.a_mn ? 1 : q.M / q.T) * p.mt_entry * (long long)p.nt * p.parts;
  if (plan.parts > 1 && !plan.shared) { p.part = static_cast<float*>(part); p.part_pitch = (q.N + 3) / 4 * 4; }
  const int stage = (BM + plan.bn / plan.cg) * BK * 2;
  p.stages = std::min((SMEM_MAX - 1024 - STAGES_OFF) / stage, MAX_STAGES);
  r.smem = 1024 + STAGES_OFF + (size_t)p.stages * stage;
  Maps& m = r.m;
  auto boxes = [&](const as_rows_t& x, CUtensorMap* map) {             // (a map that the driver does not take leaves it to the warps)
    const bool spread = (x.tokens == 1 || x.stride_token > 0) && (x.tokens == q.M || x.stride_batch > 0) && (x.head_dim == q.N || x.stride_head > 0);
    return plan.parts == 1 && x.data != nullptr && spread && rows_vec16(x) && (x.head_dim == q.N || x.head_dim % 32 == 0) && as_tc::make_map_strips(map, x, q.M, q.N);
  };
  p.e.boxes = boxes(out, &m.out);
  p.e.pre_boxes = boxes(pre, &m.pre);
  p.e.res_boxes = p.e.boxes && pre.data == nullptr && res.dtype == out.dtype && boxes(res, &m.res);
  const long long a_rows = q.a_mn ? q.K : q.M, a_cols = q.a_mn ? q.M : q.K, b_rows = q.b_mn ? q.K : q.N, b_cols = q.b_mn ? q.N : q.K;
  // (boxes behind the last column of a matrix without heads begin at their column, a multiple of 64, not at what is left of it behind a "head" of any width: a copy has to begin on 16 bytes)
  p.a_hd = q.a.head_dim == a_cols ? INT32_MAX : q.a.head_dim;
  p.b_hd = q.b.head_dim == b_cols ? INT32_MAX : q.b.head_dim;
  if (!as_tc::make_map_boxes(&m.a, in_entries(q.a, a_rows, q.T), a_rows, a_cols, q.a_mn ? 64 : BM) ||
      !as_tc::make_map_boxes(&m.b, q.a_mn ? in_entries(q.b, b_rows, q.T) : q.b, b_rows, b_cols, q.b_mn ? 64 : plan.bn / plan.cg))
    return cudaErrorInvalidValue;
  return cudaSuccess;
}
// Sums of parts, where there are any, behind their product.
cudaError_t finish(as_fp8_context_t h, const Product& q, const GemmParams& p, cudaStream_t st) {
  if (p.part == nullptr) return cudaSuccess;
  FinishParams f{};
  f.e = p.e; f.part = p.part; f.pitch = p.part_pitch; f.M = p.M; f.parts = p.parts;
  f.pieces = (unsigned)(q.M * (p.part_pitch / 4));          // (parts are of results that leave SMs idle: far below 2^32)
  const long long pieces = (f.pieces + 255ll) / 256;
  return as_launch_dependent(finish_kernel, dim3((unsigned)std::min<long long>(pieces, 8ll * h->sms)), dim3(256), 0, st, f);
}
cudaError_t run_product(as_fp8_context_t h, const Product& q, const Epilogue& e, const as_rows_t& out, const as_rows_t& pre, const as_rows_t& res, void* part, cudaStream_t st) {
  const Plan& plan = q.plan;
  Prepared r{};
  if (const cudaError_t err = prepare(h, q, e, out, pre, res, part, r); err != cudaSuccess) return err;
  const Maps& m = r.m;
  const GemmParams& p = r.p;
  const size_t smem = r.smem;
  const int units = plan.shared ? (int)p.units : (int)std::min<long long>(p.units, h->sms / plan.cg);
  cudaError_t err;
  auto run = [&](auto cg) {
    constexpr int CG = decltype(cg)::value;
    auto by_length = [&](auto mode) {
      constexpr int MODE = decltype(mode)::value;
      if (q.a_mn) return launch<CG, true, true, MODE>(m, p, units, smem, st);
      if (q.b_mn) return launch<CG, false, true, MODE>(m, p, units, smem, st);
      return launch<CG, false, false, MODE>(m, p, units, smem, st);
    };
    return long_sums(q, plan, e.out_f32) ? by_length(std::integral_constant<int, LONG_SUMS>{}) : by_length(std::integral_constant<int, PLAIN>{});
  };
  if (plan.shared)
    return q.a_mn ? launch<1, true, true, SHARED>(m, p, units, smem, st) : q.b_mn ? launch<1, false, true, SHARED>(m, p, units, smem, st) : launch<1, false, false, SHARED>(m, p, units, smem, st);
  err = plan.cg == 2 ? run(std::integral_constant<int, 2>{}) : run(std::integral_constant<int, 1>{});
  return err != cudaSuccess ? err : finish(h, q, p, st);
}
// Two products at once.
cudaError_t run_two(as_fp8_context_t h, const Product (&q)[2], const Epilogue (&e)[2], const as_rows_t (&out)[2], void* const (&part)[2], cudaStream_t st) {
  Prepared r[2]{};
  Two t{};
  int ctas[2];
  for (int i = 0; i < 2; ++i) {
    if (const cudaError_t err = prepare(h, q[i], e[i], out[i], as_rows_t{}, as_rows_t{}, part[i], r[i]); err != cudaSuccess) return err;
    t.a[i] = r[i].m.a; t.b[i] = r[i].m.b; t.out[i] = r[i].m.out; t.p[i] = r[i].p;
    ctas[i] = (int)std::min<long long>(r[i].p.units, h->sms / 2);
  }
  t.first = ctas[0];
  if (const cudaError_t err = as_launch_dependent(linear_two_kernel, dim3((unsigned)(ctas[0] + ctas[1])), dim3(LIN_THREADS), std::max(r[0].smem, r[1].smem), st, t); err != cudaSuccess) return err;
  for (int i = 0; i < 2; ++i)
    if (const cudaError_t err = finish(h, q[i], r[i].p, st); err != cudaSuccess) return err;
  return cudaSuccess;
}

bool dtype_ok(int t) { return t == AS_DTYPE_BF16 || t == AS_DTYPE_F32; }
bool act_ok(int a) { return a >= AS_ACT_NONE && a <= AS_ACT_GELU_TANH; }
bool vector_ok(const void* p, int dtype) { return p == nullptr || (dtype_ok(dtype) && aligned(p, dtype == AS_DTYPE_BF16 ? 2 : 4)); }
bool sizes_ok(long long rows, long long cols, long long out_cols) {
  return rows >= 0 && rows <= (1ll << 30) && cols >= 1 && cols <= (1 << 20) && out_cols >= 1 && out_cols <= (1 << 20);
}
bool gate_ok(const void* gate, int dtype, long long gates, long long stride, long long rows, long long n) {
  if (gate == nullptr) return true;
  return vector_ok(gate, dtype) && gates >= 1 && gates <= 65534 && rows % gates == 0 && (gates == 1 || stride >= 0) && n >= 1;
}
// Units of work are counted in 32 bits: an entry's tile of 64 columns for each row at the worst.  (What a device holds has fewer.)
bool units_fit(long long rows, long long cols) { return rows * ((cols + 63) / 64) < (1ll << 32); }
bool heads_fit(const as_rows_t& x, long long cols) { return x.data == nullptr || x.head_dim == cols || cols * (long long)x.head_dim <= (1ll << 32); }

as_status_t device_of(as_fp8_context_t h) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return failed();
  return dev == h->device ? AS_OK : AS_ERR_INVALID_ARG;
}

as_status_t linear_ok(as_fp8_context_t h, const as_linear_t* a) {
  if (h == nullptr || a == nullptr || a->struct_size != sizeof(as_linear_t) || !sizes_ok(a->rows, a->cols, a->out_cols) || !act_ok(a->activation)) return AS_ERR_INVALID_ARG;
  if (!rows_ok(a->x, a->rows, a->cols) || a->x.dtype != AS_DTYPE_BF16 || !rows_ok(a->w, a->out_cols, a->cols) || a->w.dtype != AS_DTYPE_BF16 || a->w.head_dim != a->cols ||
      a->w.tokens != a->out_cols)
    return AS_ERR_INVALID_ARG;
  if (!rows_ok(a->out, a->rows, a->out_cols) || !apart(a->out, a->rows, a->out_cols)) return AS_ERR_INVALID_ARG;
  if (a->residual.data != nullptr && !rows_ok(a->residual, a->rows, a->out_cols)) return AS_ERR_INVALID_ARG;
  if (a->pre.data != nullptr && (!rows_ok(a->pre, a->rows, a->out_cols) || a->pre.dtype != AS_DTYPE_BF16 || !apart(a->pre, a->rows, a->out_cols))) return AS_ERR_INVALID_ARG;
  if (a->rows > 0) {                         // results over the residual itself only
    const void *out = a->out.data, *pre = a->pre.data;
    if (out == a->x.data || out == a->w.data || out == pre || !in_place_ok(a->out, a->residual, a->rows, a->out_cols)) return AS_ERR_INVALID_ARG;
    if (pre != nullptr && (pre == a->x.data || pre == a->w.data || pre == a->residual.data)) return AS_ERR_INVALID_ARG;
  }
  if (!vector_ok(a->bias, a->bias_dtype) || !gate_ok(a->gate, a->gate_dtype, a->gates, a->gate_stride, a->rows, a->out_cols)) return AS_ERR_INVALID_ARG;
  if (!units_fit(a->rows, a->out_cols) || !heads_fit(a->x, a->cols) || !heads_fit(a->out, a->out_cols) || !heads_fit(a->residual, a->out_cols) || !heads_fit(a->pre, a->out_cols)) return AS_ERR_UNSUPPORTED;
  return AS_OK;
}

// Warps that share a tile of w, and how long that takes: turns of all SMs x blocks of a warp, of which a turn's first costs about one more, at 0.95 us a block (up to 8 rows 0.75; 2 rows by
// 9216 x 1536 6.3 us, 16 rows 9.0, by 1536 x 1536 3.2 and 4.3, by 6144 x 6144 14 and 24), from 1.2 us on.  Up to 16 rows always; more of them in parts of 16 where the tile kernel, whose time is its
// plan's and 4.5 us, takes longer (64 rows by 1536 x 1536 8.3, 512 rows 10.4).
struct Few { int split, mt; double ns; };
Few few_of(int M, int N, int K, int sms) {
  const int tiles = (N + FEW_ROWS_W - 1) / FEW_ROWS_W, kb = (K + BK - 1) / BK, mt = M <= 8 ? 1 : (M + 15) / 16;
  Few best{1, mt, 1e300};
  for (int split = 1; split <= FEW_WARPS; split *= 2) {
    const long long units = (tiles + FEW_WARPS / split - 1) / (FEW_WARPS / split) * (long long)mt;
    const double t = 1200. + (M <= 8 ? 750. : 950.) * (double)((units + sms - 1) / sms) * ((kb + split - 1) / split + 1);
    if (t <= best.ns) best = {split, mt, t};
  }
  return best;
}

struct LinearPlan { Operand x, w; Product q; bool few; uint64_t bytes; };
LinearPlan plan_linear(as_fp8_context_t h, const as_linear_t& a) {
  LinearPlan l{};
  l.w = operand_of(a.w, a.out_cols, a.cols);
  // few rows read x where it lies: 8 columns at a time
  l.x = operand_of(a.x, a.rows, a.cols);
  l.q = Product{l.x.rows, l.w.rows, false, false, a.rows, a.out_cols, a.cols, l.x.rows.tokens};
  l.few = a.rows <= 16;
  if (!l.few) {
    l.q.plan = plan_for(l.q, a.out.dtype == AS_DTYPE_F32, h, h->sms);
    l.few = a.rows <= 256 && few_of((int)a.rows, (int)a.out_cols, (int)a.cols, h->sms).ns < l.q.plan.ns + 4500.;
  }
  if (l.few && aligned(a.x.data, 16) && ((a.x.stride_batch | a.x.stride_head | a.x.stride_token) & 7) == 0 && (a.x.head_dim == a.cols || a.x.head_dim % 8 == 0)) l.x = Operand{a.x, false, a.x};
  l.bytes = copy_bytes(l.x, a.rows) + copy_bytes(l.w, a.out_cols);
  if (!l.few) l.bytes += part_bytes(l.q);
  return l;
}
bool workspace_ok(const void* p, uint64_t has, uint64_t need) { return need == 0 || (p != nullptr && aligned(p, 256) && has >= need); }

}  // namespace

cudaError_t as_linear_init() {
  cudaError_t e = cudaSuccess;
  auto opt = [&](auto kernel, int bytes) { if (e == cudaSuccess) e = as_tc::opt_in_smem(kernel, bytes); };
  auto opt_modes = [&](auto cg) {
    constexpr int CG = decltype(cg)::value;
    opt(linear_kernel<CG, false, false, PLAIN>, SMEM_MAX); opt(linear_kernel<CG, false, true, PLAIN>, SMEM_MAX); opt(linear_kernel<CG, true, true, PLAIN>, SMEM_MAX);
    opt(linear_kernel<CG, false, false, LONG_SUMS>, SMEM_MAX); opt(linear_kernel<CG, false, true, LONG_SUMS>, SMEM_MAX); opt(linear_kernel<CG, true, true, LONG_SUMS>, SMEM_MAX);
  };
  opt_modes(std::integral_constant<int, 1>{});
  opt_modes(std::integral_constant<int, 2>{});
  opt(linear_kernel<1, false, false, SHARED>, SMEM_MAX); opt(linear_kernel<1, false, true, SHARED>, SMEM_MAX); opt(linear_kernel<1, true, true, SHARED>, SMEM_MAX);
  opt(linear_two_kernel, SMEM_MAX);
  opt(linear_few_kernel<1>, few_smem(1)); opt(linear_few_kernel<2>, few_smem(2));
  return e;
}

extern "C" as_status_t as_linear_workspace_bytes(as_fp8_context_t h, const as_linear_t* a, uint64_t* bytes) {
  if (bytes == nullptr) return AS_ERR_INVALID_ARG;
  if (const as_status_t s = linear_ok(h, a); s != AS_OK) return s;
  *bytes = a->rows == 0 ? 0 : plan_linear(h, *a).bytes;
  return AS_OK;
}

extern "C" as_status_t as_linear(as_fp8_context_t h, const as_linear_t* a, void* cuda_stream) {
  if (const as_status_t s = linear_ok(h, a); s != AS_OK) return s;
  if (const as_status_t s = device_of(h); s != AS_OK) return s;
  if (a->rows == 0) return AS_OK;
  LinearPlan l = plan_linear(h, *a);
  if (!workspace_ok(a->workspace, a->workspace_bytes, l.bytes)) return AS_ERR_WORKSPACE;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  uint8_t* room = static_cast<uint8_t*>(a->workspace);
  const Copy copies[2] = {{&l.x, a->rows, a->cols}, {&l.w, a->out_cols, a->cols}};
  if (run_copies(copies, room, h->sms, st) != cudaSuccess) return failed();
  Epilogue e{};
  e.out = rows_of(a->out, a->rows, a->out_cols);
  if (a->residual.data != nullptr) e.res = rows_of(a->residual, a->rows, a->out_cols);
  if (a->pre.data != nullptr) e.pre = rows_of(a->pre, a->rows, a->out_cols);
  e.bias = a->bias; e.gate = a->gate;
  e.gate_stride = a->gate_stride;
  e.gate_rows = a->gate != nullptr && a->gates > 1 ? (unsigned)(a->rows / a->gates) : 0u;
  e.N = (int)a->out_cols; e.act = a->activation;
  e.out_f32 = a->out.dtype == AS_DTYPE_F32; e.res_f32 = a->residual.dtype == AS_DTYPE_F32; e.bias_f32 = a->bias_dtype == AS_DTYPE_F32; e.gate_f32 = a->gate_dtype == AS_DTYPE_F32;
  e.vec = a->out_cols % 4 == 0 && vec4(a->out) && vec4(a->residual) && vec4(a->pre) &&
          (a->gate == nullptr || (aligned(a->gate, e.gate_f32 ? 16 : 8) && (a->gates == 1 || a->gate_stride % 4 == 0)));
  if (l.few) {
    FewParams p{};
    p.e = e;
    p.x = rows_of(l.x.rows, a->rows, a->cols);
    p.w = static_cast<const bf*>(l.w.rows.data); p.w_pitch = l.w.rows.stride_token;
    p.M = (int)a->rows; p.K = (int)a->cols;
    const Few few = few_of(p.M, e.N, p.K, h->sms);
    p.split = few.split;
    p.units = ((e.N + FEW_ROWS_W - 1) / FEW_ROWS_W + FEW_WARPS / p.split - 1) / (FEW_WARPS / p.split);
    const dim3 grid((unsigned)std::min(p.units, std::max(1, h->sms / few.mt)), (unsigned)few.mt), block(FEW_WARPS * 32);
    const cudaError_t err = a->rows <= 8 ? as_launch_dependent(linear_few_kernel<1>, grid, block, few_smem(1), st, p) : as_launch_dependent(linear_few_kernel<2>, grid, block, few_smem(2), st, p);
    return err == cudaSuccess ? AS_OK : failed();
  }
  l.q.a = l.x.rows; l.q.b = l.w.rows;
  return run_product(h, l.q, e, a->out, a->pre, a->residual, room, st) == cudaSuccess ? AS_OK : failed();
}

namespace {

struct BackPlan {
  Operand x, w, dy;
  bool two;                                  // both products in one launch
  bool dz, sums, direct;                     // dz is computed (else dy is the operand as it lies); sums are taken, in one step
  long long pitch;
  int runs;
  Product dx, dw;
  uint64_t bytes;
};

as_status_t back_ok(as_fp8_context_t h, const as_linear_backward_t* a) {
  if (h == nullptr || a == nullptr || a->struct_size != sizeof(as_linear_backward_t) || !sizes_ok(a->rows, a->cols, a->out_cols) || !act_ok(a->activation)) return AS_ERR_INVALID_ARG;
  if (!rows_ok(a->dy, a->rows, a->out_cols)) return AS_ERR_INVALID_ARG;
  const bool dx = a->dx.data != nullptr, dw = a->dw.data != nullptr;
  if (dx && (!rows_ok(a->w, a->out_cols, a->cols) || a->w.dtype != AS_DTYPE_BF16 || a->w.head_dim != a->cols || a->w.tokens != a->out_cols)) return AS_ERR_INVALID_ARG;
  if (dx && (!rows_ok(a->dx, a->rows, a->cols) || a->dx.dtype != AS_DTYPE_BF16 || !apart(a->dx, a->rows, a->cols))) return AS_ERR_INVALID_ARG;
  if (dw && (!rows_ok(a->x, a->rows, a->cols) || a->x.dtype != AS_DTYPE_BF16)) return AS_ERR_INVALID_ARG;
  if (dw && (!rows_ok(a->dw, a->out_cols, a->cols) || a->dw.dtype != AS_DTYPE_BF16 || a->dw.head_dim != a->cols || a->dw.tokens != a->out_cols || !apart(a->dw, a->out_cols, a->cols)))
    return AS_ERR_INVALID_ARG;
  if (a->rows > 0) {                         // results over none of the inputs, nor over each other
    const void* to[] = {a->dx.data, a->dw.data, a->dbias, a->dgate};
    for (int i = 0; i < 4; ++i) {
      if (to[i] == nullptr) continue;
      for (const void* in : {(const void*)a->dy.data, (const void*)a->x.data, (const void*)a->w.data, (const void*)a->pre.data, a->gate})
        if (to[i] == in) return AS_ERR_INVALID_ARG;
      for (int j = 0; j < i; ++j)
        if (to[i] == to[j]) return AS_ERR_INVALID_ARG;
    }
  }
  const bool pre = a->pre.data != nullptr;
  if (pre && (!rows_ok(a->pre, a->rows, a->out_cols) || a->pre.dtype != AS_DTYPE_BF16)) return AS_ERR_INVALID_ARG;
  if (!pre && (a->activation != AS_ACT_NONE || a->dgate != nullptr)) return AS_ERR_INVALID_ARG;
  if (!vector_ok(a->dbias, a->bias_dtype) || !vector_ok(a->dgate, a->gate_dtype) || (a->dgate != nullptr && a->gate == nullptr)) return AS_ERR_INVALID_ARG;
  if (!gate_ok(a->gate, a->gate_dtype, a->gates, a->gate_stride, a->rows, a->out_cols)) return AS_ERR_INVALID_ARG;
  if (!units_fit(a->rows, a->cols) || !units_fit(a->out_cols, a->cols) || !heads_fit(a->dy, a->out_cols) || !heads_fit(a->pre, a->out_cols) || (dw && !heads_fit(a->x, a->cols)) || !heads_fit(a->dx, a->cols)) return AS_ERR_UNSUPPORTED;
  return AS_OK;
}

// Runs of the rows of a gate: `at_once` CTAs run at a time, `each` is how many a run has; a CTA takes its rows and, to start and to end, about as long as 32 more.
int runs_of(long long each, long long rows, long long at_once) {
  int best = 1;
  double least = 1e300;
  for (long long runs = 1; runs <= std::max(1ll, rows / 16) && (runs - 1) * each < 4 * at_once; ++runs) {
    const double t = (double)((each * runs + at_once - 1) / at_once) * ((double)rows / runs + 32.);
    if (t < least) { least = t; best = (int)runs; }
  }
  return best;
}
BackPlan plan_back(as_fp8_context_t h, const as_linear_backward_t& a) {
  BackPlan b{};
  const bool dx = a.dx.data != nullptr, dw = a.dw.data != nullptr;
  b.sums = a.dbias != nullptr || a.dgate != nullptr;
  b.dy = operand_of(a.dy, a.rows, a.out_cols);
  b.x = dw ? operand_of(a.x, a.rows, a.cols) : Operand{};
  b.w = dx ? operand_of(a.w, a.out_cols, a.cols) : Operand{};
  // entries of x and of dy that differ: dy goes through dz
  b.dz = (dx || dw) && (a.activation != AS_ACT_NONE || a.gate != nullptr || b.dy.copy || (dw && b.dy.rows.tokens != a.rows && b.x.rows.tokens != b.dy.rows.tokens));
  b.pitch = pitch_of(a.out_cols);
  const long long gates = a.gate != nullptr ? a.gates : 1, across = (a.out_cols + DZ_COLS - 1) / DZ_COLS, rows_gate = a.rows / gates;
  // up to 64 rows are one run, which needs no second step
  b.runs = rows_gate <= 64 && gates == 1 ? 1 : runs_of(across * gates, rows_gate, 3ll * h->sms);
  if (b.dz) b.bytes += up256((uint64_t)a.rows * (uint64_t)b.pitch * 2);
  b.direct = gates * b.runs == 1;
  if (a.dbias != nullptr && !b.direct) b.bytes += up256((uint64_t)gates * b.runs * a.out_cols * 4);
  if (a.dgate != nullptr && !b.direct) b.bytes += up256((uint64_t)gates * b.runs * a.out_cols * 4);
  b.bytes += copy_bytes(b.x, a.rows) + copy_bytes(b.w, a.out_cols);
  const as_rows_t dz = b.dz ? plain_rows(nullptr, a.rows, a.out_cols, b.pitch) : b.dy.rows;
  if (dx) {
    b.dx = Product{dz, b.w.rows, false, true, a.rows, a.cols, a.out_cols, dz.tokens};
    b.dx.plan = plan_for(b.dx, false, h, h->sms);
  }
  if (dw) {
    const long long T = std::min(dz.tokens, b.x.rows.tokens);
    b.dw = Product{dz, b.x.rows, true, true, a.out_cols, a.cols, a.rows, T};
    b.dw.plan = plan_for(b.dw, false, h, h->sms);
  }
  if (dx && dw) {                            // at once, by half of the SMs each, where that is the sooner: a launch of its own is 4.5 us beside what the plans count
    const Plan x = plan_for(b.dx, false, h, h->sms / 2, false), w = plan_for(b.dw, false, h, h->sms / 2, false);
    b.two = std::max(x.ns, w.ns) < b.dx.plan.ns + b.dw.plan.ns + 4500. && !long_sums(b.dx, x, false) && !long_sums(b.dw, w, false);
    if (b.two) { b.dx.plan = x; b.dw.plan = w; }
  }
  const uint64_t of_dx = dx ? part_bytes(b.dx) : 0, of_dw = dw ? part_bytes(b.dw) : 0;
  b.bytes += b.two ? of_dx + of_dw : std::max(of_dx, of_dw);
  return b;
}

as_status_t zero(void* p, long long n, int dtype, cudaStream_t st) {
  if (p == nullptr) return AS_OK;
  return cudaMemsetAsync(p, 0, (size_t)n * (dtype == AS_DTYPE_BF16 ? 2 : 4), st) == cudaSuccess ? AS_OK : failed();
}

}  // namespace

extern "C" as_status_t as_linear_backward_workspace_bytes(as_fp8_context_t h, const as_linear_backward_t* a, uint64_t* bytes) {
  if (bytes == nullptr) return AS_ERR_INVALID_ARG;
  if (const as_status_t s = back_ok(h, a); s != AS_OK) return s;
  *bytes = a->rows == 0 ? 0 : plan_back(h, *a).bytes;
  return AS_OK;
}

extern "C" as_status_t as_linear_backward(as_fp8_context_t h, const as_linear_backward_t* a, void* cuda_stream) {
  if (const as_status_t s = back_ok(h, a); s != AS_OK) return s;
  if (const as_status_t s = device_of(h); s != AS_OK) return s;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (a->rows == 0) {                        // sums over nothing
    as_status_t s = zero(a->dbias, a->out_cols, a->bias_dtype, st);
    if (s == AS_OK) s = zero(a->dgate, a->out_cols * a->gates, a->gate_dtype, st);
    if (s == AS_OK && a->dw.data != nullptr && cudaMemset2DAsync(a->dw.data, (size_t)std::max<int64_t>(a->dw.stride_token, a->cols) * 2, 0, (size_t)a->cols * 2, (size_t)a->out_cols, st) != cudaSuccess)
      s = failed();
    return s;
  }
  BackPlan b = plan_back(h, *a);
  if (!workspace_ok(a->workspace, a->workspace_bytes, b.bytes)) return AS_ERR_WORKSPACE;
  uint8_t* room = static_cast<uint8_t*>(a->workspace);
  const long long gates = a->gate != nullptr ? a->gates : 1;
  DzParams z{};
  z.dy = rows_of(a->dy, a->rows, a->out_cols);
  if (a->pre.data != nullptr) z.pre = rows_of(a->pre, a->rows, a->out_cols);
  z.gate = a->gate;
  z.gate_stride = a->gate_stride;
  z.pitch = b.pitch;
  z.N = (int)a->out_cols; z.act = a->activation;
  z.rows_gate = (int)(a->rows / gates); z.runs = b.runs;
  z.gate_f32 = a->gate_dtype == AS_DTYPE_F32;
  z.vec = a->out_cols % 8 == 0 && a->dy.head_dim % 8 == 0 && rows_vec16(a->dy) && (a->pre.data == nullptr || rows_vec(a->pre, 16));
  if (b.dz) { z.dz = reinterpret_cast<bf*>(room); room += up256((uint64_t)a->rows * (uint64_t)b.pitch * 2); }
  const uint64_t sum_bytes = up256((uint64_t)gates * b.runs * a->out_cols * 4);
  if (b.direct) {
    z.dbias = a->dbias; z.bias_f32 = a->bias_dtype == AS_DTYPE_F32;
    z.dgate = a->dgate;
  } else {
    if (a->dbias != nullptr) { z.part_b = reinterpret_cast<float*>(room); room += sum_bytes; }
    if (a->dgate != nullptr) { z.part_g = reinterpret_cast<float*>(room); room += sum_bytes; }
  }
  if (gates * b.runs > 65535) return AS_ERR_UNSUPPORTED;
  if (b.dz || b.sums) {
    const dim3 grid((unsigned)((a->out_cols + DZ_COLS - 1) / DZ_COLS), (unsigned)(gates * b.runs));
    if ((a->dy.dtype == AS_DTYPE_F32 ? launch_dz<float>(z, grid, st) : launch_dz<bf>(z, grid, st)) != cudaSuccess) return failed();
  }
  if (b.sums && !b.direct) {
    ColumnSumParams c{z.part_b, z.part_g, a->dbias, a->dgate, z.N, b.runs, (int)gates, a->bias_dtype == AS_DTYPE_F32, z.gate_f32};
    if (as_launch_dependent(column_sum_kernel, dim3((unsigned)((z.N + 31) / 32), (unsigned)(1 + (a->dgate != nullptr ? gates : 0))), dim3(256), 0, st, c) != cudaSuccess) return failed();
  }
  const Copy copies[2] = {{&b.x, a->rows, a->cols}, {&b.w, a->out_cols, a->cols}};
  if (run_copies(copies, room, h->sms, st) != cudaSuccess) return failed();
  const as_rows_t dz = b.dz ? plain_rows(z.dz, a->rows, a->out_cols, b.pitch) : b.dy.rows;
  Epilogue e[2]{};
  const as_rows_t to[2] = {a->dx, a->dw};
  Product q[2] = {b.dx, b.dw};
  q[0].b = b.w.rows; q[1].b = b.x.rows;
  for (int i = 0; i < 2; ++i) {
    if (to[i].data == nullptr) continue;
    q[i].a = dz;
    e[i].N = (int)a->cols; e[i].act = AS_ACT_NONE;
    e[i].out = rows_of(to[i], i == 0 ? a->rows : a->out_cols, a->cols);
    e[i].vec = a->cols % 4 == 0 && vec4(to[i]);
    if (!b.two && run_product(h, q[i], e[i], to[i], as_rows_t{}, as_rows_t{}, room, st) != cudaSuccess) return failed();
  }
  if (b.two) {
    void* const part[2] = {room, room + part_bytes(q[0])};
    if (run_two(h, q, e, to, part, st) != cudaSuccess) return failed();
  }
  return AS_OK;
}
