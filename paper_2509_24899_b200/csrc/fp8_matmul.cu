// out = a w^T + bias of two matrices in 8-bit form, on the tensor cores' block-scaled kind: an MMA takes 32 columns of 8-bit values from shared memory and the
// power-of-two scales of their rows from tensor memory, and adds their product in fp32 to its accumulator there.
//
// A pair of CTAs (cta_group::2) computes a tile of 256 rows of a and BN rows of w: each holds 128 rows of a, half of the rows of w and the tile's 128 rows
// of results, so that an operand byte in shared memory is used 2 * BN or 512 times.  The grid is persistent, one CTA per SM; a tile's results are read out
// while the next one is computed, from the other of two accumulators.
//
//   warp 0       copies of a and w (TMA, 128 columns a stage, 128-byte swizzle), told by the leading CTA's barrier
//   warp 1       the MMAs (leading CTA only): four of 32 columns a stage, which share the byte of their scale words that the stage's block of 128 columns has
//   warp 2       allocates tensor memory
//   warps 4-7    scales: the words of 512 columns (one for each of the CTA's rows of a, one for each of the tile's rows of w) from global memory into tensor memory,
//                the same for each of the four quarters of the lanes, a ring of four
//   warps 8-15   results: tensor memory -> registers, bias, bf16, a strip of shared memory per warp, from where TMA takes it (or the warp itself does, in
//                layouts that TMA has no boxes for)
//
// Few tiles with long columns: a cluster of single CTAs shares a tile's columns (PARTS).  Few rows of a: few_rows_kernel, further down.
#include <algorithm>
#include <mutex>
#include <new>

#include "fp8_common.cuh"
#include "fp8_maps.h"
#include "tensor_common.cuh"

namespace {

using namespace as_fp8;
using namespace sm100;

constexpr int MM_THREADS = 512;
constexpr int BM = 128;                     // rows of a per CTA
constexpr int BK = 128;                     // columns of a stage, one scale
constexpr int MAX_BN = 224;                 // two accumulators of it, and the scales, fill the 512 columns of tensor memory; tiles are multiples of 32 wide
constexpr int MAX_STAGES = 10;
constexpr int SF_SLOTS = 4;
constexpr int SMEM_MAX = 227 * 1024;

// tensor memory: accumulators at 0 and 256, scale slots (words of a: 4 columns, of w: 8) two behind each
AS_DEV constexpr uint32_t sf_col(int slot) { return (slot < 2 ? 224u : 448u) + 16u * (uint32_t)slot; }

enum { B_FULL = 0, B_EMPTY = B_FULL + MAX_STAGES, B_SFULL = B_EMPTY + MAX_STAGES, B_SEMPTY = B_SFULL + SF_SLOTS, B_AFULL = B_SEMPTY + SF_SLOTS,
       B_AEMPTY = B_AFULL + 2, B_COUNT = B_AEMPTY + 2 };
// shared memory: barriers, tensor-memory address, abort flag; for each of the eight result warps a strip of 32 rows x 32 columns of results, and its biases; then the
// stages.  (Strips twice as large cost a stage, and the products 3 %.)
constexpr int STRIP = 32 * 64;
constexpr int STRIPS_OFF = 1024;
constexpr int BIAS_OFF = STRIPS_OFF + 8 * STRIP;
constexpr int STAGES_OFF = BIAS_OFF + 8 * 128;
static_assert(B_COUNT * 8 + 8 <= STRIPS_OFF && STAGES_OFF % 1024 == 0, "");
// Byte of 16-byte chunk `ch` of a strip's row: the 64-byte swizzle.
AS_DEV uint32_t swz64(int row, int ch) { return (uint32_t)(row * 64 + ((ch ^ (row >> 1 & 3)) << 4)); }

struct MMParams {
  const uint8_t *sa, *sw;
  const __nv_bfloat16* bias;
  Rows out;
  uint32_t* status;
  long long sa_rows, sw_rows;
  int M, N, kb;                             // kb: blocks of 128 columns
  int bn, stages, nt;
  int sharers;                              // CTAs of a cluster that share a tile's columns of a and w (1: none)
  long long tiles;
  bool vec, copies;                         // results move 16 bytes at a time, or in boxes of 32 rows x 32 columns by TMA
};

// ---------------------------------------------------------------- instructions of CTA pairs and of the block-scaled kind
template <int CG>
AS_DEV void alloc_tmem(uint32_t slot) {
  if constexpr (CG == 1) { tmem_alloc(slot, 512); tmem_relinquish(); }
  else asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;\n\ttcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::"r"(slot) : "memory");
}
template <int CG>
AS_DEV void free_tmem(uint32_t at) {
  if constexpr (CG == 1) tmem_dealloc(at, 512);
  else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(at) : "memory");
}
// Copy of a box; a pair's copies are told to the leading CTA's barrier, each lands in its own CTA's shared memory.
template <int CG>
AS_DEV void load_box(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y) {
  if constexpr (CG == 1)
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y) : "memory");
}
// Copy of a strip of results out: column of the head, token, head, batch entry.
AS_DEV void store_box(const CUtensorMap* m, uint32_t src, int x, int t, int h, int b) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(src), "r"(x), "r"(t), "r"(h), "r"(b) : "memory");
}
// One arrival at `bar`, of both CTAs of a pair, when the MMAs issued so far have completed.
template <int CG>
AS_DEV void commit(uint32_t bar) {
  if constexpr (CG == 1) tc_commit(bar);
  else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
template <int CG>
AS_DEV void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  if constexpr (CG == 1)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// Instruction descriptor of the kind: e4m3 operands (format 0), both K-major, scales of type ue8m0; the byte of the scale words at 4 (w) and 29 (a).
AS_DEV constexpr uint32_t scaled_idesc(int M, int N) { return (uint32_t)(N >> 3) << 17 | 1u << 23 | (uint32_t)(M >> 7) << 27; }
AS_DEV constexpr uint32_t scale_byte_of(int k) { return (uint32_t)k << 4 | (uint32_t)k << 29; }

AS_DEV uint32_t cta_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
// The address of the leading CTA's copy of a shared-memory word, for arrivals and copies across the pair.
AS_DEV uint32_t leaders(uint32_t addr) { uint32_t r; asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr)); return r; }
// Arrives at the leading CTA's barrier behind this warp's accesses to tensor memory, which tcgen05.wait has seen to the end and tcgen05.fence orders: nothing else is
// handed over, so nothing is released (a release to the cluster waits for the warp's stores to global memory, and an acquire of it by the warp that issues the MMAs took 700 clk
// each time: 36 % of the products' time).
template <int CG>
AS_DEV void arrive_leader(uint32_t bar) {
  if constexpr (CG == 1) mbar_arrive(bar);
  else asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(leaders(bar)) : "memory");
}
AS_DEV void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
AS_DEV void tmem_st4(uint32_t at, const uint32_t (&r)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
AS_DEV void tmem_st8(uint32_t at, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}

// A position in a ring of barriers: the slot, and the parity of the turn.
struct Ring {
  int slot = 0;
  uint32_t turn = 0;
  AS_DEV void next(int n) { if (++slot == n) { slot = 0; turn ^= 1u; } }
};

template <int CG>
struct Ctx {
  uint32_t sbase, tmem;
  WaitCtx wc;
  uint32_t rank;                             // of the CTA in its pair
  long long unit, units;                     // this pair (CTA), all of them: tiles unit, unit + units, ...
  int kb0, kb1;                              // its blocks of 128 columns; kb0 is a multiple of 4
  AS_DEV uint32_t bar(int i) const { return sbase + 8 * i; }
  AS_DEV bool wait(int i, uint32_t parity) const { return mbar_wait(bar(i), parity, wc); }
};

// ---------------------------------------------------------------- roles
template <int CG>
AS_DEV void mm_copies(const MMParams& p, const Ctx<CG>& c, const CUtensorMap* ma, const CUtensorMap* mw) {
  const int rows_w = p.bn / CG;
  const uint32_t stage_bytes = (uint32_t)(BM + rows_w) * BK;
  Ring r;
  for (long long t = c.unit; t < p.tiles; t += c.units) {
    const int m0 = (int)(t / p.nt) * (BM * CG) + (int)c.rank * BM, n0 = (int)(t % p.nt) * p.bn + (int)c.rank * rows_w;
    for (int k = c.kb0; k < c.kb1; ++k) {
      if (!c.wait(B_EMPTY + r.slot, r.turn ^ 1u)) goto out;
      const uint32_t at = c.sbase + STAGES_OFF + (uint32_t)r.slot * stage_bytes;
      if (c.rank == 0) mbar_expect_tx(c.bar(B_FULL + r.slot), stage_bytes * CG);
      const uint32_t bar = CG == 1 ? c.bar(B_FULL + r.slot) : leaders(c.bar(B_FULL + r.slot));
      load_box<CG>(at, ma, bar, k * BK, m0);
      load_box<CG>(at + BM * BK, mw, bar, k * BK, n0);
      r.next(p.stages);
    }
  }
out:
  // Every copy has landed, and every MMA has read its operands, before the CTA may end: the last turn of each stage has been given back (a stage
  // that was never used passes at once).
  for (int s = 0; s < p.stages; ++s) {
    if (!c.wait(B_EMPTY + r.slot, r.turn ^ 1u)) break;
    r.next(p.stages);
  }
}

// One lane walks the loop.
template <int CG>
AS_DEV void mm_issue(const MMParams& p, const Ctx<CG>& c) {
  const uint32_t stage_bytes = (uint32_t)(BM + p.bn / CG) * BK;
  const uint32_t idesc0 = scaled_idesc(BM * CG, p.bn);
  Ring r, sf;
  uint32_t buf = 0, turn = 0;
  for (long long t = c.unit; t < p.tiles; t += c.units) {
    if (!c.wait(B_AEMPTY + buf, turn ^ 1u)) return;
    const uint32_t d = c.tmem + buf * 256u;
    for (int k = c.kb0; k < c.kb1; ++k) {
      if (k % 4 == 0)
        if (!c.wait(B_SFULL + sf.slot, sf.turn)) return;
      if (!c.wait(B_FULL + r.slot, r.turn)) return;
      tc_fence_after();
      const uint32_t at = c.sbase + STAGES_OFF + (uint32_t)r.slot * stage_bytes;
      const uint64_t da = make_sdesc(at, 16, 1024), db = make_sdesc(at + BM * BK, 16, 1024);
      const uint32_t idesc = idesc0 | scale_byte_of(k % 4), s = c.tmem + sf_col(sf.slot);
#pragma unroll
      for (int i = 0; i < 4; ++i) mma_scaled<CG>(d, da + 2 * i, db + 2 * i, idesc, s, s + 8, k > c.kb0 || i > 0 ? 1u : 0u);
      commit<CG>(c.bar(B_EMPTY + r.slot));
      r.next(p.stages);
      if (k % 4 == 3 || k == c.kb1 - 1) {
        commit<CG>(c.bar(B_SEMPTY + sf.slot));
        sf.next(SF_SLOTS);
      }
    }
    commit<CG>(c.bar(B_AFULL + buf));
    buf ^= 1u;
    if (buf == 0) turn ^= 1u;
  }
}

// The words of the next 512 columns are on their way from global memory while those of the ones before wait for their slot.
template <int CG>
AS_DEV void mm_scales(const MMParams& p, const Ctx<CG>& c, int lane, int quarter) {
  const uint32_t lanes = (uint32_t)quarter * 32u << 16;
  const int g0 = c.kb0 / 4, groups = (c.kb1 + 3) / 4;
  const uint32_t ones = 0x7f7f7f7fu;         // rows that are not there
  uint32_t a[4], w[8];
  auto fetch = [&](long long t, int g) {
    if (t >= p.tiles) return;
    const int m0 = (int)(t / p.nt) * (BM * CG) + (int)c.rank * BM + lane, n0 = (int)(t % p.nt) * p.bn + lane;
    const uint32_t* ga = reinterpret_cast<const uint32_t*>(p.sa) + (long long)g * p.sa_rows;
    const uint32_t* gw = reinterpret_cast<const uint32_t*>(p.sw) + (long long)g * p.sw_rows;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = m0 + 32 * j < p.M ? __ldg(ga + m0 + 32 * j) : ones;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = 32 * j < p.bn && n0 + 32 * j < p.N ? __ldg(gw + n0 + 32 * j) : ones;
  };
  Ring sf;
  long long t = c.unit;
  int g = g0;
  fetch(t, g);
  while (t < p.tiles) {
    uint32_t a0[4], w0[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) a0[j] = a[j];
#pragma unroll
    for (int j = 0; j < 8; ++j) w0[j] = w[j];
    if (++g == groups) { g = g0; t += c.units; }
    fetch(t, g);
    const bool ok = c.wait(B_SEMPTY + sf.slot, sf.turn ^ 1u);
    if (!__all_sync(0xffffffffu, ok)) return;
    tc_fence_after();
    const uint32_t at = c.tmem + lanes + sf_col(sf.slot);
    tmem_st4(at, a0);
    tmem_st8(at + 8, w0);
    tmem_st_wait();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) arrive_leader<CG>(c.bar(B_SFULL + sf.slot));
    sf.next(SF_SLOTS);
  }
}

// Results of a tile: this warp's 32 rows, every second 32 columns, through a strip of shared memory.
template <int CG>
AS_DEV void mm_results(const MMParams& p, const Ctx<CG>& c, const CUtensorMap* mo, int lane, int warp) {
  const int quarter = warp & 3, half = warp >> 2;
  const uint32_t lanes = (uint32_t)quarter * 32u << 16;
  const uint32_t strip = c.sbase + STRIPS_OFF + (uint32_t)warp * STRIP, sbias = c.sbase + BIAS_OFF + (uint32_t)warp * 128;
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out.data);
  uint32_t buf = 0, turn = 0;
  for (long long t = c.unit; t < p.tiles; t += c.units) {
    const int m0 = (int)(t / p.nt) * (BM * CG) + (int)c.rank * BM + quarter * 32, n0 = (int)(t % p.nt) * p.bn;
    const long long my_row = m0 + lane < p.M ? p.out.row((unsigned)(m0 + lane)) : 0;
    // a strip's store is one copy where its rows belong to one batch entry
    const unsigned batch = p.out.batched ? (unsigned)m0 / p.out.tokens : 0u, token = (unsigned)m0 - batch * p.out.tokens;
    const bool whole = p.copies && (int)token + min(32, p.M - m0) <= (int)p.out.tokens;
    // biases of this lane's column in each strip, while the products run
    float bias[(MAX_BN / 32 + 1) / 2];
#pragma unroll
    for (int j = 0; j < (MAX_BN / 32 + 1) / 2; ++j) {
      const int n = n0 + 64 * j + 32 * half + lane;
      bias[j] = p.bias != nullptr && n < p.N ? __bfloat162float(p.bias[n]) : 0.f;
    }
    if (!mbar_wait_warp(c.bar(B_AFULL + buf), turn, c.wc)) break;
    tc_fence_after();
    if (32 * half >= p.bn) {
      __syncwarp();
      if (lane == 0) arrive_leader<CG>(c.bar(B_AEMPTY + buf));
    }
#pragma unroll
    for (int j = 0; j < (MAX_BN / 32 + 1) / 2; ++j) {
      const int c0 = 64 * j + 32 * half, n1 = n0 + c0;
      if (c0 >= p.bn) break;
      uint32_t x[32];
      tmem_ld32(c.tmem + lanes + buf * 256u + c0, x);
      if (lane == 0) tma_store_wait_read();   // the copy of the strip before has read it
      if (p.bias != nullptr) asm volatile("st.shared.f32 [%0], %1;" ::"r"(sbias + lane * 4), "f"(bias[j]) : "memory");
      __syncwarp();
      tmem_ld_wait(x);
      if (c0 + 64 >= p.bn) {                  // this warp has read its part of the accumulator
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_leader<CG>(c.bar(B_AEMPTY + buf));
      }
      if (p.bias != nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float4 b;
          asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(b.x), "=f"(b.y), "=f"(b.z), "=f"(b.w) : "r"(sbias + i * 16) : "memory");
          x[4 * i] = __float_as_uint(__uint_as_float(x[4 * i]) + b.x); x[4 * i + 1] = __float_as_uint(__uint_as_float(x[4 * i + 1]) + b.y);
          x[4 * i + 2] = __float_as_uint(__uint_as_float(x[4 * i + 2]) + b.z); x[4 * i + 3] = __float_as_uint(__uint_as_float(x[4 * i + 3]) + b.w);
        }
      }
      // this lane's row of 64 bytes into the strip, with the 64-byte swizzle
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = pack_bf16(__uint_as_float(x[8 * i + 2 * k]), __uint_as_float(x[8 * i + 2 * k + 1]));
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(strip + swz64(lane, i)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
      }
      if (whole) {
        fence_proxy_async();
        __syncwarp();
        if (lane == 0 && m0 < p.M && n1 < p.N) {
          const unsigned head = p.out.hd == p.N ? 0u : (unsigned)n1 / (unsigned)p.out.hd;
          store_box(mo, strip, n1 - (int)head * p.out.hd, (int)token, (int)head, (int)batch);
          tma_store_commit();
        }
      } else if (p.vec) {
        __syncwarp();
        // four lanes a row, 16 bytes a lane
        const int ch = lane & 3, n = n1 + ch * 8;
        const bool there = n < p.N;
        __nv_bfloat16* at = out + (there ? p.out.col((unsigned)n) : 0);
        uint4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i].x), "=r"(w[i].y), "=r"(w[i].z), "=r"(w[i].w) : "r"(strip + swz64(i * 8 + lane / 4, ch)) : "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = i * 8 + lane / 4;
          const long long row = __shfl_sync(0xffffffffu, my_row, r);
          if (there && m0 + r < p.M) *reinterpret_cast<uint4*>(at + row) = w[i];
        }
        __syncwarp();
      } else {
        __syncwarp();
        const bool there = n1 + lane < p.N;
        __nv_bfloat16* at = out + (there ? p.out.col((unsigned)(n1 + lane)) : 0);
#pragma unroll 8
        for (int r = 0; r < 32; ++r) {
          const long long row = __shfl_sync(0xffffffffu, my_row, r);
          uint16_t v;
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(strip + swz64(r, lane / 8) + (lane % 8) * 2) : "memory");
          if (there && m0 + r < p.M) *reinterpret_cast<uint16_t*>(at + row) = v;
        }
        __syncwarp();
      }
    }
    buf ^= 1u;
    if (buf == 0) turn ^= 1u;
  }
  if (lane == 0) tma_store_wait_read();       // (the writes land by the end of the kernel)
}

// A tile whose columns of a and w are shared by a cluster of CTAs: each leaves its sums in its shared memory, in fp32 and where the stages were, and adds up a part of the tile's 8-column
// pieces over all of them, in the order of their ranks.
constexpr int PART_PAD = 16;                  // bytes behind a row of sums, so that rows begin in other banks
AS_DEV void part_leave(const MMParams& p, const Ctx<1>& c, int lane, int warp) {
  const int quarter = warp & 3, half = warp >> 2;
  if (!mbar_wait_warp(c.bar(B_AFULL), 0, c.wc)) return;
  tc_fence_after();
  const uint32_t row = c.sbase + STAGES_OFF + (uint32_t)(quarter * 32 + lane) * (uint32_t)(p.bn * 4 + PART_PAD);
  for (int c0 = 32 * half; c0 < p.bn; c0 += 64) {
    uint32_t x[32];
    tmem_ld32(c.tmem + ((uint32_t)quarter * 32u << 16) + c0, x);
    tmem_ld_wait(x);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row + c0 * 4 + i * 16), "r"(x[4 * i]), "r"(x[4 * i + 1]), "r"(x[4 * i + 2]), "r"(x[4 * i + 3]) : "memory");
  }
}
AS_DEV void part_add(const MMParams& p, const Ctx<1>& c, int rank) {
  const int m0 = (int)(c.unit / p.nt) * BM, n0 = (int)(c.unit % p.nt) * p.bn, across = p.bn / 8, pieces = BM * across;
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out.data);
  for (int e = pieces * rank / p.sharers + threadIdx.x; e < pieces * (rank + 1) / p.sharers; e += MM_THREADS) {
    const int r = e / across, n = n0 + e % across * 8, m = m0 + r;
    if (m >= p.M || n >= p.N) continue;
    const uint32_t at = c.sbase + STAGES_OFF + (uint32_t)r * (uint32_t)(p.bn * 4 + PART_PAD) + (uint32_t)(e % across) * 32u;
    float f[8] = {};
    for (int q = 0; q < p.sharers; ++q) {
      uint32_t from;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(at), "r"(q));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float4 v;
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(from + 16 * h) : "memory");
        f[4 * h] += v.x; f[4 * h + 1] += v.y; f[4 * h + 2] += v.z; f[4 * h + 3] += v.w;
      }
    }
    if (p.bias != nullptr) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (n + i < p.N) f[i] += __bfloat162float(p.bias[n + i]);
    }
    const long long row = p.out.row((unsigned)m);
    if (p.vec) {
      *reinterpret_cast<uint4*>(out + row + p.out.col((unsigned)n)) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (n + i < p.N) out[row + p.out.col((unsigned)(n + i))] = __float2bfloat16_rn(f[i]);
    }
  }
}

// PARTS: p.sharers CTAs share a tile, one tile each cluster (CG == 1).
template <int CG, bool PARTS>
__global__ void __launch_bounds__(MM_THREADS, 1)
matmul_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mw, const __grid_constant__ CUtensorMap mo,
              const __grid_constant__ MMParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);      // the same in both CTAs of a pair
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + 8 * B_COUNT);
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + 8 * B_COUNT + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t in_cluster = CG == 1 && !PARTS ? 0u : cta_rank();
  const int sharing = PARTS ? p.sharers : CG, groups = (p.kb + 3) / 4;
  Ctx<CG> c{smem_u32(smem), 0u, WaitCtx{p.status, abort_flag}, PARTS ? 0u : in_cluster, blockIdx.x / sharing, gridDim.x / sharing, 0, p.kb};
  if constexpr (PARTS) {
    c.kb0 = groups * (int)in_cluster / p.sharers * 4;
    c.kb1 = min(groups * ((int)in_cluster + 1) / p.sharers * 4, p.kb);
  }
  if (threadIdx.x == 0) {
    *abort_flag = 0u;
    for (int s = 0; s < MAX_STAGES; ++s) { mbar_init(c.bar(B_FULL + s), 1); mbar_init(c.bar(B_EMPTY + s), 1); }
    for (int s = 0; s < SF_SLOTS; ++s) { mbar_init(c.bar(B_SFULL + s), 4 * CG); mbar_init(c.bar(B_SEMPTY + s), 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(c.bar(B_AFULL + s), 1); mbar_init(c.bar(B_AEMPTY + s), 8 * CG); }
    fence_barrier_init();
    fence_proxy_async();
    tma_prefetch_desc(&ma); tma_prefetch_desc(&mw);
  }
  if (warp == 2) { alloc_tmem<CG>(smem_u32(tmem_slot)); griddep_launch(); }
  tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2) cluster_sync();       // the peer's barriers stand before anything arrives there
  tc_fence_after();
  c.tmem = *tmem_slot;
  griddep_wait();
  if (warp == 0) {
    if (elect_one()) mm_copies<CG>(p, c, &ma, &mw);
    __syncwarp();
  } else if (warp == 1) {
    if (c.rank == 0 && elect_one()) mm_issue<CG>(p, c);
    __syncwarp();
  } else if (warp >= 4 && warp < 8) {
    mm_scales<CG>(p, c, lane, warp - 4);
  } else if (warp >= 8) {
    if constexpr (PARTS) part_leave(p, c, lane, warp - 8);
    else mm_results<CG>(p, c, &mo, lane, warp - 8);
  }
  if constexpr (PARTS) {
    __syncthreads();
    cluster_sync();                            // all sums of the tile stand
    part_add(p, c, (int)in_cluster);
  }
  if (*abort_flag != 0u) {                     // a wait ran out: copies and MMAs under way get 20 us (they take two) before memory is given back
    const long long t0 = clock64();
    while (clock64() - t0 < 40000) {}
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2 || PARTS) cluster_sync();        // nothing of this CTA is reached from the others any more
  if (warp == 2) {
    tc_fence_after();
    free_tmem<CG>(c.tmem);
  }
}

// ---------------------------------------------------------------- few rows
// Few rows of a, where a tile of the pair would be empty but for some and few CTAs would walk all columns: here w is read by all SMs, into the operands of the warps' own matrix
// instructions (16 rows of w, 8 of a, 32 columns).  A CTA takes units of 16 rows of w by 8 or 16 of a; its warps take every sixteenth block of 128 columns each, with one scale for a
// row and block: four instructions into fresh sums, which are scaled and added up in fp32.  Which columns an instruction calls its k-th does not matter as long as both
// operands agree: a lane holds columns 16 q .. 16 q + 15 of each half of its rows' block, so that four lanes copy 64 bytes in a run.  The warps' sums meet in shared
// memory, in the order of the warps.
//
// What bounds it is the latency of memory, and then the number of copies: a warp's operands come by asynchronous copies into slots that it alone reads, two or three blocks ahead and
// on into the next unit, one copy for all scales of a block.  (2 rows by w of 1536 x 1536, 9216 x 1536, 1536 x 6144, 6144 x 6144: straight into registers 2.7, 5.5, 5.7, 13.2 us;
// two CTAs of 8 warps an SM 2.6, 4.5, 6.4, 12.7; one of 16 warps 2.0, 4.8, 4.0, 10.5 us (3.6 TB/s).)
constexpr int FEW_WARPS = 16, FEW_COLS = 16;
// With NT tiles of 8 rows of a: blocks of a warp under way (one CTA an SM), bytes of one: per lane 64 of w and 32 NT of a, the scale words of 16 rows of w and 8 NT of a
__host__ __device__ constexpr int few_ahead(int nt) { return nt == 1 ? 3 : 2; }
__host__ __device__ constexpr int few_slot(int nt) { return (4 + 2 * nt) * 512 + 64 + 32 * nt + (nt == 1 ? 32 : 0); }
constexpr int few_smem(int nt) { return FEW_WARPS * few_ahead(nt) * few_slot(nt); }
static_assert(few_slot(1) % 128 == 0 && few_slot(2) % 128 == 0, "");

struct FewParams {
  const uint8_t *a, *w, *sa, *sw;
  const __nv_bfloat16* bias;
  Rows out;
  long long a_pitch, w_pitch, sa_rows, sw_rows;
  int M, N, K, units, mt;                   // mt: units of a tile of w, one for each 8 NT rows of a
};

// 16 bytes, of which `bytes` come from memory and the rest are 0: of w past the first-level cache, of a, which every CTA reads, through it (past it they all
// meet at the same lines of the second one: eight times as long).
AS_DEV void few_copy_w(uint32_t dst, const void* src, int bytes) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory"); }
AS_DEV void few_copy_a(uint32_t dst, const void* src, int bytes) { asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory"); }
AS_DEV void few_copy4(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory"); }
AS_DEV void few_read(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// 2^(e - 127) of a scale byte (NaN for 255) as two factors of about half its exponent.  A block's sum is multiplied by the first factors of both matrices' scales and then by the
// second ones: as one scale after the other it would leave fp32's range where the product of both scales does not.  The halves that are rounded down take 2^-63 of w's scale
// and 2^-64 of a's, the others 2^-64 and 2^-63, so that a product of two lies between 2^-127 and 2^127 and is exact; the second is at least the first, so a sum
// between them overflows, or loses bits, only where the result does.
struct FewScale { float first, second; };
template <int OF_W> AS_DEV FewScale few_scale(uint32_t e) {
  const uint32_t h = e >> 1;
  return {__uint_as_float(e == 255u ? 0x7fc00000u : (h + 63u + OF_W) << 23), __uint_as_float((e - h + 64u - OF_W) << 23)};
}

template <int NT>
__global__ void __launch_bounds__(FEW_WARPS * 32, 1) few_rows_kernel(const __grid_constant__ FewParams p) {
  constexpr int AHEAD = few_ahead(NT), SLOT = few_slot(NT), SCALES = (4 + 2 * NT) * 512;
  griddep_launch();
  extern __shared__ __align__(16) uint8_t slots[];
  __shared__ float sums[2][FEW_WARPS][8 * NT][FEW_COLS + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane / 4, q = lane % 4;
  const int kb = (p.K + BK - 1) / BK;
  const uint32_t mine = smem_u32(slots) + (uint32_t)warp * (AHEAD * SLOT);
  griddep_wait();
  int unit = blockIdx.x, block = warp, slot = 0;                      // what is asked for next, and its first rows of w and a
  int n1 = (NT == 1 ? unit : unit / p.mt) * FEW_COLS, m1 = NT == 1 ? 0 : unit % p.mt * (8 * NT);
  auto ask = [&] {
    if (block < kb && unit < p.units) {
      const uint32_t at = mine + slot * SLOT, own = at + lane * 16;
      const int c = block * BK + q * 16, n = n1 + g, m0 = m1;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int bytes = max(0, min(16, p.K - c - 64 * i)), c1 = bytes > 0 ? c + 64 * i : 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) few_copy_w(own + (2 * h + i) * 512, p.w + (long long)min(n + 8 * h, p.N - 1) * p.w_pitch + c1, bytes);
#pragma unroll
        for (int t = 0; t < NT; ++t)        // (a row that is not there leaves its results, which are not written, to chance)
          if (m0 + 8 * t + g < p.M) few_copy_a(own + (4 + 2 * t + i) * 512, p.a + (long long)(m0 + 8 * t + g) * p.a_pitch + c1, bytes);
      }
      const uint8_t* scale = q < 2 ? p.sw + ((long long)(block / 4) * p.sw_rows + min(n + 8 * q, p.N - 1)) * 4
                                   : p.sa + ((long long)(block / 4) * p.sa_rows + min(m0 + 8 * (q - 2) + g, p.M - 1)) * 4;
      if (q < 2 + NT) few_copy4(at + SCALES + (8 * q + g) * 4, scale);
      if (++slot == AHEAD) slot = 0;
      if ((block += FEW_WARPS) >= kb) {
        block = warp;
        unit += gridDim.x;
        n1 = (NT == 1 ? unit : unit / p.mt) * FEW_COLS;
        m1 = NT == 1 ? 0 : unit % p.mt * (8 * NT);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");              // (an empty group where there is nothing left: the waits below count groups)
  };
#pragma unroll
  for (int i = 0; i < AHEAD - 1; ++i) ask();
  int take = 0, turn = 0;
  for (int u = blockIdx.x; u < p.units; u += gridDim.x, turn ^= 1) {
    float acc[NT][4] = {};
    for (int k = warp; k < kb; k += FEW_WARPS) {
      __syncwarp();                                                   // every lane has read the slot that is filled next
      ask();
      asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
      __syncwarp();                                                   // the other lanes' scales have come as well
      const uint32_t at = mine + take * SLOT, own = at + lane * 16;
      if (++take == AHEAD) take = 0;
      auto byte_of = [&](int i) {
        uint32_t e;
        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(e) : "r"(at + SCALES + i * 4 + k % 4) : "memory");
        return e;
      };
      uint32_t w[2][2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        few_read(own + i * 512, w[0][i]);
        few_read(own + (2 + i) * 512, w[1][i]);
      }
      const FewScale fw[2] = {few_scale<1>(byte_of(g)), few_scale<1>(byte_of(8 + g))};      // rows g and g + 8 of w; of a: rows 2 q and 2 q + 1 of each tile
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        uint32_t a[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) few_read(own + (4 + 2 * t + i) * 512, a[i]);
        const FewScale fa[2] = {few_scale<0>(byte_of(16 + 8 * t + 2 * q)), few_scale<0>(byte_of(17 + 8 * t + 2 * q))};
        float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                       : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                       : "r"(w[0][i / 2][2 * (i % 2)]), "r"(w[1][i / 2][2 * (i % 2)]), "r"(w[0][i / 2][2 * (i % 2) + 1]), "r"(w[1][i / 2][2 * (i % 2) + 1]),
                         "r"(a[i / 2][2 * (i % 2)]), "r"(a[i / 2][2 * (i % 2) + 1]));
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[t][j] = fmaf(d[j] * (fw[j / 2].first * fa[j % 2].first), fw[j / 2].second * fa[j % 2].second, acc[t][j]);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) sums[turn][warp][8 * t + 2 * q + j % 2][g + 8 * (j / 2)] = acc[t][j];
    __syncthreads();                                                  // (one for a unit: the next one's sums go to the other half)
    if (threadIdx.x < 8 * NT * FEW_COLS) {
      const int i0 = threadIdx.x / FEW_COLS, j = threadIdx.x % FEW_COLS, n = (NT == 1 ? u : u / p.mt) * FEW_COLS + j, m = (NT == 1 ? 0 : u % p.mt * (8 * NT)) + i0;
      if (m < p.M && n < p.N) {
        float f = 0.f;
#pragma unroll
        for (int i = 0; i < FEW_WARPS; ++i) f += sums[turn][i][i0][j];
        if (p.bias != nullptr) f += __bfloat162float(p.bias[n]);
        static_cast<__nv_bfloat16*>(p.out.data)[p.out.row((unsigned)m) + p.out.col((unsigned)n)] = __float2bfloat16_rn(f);
      }
    }
  }
}

// The shape of a tile - CTAs that share its rows or its columns, rows of w - by the time that its turns take on all SMs: turns x blocks of 128 columns x ns a block, and what the
// reading out of the last turn's results and the meeting of a pair add.  ns: measured with all SMs busy, at 7800 x 4608 x 1536 and what the largest products make of it.  What a block
// takes is its copies at every width, 64 bytes a clock into an SM (a pair halves those of w): with 192 rows of w a pair's 28672 bytes an SM are 448 clk beside 384 of MMAs, with 224
// 30720 and 480 beside 448.  At 32760 x 4608 x 1536, back to back, 192 and 224 rows take 212 and 209 us at 1.45 GHz.  The last turn counts half of what it leaves idle, as the clock
// rises meanwhile; a single turn counts whole.  Few rows go to single CTAs and narrow tiles: 512 x 1536 x 1536 takes 6.1 us with {1, 64}, 7.2 with {2, 192}.
//
// Few tiles with long columns go to clusters of CTAs that share a tile's columns, by whole groups of four blocks, as many as the device holds at once (`clusters`, by size): 2 us more
// for the meeting and the sums, and more with every CTA beyond two (128 x 1536 x 6144 14.0 us by single CTAs, 9.4 by three, 9.6 by five; 512 x 1536 x 6144 15.0, 11.5 by two, 13.2 by three;
// 300 x 512 x 4096 10.1 and 8.0; but 512 x 1536 x 1536 5.9 and 8.1, 1024 x 512 x 2048 6.5 and 7.4).
struct Tile { int cg, bn, parts; double ns; };
constexpr int MAX_PARTS = 8;
Tile tile_of(int M, int N, int kb, int sms, const int (&clusters)[MAX_PARTS + 1]) {
  static const int ns[2][7] = {{230, 250, 265, 300, 345, 385, 440}, {228, 230, 240, 262, 297, 320, 365}};
  Tile best{1, 32, 1, 1e300};
  for (int cg = 1; cg <= 2; ++cg)
    for (int i = 0; i < 7; ++i) {
      const int bn = 32 * (i + 1);
      const long long tiles = ((long long)M + BM * cg - 1) / (BM * cg) * ((N + bn - 1) / bn), units = sms / cg, whole = (tiles + units - 1) / units;
      const double turns = whole == 1 ? 1. : 0.5 * ((double)tiles / units + whole);
      const double t = turns * kb * ns[cg - 1][i] + 7. * bn + (cg == 2 ? 400. : 0.);
      if (t < best.ns) best = {cg, bn, 1, t};
      const int groups = (kb + 3) / 4;
      for (int parts = 2; cg == 1 && parts <= std::min(MAX_PARTS, groups); ++parts) {
        const double shared = 4. * ((groups + parts - 1) / parts) * ns[0][i] + 7. * bn + 2000. + 8. * std::max(bn - 64, 0) + (parts - 2) * (700. + 10. * (bn - 32));
        if (tiles <= clusters[parts] && shared < best.ns) best = {1, bn, parts, shared};
      }
    }
  return best;
}

// Whether a product goes to few_rows_kernel: up to 16 rows of a, and up to 256 where its turns - units of 16 rows of a and of w, sixteen blocks of 128 columns at a time - take
// less than the tile's: 1.5 us each, the first one 0.7, from 0.5 us less of setting up.  (us by the one and the other: 16 rows by 1536 x 1536 2.8 and 5.3, by 9216 x 1536 7.5 and 7.9,
// by 1536 x 6144 6.0 and 9.8, by 6144 x 6144 14.7 and 16.6; the exception is a wide w of short rows, 20000 x 192 10.2 and 5.6.  32 rows by 1536 x 1536 4.3 and 5.3, by 9216 x 1536
// 13.8 and 7.5; 64 rows by 512 x 1280 2.7 and 4.8, by 1536 x 1536 6.0 and 5.3; 256 rows by 128 x 2392 3.8 and 6.9.)
bool few_rows(int M, int N, int kb, int sms, const Tile& tile) {
  if (M <= 16) return true;
  if (M > 256) return false;
  const long long units = (long long)((N + FEW_COLS - 1) / FEW_COLS) * ((M + 15) / 16), turns = (units + sms - 1) / sms * ((kb + FEW_WARPS - 1) / FEW_WARPS);
  return 700. + 1500. * (double)(turns - 1) < tile.ns + 500.;
}

template <int CG, bool PARTS>
cudaError_t launch(const CUtensorMap& ma, const CUtensorMap& mw, const CUtensorMap& mo, const MMParams& p, int units, size_t smem, cudaStream_t st) {
  const int sharing = PARTS ? p.sharers : CG;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = sharing; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(units * sharing)); cfg.blockDim = dim3(MM_THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cfg.attrs = attr; cfg.numAttrs = sharing == 1 ? 1 : 2;
  return cudaLaunchKernelEx(&cfg, matmul_kernel<CG, PARTS>, ma, mw, mo, p);
}

// The status word is read and cleared in one step: a bit that a product on another stream raises stands before it or after it.
constexpr int TAKEN = 32;
__global__ void take_status_kernel(uint32_t* status) { status[TAKEN] = atomicExch(status, 0u); }

}  // namespace

struct as_fp8_context_s {
  int device = -1, sms = 0;
  int clusters[MAX_PARTS + 1] = {};          // of so many CTAs that the device holds at once
  uint32_t* status = nullptr;
  std::mutex reading;                        // of the word behind the status word, where a read leaves what it took
};

extern "C" as_status_t as_fp8_create(as_fp8_context_t* out) {
  if (out == nullptr) return AS_ERR_INVALID_ARG;
  int dev = 0, major = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return failed();
  if (major != 10) return AS_ERR_ARCH;
  if (as_tensor_init() != cudaSuccess || as_tc::opt_in_smem(matmul_kernel<1, false>, SMEM_MAX) != cudaSuccess || as_tc::opt_in_smem(matmul_kernel<2, false>, SMEM_MAX) != cudaSuccess ||
      as_tc::opt_in_smem(matmul_kernel<1, true>, SMEM_MAX) != cudaSuccess ||
      as_tc::opt_in_smem(few_rows_kernel<1>, few_smem(1)) != cudaSuccess || as_tc::opt_in_smem(few_rows_kernel<2>, few_smem(2)) != cudaSuccess)
    return failed();
  as_fp8_context_s* h = new (std::nothrow) as_fp8_context_s;
  if (h == nullptr) return AS_ERR_ALLOC;
  h->device = dev;
  h->sms = sms;
  for (int parts = 2; parts <= MAX_PARTS; ++parts) {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = parts; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)parts); cfg.blockDim = dim3(MM_THREADS); cfg.dynamicSmemBytes = SMEM_MAX;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&h->clusters[parts], matmul_kernel<1, true>, &cfg) != cudaSuccess) { delete h; return failed(); }
  }
  if (cudaMalloc(&h->status, 256) != cudaSuccess) { delete h; return failed(AS_ERR_ALLOC); }
  if (cudaMemset(h->status, 0, 256) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) { cudaFree(h->status); delete h; return failed(); }
  *out = h;
  return AS_OK;
}

extern "C" as_status_t as_fp8_destroy(as_fp8_context_t h) {
  if (h == nullptr) return AS_OK;
  cudaFree(h->status);
  delete h;
  return AS_OK;
}

extern "C" as_status_t as_fp8_last_status(as_fp8_context_t h, void* cuda_stream) {
  if (h == nullptr) return AS_ERR_INVALID_ARG;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  uint32_t word = 0;
  std::lock_guard<std::mutex> hold(h->reading);
  take_status_kernel<<<1, 1, 0, st>>>(h->status);
  if (cudaGetLastError() != cudaSuccess || cudaMemcpyAsync(&word, h->status + TAKEN, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
    return failed();
  return word == 0 ? AS_OK : AS_ERR_DEVICE_TIMEOUT;
}

extern "C" as_status_t as_fp8_debug_expire_wait(as_fp8_context_t h, int64_t limit_cycles, void* cuda_stream) {
  int dev = 0;
  if (h == nullptr || limit_cycles < 1 || limit_cycles > 100000000) return AS_ERR_INVALID_ARG;       // at most about 50 ms
  if (cudaGetDevice(&dev) != cudaSuccess) return failed();
  if (dev != h->device) return AS_ERR_INVALID_ARG;
  return as_tensor_expire_wait(h->status, limit_cycles, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? AS_OK : failed();
}

extern "C" as_status_t as_matmul_fp8(as_fp8_context_t h, const as_matmul_fp8_t* a, void* cuda_stream) {
  if (h == nullptr || a == nullptr || a->struct_size != sizeof(as_matmul_fp8_t)) return AS_ERR_INVALID_ARG;
  if (a->cols < 1 || a->cols > (1 << 20) || a->rows < 0 || a->rows > (1ll << 30) || a->out_cols < 1 || a->out_cols > (1ll << 24)) return AS_ERR_INVALID_ARG;
  if (!matrix_ok(a->a, a->rows, a->cols) || !matrix_ok(a->w, a->out_cols, a->cols) || !aligned(a->bias, 2)) return AS_ERR_INVALID_ARG;
  if (!rows_ok(a->out, a->rows, a->out_cols) || a->out.dtype != AS_DTYPE_BF16 || !apart(a->out, a->rows, a->out_cols)) return AS_ERR_INVALID_ARG;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return failed();
  if (dev != h->device) return AS_ERR_INVALID_ARG;
  const Rows out = rows_of(a->out, a->rows, a->out_cols);
  if (out.split && a->out_cols * (long long)a->out.head_dim > (1ll << 32)) return AS_ERR_UNSUPPORTED;
  if (a->rows == 0) return AS_OK;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int kb = (a->cols + BK - 1) / BK;
  const Tile tile = tile_of((int)a->rows, (int)a->out_cols, kb, h->sms, h->clusters);
  if (few_rows((int)a->rows, (int)a->out_cols, kb, h->sms, tile)) {
    FewParams p{};
    p.a = static_cast<const uint8_t*>(a->a.data); p.a_pitch = a->a.pitch;
    p.w = static_cast<const uint8_t*>(a->w.data); p.w_pitch = a->w.pitch;
    p.sa = static_cast<const uint8_t*>(a->a.scales); p.sa_rows = a->a.scale_rows;
    p.sw = static_cast<const uint8_t*>(a->w.scales); p.sw_rows = a->w.scale_rows;
    p.bias = static_cast<const __nv_bfloat16*>(a->bias);
    p.out = out;
    p.M = (int)a->rows; p.N = (int)a->out_cols; p.K = a->cols;
    p.mt = p.M <= 8 ? 1 : (p.M + 15) / 16;
    p.units = (p.N + FEW_COLS - 1) / FEW_COLS * p.mt;
    const dim3 grid((unsigned)std::min(p.units, h->sms)), block(FEW_WARPS * 32);
    const cudaError_t e = p.M <= 8 ? as_launch_dependent(few_rows_kernel<1>, grid, block, few_smem(1), st, p) : as_launch_dependent(few_rows_kernel<2>, grid, block, few_smem(2), st, p);
    return e == cudaSuccess ? AS_OK : failed();
  }
  MMParams p{};
  p.out = out;
  p.M = (int)a->rows; p.N = (int)a->out_cols; p.kb = kb;
  p.sa = static_cast<const uint8_t*>(a->a.scales); p.sa_rows = a->a.scale_rows;
  p.sw = static_cast<const uint8_t*>(a->w.scales); p.sw_rows = a->w.scale_rows;
  p.bias = static_cast<const __nv_bfloat16*>(a->bias);
  p.status = h->status;
  p.vec = rows_vec(a->out, 16);
  const int CG = tile.cg;
  p.bn = tile.bn; p.sharers = tile.parts;
  p.nt = (p.N + p.bn - 1) / p.bn;
  p.tiles = ((long long)p.M + BM * CG - 1) / (BM * CG) * p.nt;
  const int stage = (BM + p.bn / CG) * BK;
  p.stages = std::min((SMEM_MAX - 1024 - STAGES_OFF) / stage, MAX_STAGES);
  const size_t smem = 1024 + STAGES_OFF + (size_t)p.stages * stage;
  CUtensorMap ma, mw, mo{};
  // results leave by TMA where 32 columns are of one head (a map that the driver does not take leaves that to the warps)
  p.copies = p.vec && (a->out.head_dim == p.N || a->out.head_dim % 32 == 0) && as_tc::make_map_rows(&mo, a->out, p.M, p.N, 32);
  if (!as_tc::make_map_bytes(&ma, a->a.data, a->cols, p.M, a->a.pitch, BM) || !as_tc::make_map_bytes(&mw, a->w.data, a->cols, p.N, a->w.pitch, p.bn / CG)) return failed();
  const int units = (int)std::min<long long>(p.tiles, h->sms / CG);
  const cudaError_t e = tile.parts > 1 ? launch<1, true>(ma, mw, mo, p, (int)p.tiles, smem, st)
                                       : CG == 2 ? launch<2, false>(ma, mw, mo, p, units, smem, st) : launch<1, false>(ma, mw, mo, p, units, smem, st);
  return e == cudaSuccess ? AS_OK : failed();
}
