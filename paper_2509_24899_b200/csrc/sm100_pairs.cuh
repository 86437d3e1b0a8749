// Instructions of CTA pairs (CG == 2; CG == 1: of a single CTA), which the products share: tensor memory, copies told to the leading CTA, arrivals across the pair.
#pragma once

#include "sm100_ptx.cuh"

namespace sm100 {

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

// A position in a ring of barriers: the slot, and the parity of the turn.
struct Ring {
  int slot = 0;
  uint32_t turn = 0;
  AS_DEV void next(int n) { if (++slot == n) { slot = 0; turn ^= 1u; } }
};

}  // namespace sm100
