// Accesses to another CTA of the cluster by the low-precision and block-attention kernels.  A
// kernel may use these only between two cluster barriers: the peer has to have started, and must
// not have left.
#pragma once

#include "common.cuh"

namespace bag {

BAG_DEV void peer_store4(uint32_t addr, float a, float b, float c, float d) { st_cluster4(addr, a, b, c, d); }
BAG_DEV void peer_store2(uint32_t addr, float a, float b) { st_cluster2(addr, a, b); }
BAG_DEV void peer_store1(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
BAG_DEV void peer_arrive(uint32_t mbar_cluster) { mbar_arrive_remote(mbar_cluster); }
// The same where nothing in memory is handed over (a thread tells that it has read its tensor
// memory): without release semantics, whose wait for the thread's earlier stores cost about 700
// cycles between two tiles of the 8-bit product.
BAG_DEV void peer_signal(uint32_t mbar_cluster) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(mbar_cluster) : "memory");
}
BAG_DEV void pair_load_2d(void* smem_dst, const CUtensorMap* map, int x, int y, uint32_t mbar_cluster) {
  tma_load_2d_pair(smem_dst, map, x, y, mbar_cluster);
}
BAG_DEV void pair_commit(uint64_t* bar, uint16_t mask) { mma_commit_pair(bar, mask); }

// mbar_wait_warp for a barrier that the peer arrives on after writing its own shared memory: the
// wait acquires at the cluster's scope.
BAG_DEV bool try_wait_cluster(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
BAG_DEV bool wait_warp_cluster(uint64_t* bar, uint32_t parity, volatile int* abort) {
  return mbar_wait_warp(bar, parity, abort) && __all_sync(0xffffffffu, try_wait_cluster(bar, parity));
}

}  // namespace bag
