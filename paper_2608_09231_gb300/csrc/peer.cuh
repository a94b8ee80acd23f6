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

}  // namespace bag
