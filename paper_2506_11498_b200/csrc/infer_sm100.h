// What the decode kernels of the caches share: warp-level products, cluster accesses, the terms of their plans.
#pragma once

#include "lrsa_internal.h"
#include "sm100_ptx.h"

namespace lrsa {

__device__ __forceinline__ void wait_for_front() {
  asm volatile("griddepcontrol.wait;" ::: "memory");   // may be launched before the kernel in front of it has ended
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

constexpr int kDecMaxWarps = 16;
// Warps of the largest CTA: 128 registers hold the operands of one group of 8 heads; two groups take more.
__host__ __device__ constexpr int dec_max_warps(int nh) { return nh == 1 ? kDecMaxWarps : kDecMaxWarps / 2; }

// D (16x8, fp32) += A (16x16, bf16, row) * B (16x8, bf16, col)
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// transpose of an 8x8 matrix of 16-bit elements held two per lane
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// this CTA's variable at `p` as CTA `rank` of the cluster has it
__device__ __forceinline__ float ld_cluster(const float* p, int rank) {
  float v;
  uint32_t addr;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(ptx::smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// How the keys of the (batch, KV head) pairs are dealt out: to `groups` clusters of `splits` CTAs of `warps` warps each.
struct DecodePlan { int nh, warps, blocks, splits, groups; };
constexpr int kDecMaxSplits = 16, kDecMaxGroups = 16;

}  // namespace lrsa
