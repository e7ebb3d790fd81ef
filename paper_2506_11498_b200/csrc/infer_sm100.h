// What the decode kernels of the caches share: warp-level products, cluster accesses, how the keys are dealt out, the merge
// of partial results.
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
__device__ __forceinline__ uint4 ld_stream(const void* p) {   // read once: no place in L1
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// One CTA per (batch, query head): merges the partial results of its splits, or of its clusters.  kRows thread rows (one
// for clusters, of which there are at most kDecMaxGroups) take alternate results, four at a time with all their loads issued before the
// arithmetic (the kernel is a chain of L2 round trips otherwise), then the rows are merged through shared memory.
constexpr int kMergeRows = 8;
namespace {   // a copy for each user
template <int D, int kRows>
__global__ void __launch_bounds__(kRows * D) decode_merge_kernel(const float* part, __nv_bfloat16* o, float* lse, int Hq,
                                                                  int Hkv, int G, int n_split) {
  __shared__ float sm_m[kRows], sm_l[kRows], sm_o[kRows][D];
  const int bhq = blockIdx.x, b = bhq / Hq, hq = bhq % Hq, hkv = hq / G, g = hq % G;
  const int c = threadIdx.x % D, row = threadIdx.x / D;
  const float* base = part + (((size_t)(b * Hkv + hkv) * n_split) * G + g) * (D + 2);
  const size_t stride = (size_t)G * (D + 2);
  float M = -INFINITY, acc = 0.f, l = 0.f;
  constexpr int kBatch = 4;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // the partial results of the kernel in front of this one
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int s0 = row; s0 < n_split; s0 += kRows * kBatch) {
    float ms[kBatch], vs[kBatch], ls[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int s = s0 + u * kRows;
      const bool in = s < n_split;
      ms[u] = in ? __ldcg(base + s * stride + D) : -INFINITY;
      vs[u] = in ? __ldcg(base + s * stride + c) : 0.f;
      ls[u] = in ? __ldcg(base + s * stride + D + 1) : 0.f;
    }
    float mn = M;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) mn = fmaxf(mn, ms[u]);
    if (mn == -INFINITY) continue;
    const float f0 = exp2f(M - mn);   // exp2f(-inf) = 0 while nothing has been merged
    acc *= f0; l *= f0;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float f = exp2f(ms[u] - mn);
      acc = fmaf(vs[u], f, acc);
      l = fmaf(ls[u], f, l);
    }
    M = mn;
  }
  sm_o[row][c] = acc;
  if (c == 0) { sm_m[row] = M; sm_l[row] = l; }
  __syncthreads();
  if (row == 0) {
    float Mt = -INFINITY;
    for (int r = 0; r < kRows; ++r) Mt = fmaxf(Mt, sm_m[r]);
    float at = 0.f, lt = 0.f;
    for (int r = 0; r < kRows; ++r) {
      const float f = sm_m[r] == -INFINITY ? 0.f : exp2f(sm_m[r] - Mt);
      at = fmaf(sm_o[r][c], f, at);
      lt = fmaf(sm_l[r], f, lt);
    }
    o[(size_t)bhq * D + c] = __float2bfloat16(at / lt);
    if (c == 0 && lse) lse[bhq] = (Mt + log2f(lt)) * 0.6931471805599453f;
  }
}

}  // namespace

// How the keys of the (batch, KV head) pairs are dealt out: to `groups` clusters of `splits` CTAs of `warps` warps each.
struct DecodePlan { int nh, warps, blocks, splits, groups; };
constexpr int kDecMaxSplits = 16, kDecMaxGroups = 16;
// (blocks: what a warp takes at a time, 8 KB of K and V, per pair)
inline DecodePlan deal_blocks(const Geom& g, int blocks, int max_splits = kDecMaxSplits) {
  DecodePlan p;
  p.nh = g.G > 8 ? 2 : 1;
  const long long BH = (long long)g.B * g.Hkv;
  p.blocks = blocks > 0 ? blocks : 1;
  // 16 warps (8 with two groups of heads) are resident per SM, as one large CTA or several small ones.  Large ones
  // have fewer partial results to merge; small ones fill the SMs more evenly when every SM has several blocks per warp
  // to do.  A round of blocks takes about 1.3 us, a CTA's start and merge as long as two, the second kernel as three; a
  // cluster lies in one group of SMs (ClusterRoom).  (One sequence, 4 heads, d = 128: 9471 keys, one cluster for a
  // head 17.7 us a token with 8 CTAs, 15.8 with 16; 66 000 keys 107 us with one cluster of 16, 34.5 with two.)
  const int max_warps = dec_max_warps(p.nh);
  p.warps = BH * p.blocks > 2LL * kSms * max_warps ? 4 : max_warps;
  const int per_sm = max_warps / p.warps;
  const ClusterRoom& room = cluster_room();
  long long best = -1;
  for (int s = 1; s <= max_splits; s *= 2) {
    const long long at_once = room.at_once(per_sm, s);
    for (int grp = 1; grp <= kDecMaxGroups; grp *= 2) {
      const int n = s * grp;
      if (n > 1 && ((n - 1) * p.warps >= p.blocks || BH * n > (long long)kSms * per_sm * 4)) break;
      const long long waves = (BH * grp + at_once - 1) / at_once;
      const int per_cta = (p.blocks + n - 1) / n;
      const long long cost = waves * ((per_cta + p.warps - 1) / p.warps + 2) + (grp > 1 ? 3 : 0);
      if (best < 0 || cost < best) { best = cost; p.splits = s; p.groups = grp; }
    }
  }
  return p;
}

}  // namespace lrsa
