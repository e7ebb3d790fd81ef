// Selection by accumulated attention weight: of every scored window the top_k heaviest positions (the alternative to the
// score of Eq. 4-8).  One CTA per window: its weights become keys in shared memory whose unsigned order is the order of
// the weights, a radix select finds the K-th, warps of consecutive tokens emit the positions by ballots.  A token is read once and K
// positions a window are written: the kernel is a chain of barriers, not of transfers.
#include "weight_select.h"

namespace lrsa {
namespace {

// fp32 bits -> uint32 whose unsigned order is the float order.
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

constexpr int kThreads = 256, kWarps = kThreads / 32, kDigit = 10, kBins = 1 << kDigit;   // a thread owns four bins

__global__ void __launch_bounds__(kThreads) weight_select_kernel(const __grid_constant__ WeightSelectArgs a) {
  static_assert(kBins == 4 * kThreads, "four bins a thread");
  extern __shared__ __align__(16) uint32_t key[];
  __shared__ __align__(16) uint32_t hist[2][kBins];   // of the digits in turn
  __shared__ uint32_t kred[2][kWarps], wsum[kWarps], found[3];
  __shared__ int above_eq[kWarps];                    // kept keys of a warp's tokens: above the K-th | equal to it << 16
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, L = a.L;
  int item = blockIdx.x, sq = 0;
  while (sq + 1 < a.n && item >= a.item0[sq + 1]) ++sq;
  item -= a.item0[sq];
  const int bh = item / a.windows[sq], w = item % a.windows[sq];
  const uint4 zero = make_uint4(0, 0, 0, 0);
  reinterpret_cast<uint4*>(hist[0])[tid] = reinterpret_cast<uint4*>(hist[1])[tid] = zero;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (a.status && blockIdx.x == 0 && tid == 0) *a.status = 0;
  const float* src = a.weight + (size_t)bh * a.row + a.first[sq] + (long long)w * L;
  uint32_t kmin = 0xffffffffu, kmax = 0u;
  const int pos0 = a.emit0[sq] + w * L;
  auto take = [&](float x, int i) {
    x += 0.f;                              // -0 and 0 are the same weight
    if (x != x) x = -INFINITY;             // NaN is kept last
    const uint32_t k = order_key(x);
    key[i] = k;
    kmin = min(kmin, k);
    kmax = max(kmax, k);
  };
  // tokens [0, in_ring) of the window are in the ring, wherever it wraps
  const int in_ring = a.ring ? min(L, max(a.ring_below - pos0, 0)) : 0;
  if (in_ring > 0) {
    const float* ring = a.ring + (size_t)bh * a.ring_len;
    const int at = (pos0 - a.ring_first) % a.ring_len;
    for (int i = tid; i < in_ring; i += kThreads) take(ring[at + i < a.ring_len ? at + i : at + i - a.ring_len], i);
  }
#pragma unroll 8
  for (int i = in_ring + tid; i < L; i += kThreads) take(src[i], i);
  kmin = __reduce_min_sync(0xffffffffu, kmin);
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  if (lane == 0) { kred[0][warp] = kmin; kred[1][warp] = kmax; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWarps; ++i) { kmin = min(kmin, kred[0][i]); kmax = max(kmax, kred[1][i]); }

  // The leading bits that all keys share are fixed at once, then ten-bit digits from the highest differing bit on.  (The first digit
  // holds the exponents of the weights and little more: with eight bits hundreds of keys meet in a bin, and their additions
  // take turns: 480 windows of 4096 tokens 16.1 us instead of 13.1.)
  const uint32_t diff = kmin ^ kmax;
  const int top = diff ? 31 - __clz(diff) : -1;
  uint32_t mask = top < 0 ? 0xffffffffu : top >= 31 ? 0u : ~((2u << top) - 1u), prefix = kmax & mask;
  int remaining = a.K;
  for (int shift = top < 0 ? -1 : max(top - (kDigit - 1), 0), pass = 0; shift >= 0; shift = shift == 0 ? -1 : max(shift - kDigit, 0), ++pass) {
    uint32_t* h = hist[pass & 1];
#pragma unroll 4
    for (int i = tid; i < L; i += kThreads) {
      const uint32_t k = key[i];
      if ((k & mask) == prefix) atomicAdd(&h[(k >> shift) & (kBins - 1)], 1u);
    }
    __syncthreads();
    // thread i owns bins 1023-4i ... 1020-4i, highest first; keys in bins above them
    uint4* own = reinterpret_cast<uint4*>(h) + (kThreads - 1 - tid);
    const uint4 x = *own;
    *own = zero;   // (the histogram of the digit after the next one)
    const uint32_t c[4] = {x.w, x.z, x.y, x.x}, tot = (x.x + x.y) + (x.z + x.w);
    uint32_t incl = tot;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t n = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += n;
    }
    if (lane == 31) wsum[warp] = incl;
    __syncthreads();
    uint32_t above = incl - tot;
#pragma unroll
    for (int j = 0; j < kWarps; ++j)
      if (j < warp) above += wsum[j];
    if (above < (uint32_t)remaining && (uint32_t)remaining <= above + tot) {   // the K-th key is in one of this thread's bins
      uint32_t bin = kBins - 1 - 4 * tid, cnt = c[0];
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (above + cnt < (uint32_t)remaining) { above += cnt; --bin; cnt = c[e + 1]; }
      found[0] = bin; found[1] = cnt; found[2] = above;
    }
    __syncthreads();
    const uint32_t bin = found[0], cnt = found[1];
    remaining -= (int)found[2];
    // (a digit that overlaps the one above it, at the last bits: its upper bits are in the prefix already)
    prefix |= bin << shift;
    mask |= (uint32_t)(kBins - 1) << shift;
    // Every key of the bin is kept: the other bits need not be resolved.  The bin's lowest key is then the border, the keys above it
    // count as above, those equal to it as equal, of which there are no more than `remaining`.
    if ((int)cnt == remaining) break;
  }
  const uint32_t kth = prefix;
  const int need_eq = remaining;   // so many of the keys equal to it are kept, the lowest positions

  // a warp takes consecutive tokens, 32 at a time
  const int per = (L + 32 * kWarps - 1) / (32 * kWarps) * 32, i0 = warp * per, i1 = min(L, i0 + per);
  int packed = 0;
  for (int i = i0; i < i1; i += 32) {
    const bool in = i + lane < i1;
    const uint32_t k = in ? key[i + lane] : 0u;
    packed += __popc(__ballot_sync(0xffffffffu, in && k > kth)) | __popc(__ballot_sync(0xffffffffu, in && k == kth)) << 16;
  }
  if (lane == 0) above_eq[warp] = packed;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int j = 0; j < kWarps; ++j)
    if (j < warp) before += above_eq[j];
  int gt = before & 0xffff, eq = before >> 16;
  int32_t* out = a.idx + ((size_t)bh * a.Wtot + a.woff[sq] + w) * a.K;
  const uint32_t lower = (1u << lane) - 1u;
  for (int i = i0; i < i1; i += 32) {
    const bool in = i + lane < i1;
    const uint32_t k = in ? key[i + lane] : 0u;
    const bool is_gt = in && k > kth, is_eq = in && k == kth;
    const uint32_t bg = __ballot_sync(0xffffffffu, is_gt), be = __ballot_sync(0xffffffffu, is_eq);
    const int my_gt = gt + __popc(bg & lower), my_eq = eq + __popc(be & lower);
    if (is_gt || (is_eq && my_eq < need_eq)) out[my_gt + min(my_eq, need_eq)] = pos0 + i + lane;
    gt += __popc(bg);
    eq += __popc(be);
  }
}

}  // namespace

int launch_weight_select(const WeightSelectArgs& a, cudaStream_t st) {
  if (a.n == 0 || a.item0[a.n] == 0) return LRSA_OK;
  const size_t smem = (size_t)a.L * 4;
  if (smem > 38 * 1024)
    LRSA_CUDA_CHECK(cudaFuncSetAttribute(weight_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  LRSA_CUDA_CHECK(launch_dependent(weight_select_kernel, dim3((unsigned)a.item0[a.n]), dim3(kThreads), smem, st, 1, a));
  launch_counter().n++;
  return LRSA_OK;
}

}  // namespace lrsa

using namespace lrsa;

extern "C" {

int lrsa_weight_select(const lrsa_params_t* params, const float* weight, int32_t* idx, void* cuda_stream) {
  NvtxRange nvtx_range("lrsa_weight_select");
  launch_counter().n = 0;
  Geom whole;
  const int rc = make_geom(params, &whole);
  if (rc != LRSA_OK) return rc;
  if (!weight || (whole.Wtot > 0 && !idx)) return LRSA_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(weight) | reinterpret_cast<uintptr_t>(idx)) & 3u) return LRSA_ERR_INVALID_ARG;
  const long long BH = (long long)whole.B * whole.Hkv;
  if (BH * whole.Wtot > 0x7fffffffLL) return LRSA_ERR_UNSUPPORTED;
  WeightSelectArgs a = {};
  a.weight = weight; a.idx = idx; a.row = whole.Nrow; a.L = whole.L; a.K = whole.K; a.Wtot = whole.Wtot;
  const int total = whole.n_seqs > 0 ? whole.n_seqs : 1;
  int woff = 0;
  for (int s = 0; s < total; ++s) {
    Geom g;
    seq_geom(whole, whole.cu, whole.n_seqs, s, woff, &g);
    woff += g.Wsel;
    if (g.Wsel > 0) {
      a.windows[a.n] = g.Wsel; a.first[a.n] = g.tok0 + g.S; a.emit0[a.n] = g.tok0 + g.S; a.woff[a.n] = g.woff;
      a.item0[a.n + 1] = a.item0[a.n] + (int)BH * g.Wsel;
      ++a.n;
    }
    if (a.n == kSelectSeqs || s + 1 == total) {
      const int r = launch_weight_select(a, static_cast<cudaStream_t>(cuda_stream));
      if (r != LRSA_OK) return r;
      a.n = 0;
    }
  }
  return LRSA_OK;
}

}  // extern "C"
