// Top-K of a window by 32-bit keys, by 256 threads (the scoring kernels and the selection by weight).
#pragma once

#include "lrsa_internal.h"

namespace lrsa {

constexpr int kSelectThreads = 256;

// fp32 bits -> uint32 whose unsigned order is the float order.
__device__ __forceinline__ uint32_t order_key(float f) {
  uint32_t u = __float_as_uint(f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
// Barrier of the 256 scoring threads (named barrier 1): the whole block in the one-unit-per-CTA kernel,
// or of the cluster kernel.
__device__ __forceinline__ void scoring_warps_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// The K largest of the L keys in shared memory (the unsigned order counts; equal keys: the lower index), whose least and
// largest are kmin and kmax: out[0 .. K) = pos0 + index, ascending.  hist: two histograms of 256 bins, zero (and seen so by
// all threads); wtot: eight words.  Ends without a barrier.
__device__ __forceinline__ void radix_select_emit(const uint32_t* key, int L, int K, uint32_t kmin, uint32_t kmax, uint32_t* hist,
                                                  int* wtot, int32_t* out, int pos0) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // The keys of a window usually share their leading bits (the scores of one window lie within a small factor of
  // each other): those bits are fixed at once, and the 8-bit passes start at the highest bit in which two
  // keys differ.  (A pass over shared bits would also send every key to one histogram bin: a thousand
  // serialised shared-memory atomics.)
  const uint32_t diff = kmin ^ kmax;
  const int top = diff ? 31 - __clz(diff) : -1;                  // highest differing bit, -1: all keys equal
  uint32_t mask = top >= 31 ? 0u : ~((2u << (top < 0 ? 0 : top)) - 1u);
  if (top < 0) mask = 0xffffffffu;
  uint32_t prefix = kmax & mask;
  int remaining = K;
  // One barrier per pass: every warp finds the bin of the K-th key itself, and the histograms take turns.  (With one warp
  // searching and four barriers a pass a call took 28.9 us instead of 27.4 at 32K tokens in windows of 1024.)
  int pass = 0;
  for (int shift = top < 0 ? -1 : max(top - 7, 0); shift >= 0; shift = shift == 0 ? -1 : max(shift - 8, 0), ++pass) {
    uint32_t* h = hist + (pass & 1) * 256;
    for (int i = tid; i < L; i += kSelectThreads) {
      const uint32_t k = key[i];
      if ((k & mask) == prefix) atomicAdd(&h[(k >> shift) & 255u], 1u);
    }
    scoring_warps_sync();
    // lane l owns bins 255-8l ... 248-8l, highest first
    const uint4 hi = *reinterpret_cast<const uint4*>(h + 252 - 8 * lane), lo = *reinterpret_cast<const uint4*>(h + 248 - 8 * lane);
    const uint32_t c[8] = {hi.w, hi.z, hi.y, hi.x, lo.w, lo.z, lo.y, lo.x};
    uint32_t tot = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) tot += c[e];
    uint32_t incl = tot;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t n = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += n;
    }
    uint32_t above = incl - tot;   // elements in bins above this lane's
    const bool mine = above < (uint32_t)remaining && (uint32_t)remaining <= incl;
    uint32_t bin = 255 - 8 * lane, cnt = c[0];
    bool more = true;
#pragma unroll
    for (int e = 0; e < 7; ++e) {
      more = more && above + c[e] < (uint32_t)remaining;
      if (more) { above += c[e]; --bin; cnt = c[e + 1]; }
    }
    const int src = __ffs(__ballot_sync(0xffffffffu, mine)) - 1;
    bin = __shfl_sync(0xffffffffu, bin, src);
    cnt = __shfl_sync(0xffffffffu, cnt, src);              // keys in the chosen bin
    remaining -= (int)__shfl_sync(0xffffffffu, above, src);
    prefix |= bin << shift;
    mask |= 255u << shift;
    // Every key of the chosen bin is kept: the remaining bits need not be resolved.  (With 8-bit digits a
    // thousand keys are alone in their bin after two passes, so this ends the search at half its length.)
    // The threshold is then the bin's lowest possible key: keys above it are kept as "greater", keys equal to
    // it as "equal", of which `remaining` is at least as many as exist.
    if ((int)cnt == remaining) break;
    if (pass > 0) {   // a third pass needs the first histogram again (windows of keys that differ in their last bits only)
      hist[((pass + 1) & 1) * 256 + tid] = 0;
      scoring_warps_sync();
    }
  }
  const uint32_t kth = prefix;    // K-th largest key
  const int need_eq = remaining;  // how many keys equal to it are kept (lowest positions first)

  // emit kept positions in ascending order: every thread takes a run of consecutive tokens, one block
  // scan gives the number of kept tokens before the run
  const int per = (L + kSelectThreads - 1) / kSelectThreads;
  const int i_lo = min(L, tid * per), i_hi = min(L, i_lo + per);
  int packed = 0;   // tokens above the K-th score | tokens equal to it << 16
  for (int i = i_lo; i < i_hi; ++i) {
    const uint32_t k = key[i];
    packed += (k > kth ? 1 : 0) | (k == kth ? 1 << 16 : 0);
  }
  int incl = packed;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int n = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += n;
  }
  if (lane == 31) wtot[warp] = incl;
  scoring_warps_sync();
  int excl = incl - packed;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < warp) excl += wtot[j];
  int gt_before = excl & 0xffff, eq_before = excl >> 16;
  for (int i = i_lo; i < i_hi; ++i) {
    const uint32_t k = key[i];
    if (k > kth) {
      out[gt_before + min(eq_before, need_eq)] = pos0 + i;
      ++gt_before;
    } else if (k == kth) {
      if (eq_before < need_eq) out[gt_before + eq_before] = pos0 + i;
      ++eq_before;
    }
  }
}

}  // namespace lrsa
