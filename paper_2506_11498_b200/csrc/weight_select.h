// The selection by accumulated weight, for the entry point and the store that keeps rows by it.
#pragma once

#include <type_traits>

#include "lrsa_internal.h"

namespace lrsa {

constexpr int kSelectSeqs = 16;   // sequences of a launch
struct WeightSelectArgs {
  const float* weight;   // [B*Hkv][row]
  int32_t* idx;          // [B*Hkv][Wtot][K]
  long long row;
  int L, K, Wtot, n;     // n sequences, with item0[n] windows over all (batch, KV head) pairs
  int item0[kSelectSeqs + 1];
  int windows[kSelectSeqs], first[kSelectSeqs];    // per pair; token of window 0 in the row
  int woff[kSelectSeqs], emit0[kSelectSeqs];       // first window in idx; position of window 0
};

// fp32 bits -> uint32 whose unsigned order is the float order.
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

constexpr int kSelSmemFree = 38 * 1024, kSelSmemMax = 128 * 1024;   // keys of a window: what needs no leave; the longest window
constexpr int kSelThreads = 256, kSelWarps = kSelThreads / 32, kDigit = 10, kBins = 1 << kDigit;   // a thread owns four bins
static_assert(kBins == 4 * kSelThreads, "four bins a thread");

struct alignas(16) SelectShared {
  uint32_t hist[2][kBins];        // of the digits in turn
  uint32_t kred[2][kSelWarps], wsum[kSelWarps], found[3];
  int above_eq[kSelWarps];        // kept keys of a warp's tokens: above the K-th | equal to it << 16
};
// (ahead of the wait for the kernel in front)
__device__ __forceinline__ void select_clear(SelectShared& sh) {
  reinterpret_cast<uint4*>(sh.hist[0])[threadIdx.x] = reinterpret_cast<uint4*>(sh.hist[1])[threadIdx.x] = make_uint4(0, 0, 0, 0);
}

// The K heaviest tokens of a window of L, by 256 threads: out[0 .. K) = pos0 + index, ascending; equal weights keep the lower
// index.  Token i < in_ring has weight ring[i], the others src[i].  key: L words of shared memory.
// The weights become keys whose unsigned order is theirs, a radix select finds the K-th, warps of consecutive tokens emit
// the positions by ballots.  A token is read once and K positions are written: a chain of barriers, not of transfers.
__device__ __forceinline__ void select_window_by_weight(SelectShared& sh, uint32_t* key, int L, int K, const float* src, const float* ring,
                                                        int in_ring, int32_t* out, int pos0) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint32_t kmin = 0xffffffffu, kmax = 0u;
  auto take = [&](float x, int i) {
    x += 0.f;                                         // -0 and 0 are the same weight
    const uint32_t k = x != x ? 0u : order_key(x);    // NaN is kept last, behind -infinity (0x007fffff)
    key[i] = k;
    kmin = min(kmin, k);
    kmax = max(kmax, k);
  };
  // n tokens a thread, all loads ahead of their use; the last ones may not be there
  auto load = [&](int i, auto n, auto whole) {
    constexpr int kAhead = decltype(n)::value;
    constexpr bool kWhole = decltype(whole)::value;
    float x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = i + u * kSelThreads;
      if (kWhole || j < L) x[u] = j < in_ring ? ring[j] : src[j];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (kWhole || i + u * kSelThreads < L) take(x[u], i + u * kSelThreads);
  };
  int at = tid;
  for (; at - tid + 16 * kSelThreads <= L; at += 16 * kSelThreads) load(at, std::integral_constant<int, 16>(), std::true_type());
  for (; at - tid < L; at += 4 * kSelThreads) load(at, std::integral_constant<int, 4>(), std::false_type());
  kmin = __reduce_min_sync(0xffffffffu, kmin);
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  if (lane == 0) { sh.kred[0][warp] = kmin; sh.kred[1][warp] = kmax; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSelWarps; ++i) { kmin = min(kmin, sh.kred[0][i]); kmax = max(kmax, sh.kred[1][i]); }

  // The leading bits that all keys share are fixed at once, then ten-bit digits from the highest differing bit on.  (The first digit
  // holds the exponents of the weights and little more: with eight bits hundreds of keys meet in a bin, and their additions
  // take turns: 480 windows of 4096 tokens took a tenth longer.)
  const uint32_t diff = kmin ^ kmax;
  const int top = diff ? 31 - __clz(diff) : -1;
  uint32_t mask = top < 0 ? 0xffffffffu : top >= 31 ? 0u : ~((2u << top) - 1u), prefix = kmax & mask;
  int remaining = K;
  for (int shift = top < 0 ? -1 : max(top - (kDigit - 1), 0), pass = 0; shift >= 0; shift = shift == 0 ? -1 : max(shift - kDigit, 0), ++pass) {
    uint32_t* h = sh.hist[pass & 1];
#pragma unroll 4
    for (int i = tid; i < L; i += kSelThreads) {
      const uint32_t k = key[i];
      if ((k & mask) == prefix) atomicAdd(&h[(k >> shift) & (kBins - 1)], 1u);
    }
    __syncthreads();
    // thread i owns bins 1023-4i ... 1020-4i, highest first; keys in bins above them
    uint4* own = reinterpret_cast<uint4*>(h) + (kSelThreads - 1 - tid);
    const uint4 x = *own;
    *own = zero;   // (the histogram of the digit after the next one)
    const uint32_t c[4] = {x.w, x.z, x.y, x.x}, tot = (x.x + x.y) + (x.z + x.w);
    uint32_t incl = tot;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t n = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += n;
    }
    if (lane == 31) sh.wsum[warp] = incl;
    __syncthreads();
    uint32_t above = incl - tot;
#pragma unroll
    for (int j = 0; j < kSelWarps; ++j)
      if (j < warp) above += sh.wsum[j];
    if (above < (uint32_t)remaining && (uint32_t)remaining <= above + tot) {   // the K-th key is in one of this thread's bins
      uint32_t bin = kBins - 1 - 4 * tid, cnt = c[0];
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (above + cnt < (uint32_t)remaining) { above += cnt; --bin; cnt = c[e + 1]; }
      sh.found[0] = bin; sh.found[1] = cnt; sh.found[2] = above;
    }
    __syncthreads();
    const uint32_t bin = sh.found[0], cnt = sh.found[1];
    remaining -= (int)sh.found[2];
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
  const int per = (L + 32 * kSelWarps - 1) / (32 * kSelWarps) * 32, i0 = warp * per, i1 = min(L, i0 + per);
  int packed = 0;
  for (int i = i0; i < i1; i += 32) {
    const bool in = i + lane < i1;
    const uint32_t k = in ? key[i + lane] : 0u;
    packed += __popc(__ballot_sync(0xffffffffu, in && k > kth)) | __popc(__ballot_sync(0xffffffffu, in && k == kth)) << 16;
  }
  if (lane == 0) sh.above_eq[warp] = packed;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int j = 0; j < kSelWarps; ++j)
    if (j < warp) before += sh.above_eq[j];
  int gt = before & 0xffff, eq = before >> 16;
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

}  // namespace lrsa
