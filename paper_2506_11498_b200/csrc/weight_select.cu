// Selection by accumulated attention weight: of every scored window the top_k heaviest positions (the alternative to the
// score of Eq. 4-8).  One CTA per window: its weights become keys in shared memory whose unsigned order is the order of
// the weights, a radix select finds the K-th, a scan emits the positions.  A token is read once and K positions a window
// are written: the kernel is a chain of barriers, not of transfers.
#include "select_sm100.h"
#include "weight_select.h"

namespace lrsa {
namespace {

__global__ void __launch_bounds__(kSelectThreads) weight_select_kernel(const __grid_constant__ WeightSelectArgs a) {
  extern __shared__ __align__(16) uint32_t sel_smem[];
  uint32_t* hist = sel_smem;               // two of 256 bins
  uint32_t* kred = hist + 512;             // [least, largest key] of the eight warps
  int* wtot = reinterpret_cast<int*>(kred + 16);
  uint32_t* key = reinterpret_cast<uint32_t*>(wtot + 8);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, L = a.L;
  int item = blockIdx.x, sq = 0;
  while (sq + 1 < a.n && item >= a.item0[sq + 1]) ++sq;
  item -= a.item0[sq];
  const int bh = item / a.windows[sq], w = item % a.windows[sq];
  hist[tid] = hist[256 + tid] = 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (a.status && blockIdx.x == 0 && tid == 0) *a.status = 0;
  const float* src = a.weight + (size_t)bh * a.row + a.first[sq] + (long long)w * L;
  uint32_t kmin = 0xffffffffu, kmax = 0u;
#pragma unroll 4
  for (int i = tid; i < L; i += kSelectThreads) {
    float x = src[i] + 0.f;                // -0 and 0 are the same weight
    if (x != x) x = -INFINITY;             // NaN is kept last
    const uint32_t k = order_key(x);
    key[i] = k;
    kmin = min(kmin, k);
    kmax = max(kmax, k);
  }
  kmin = __reduce_min_sync(0xffffffffu, kmin);
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  if (lane == 0) { kred[warp] = kmin; kred[8 + warp] = kmax; }
  scoring_warps_sync();
#pragma unroll
  for (int i = 0; i < 8; ++i) { kmin = min(kmin, kred[i]); kmax = max(kmax, kred[8 + i]); }
  radix_select_emit(key, L, a.K, kmin, kmax, hist, wtot, a.idx + ((size_t)bh * a.Wtot + a.woff[sq] + w) * a.K, a.emit0[sq] + w * L);
}

}  // namespace

int launch_weight_select(const WeightSelectArgs& a, cudaStream_t st) {
  if (a.n == 0 || a.item0[a.n] == 0) return LRSA_OK;
  const size_t smem = (512 + 16 + 8 + (size_t)a.L) * 4;
  if (smem > 48 * 1024)
    LRSA_CUDA_CHECK(cudaFuncSetAttribute(weight_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  LRSA_CUDA_CHECK(launch_dependent(weight_select_kernel, dim3((unsigned)a.item0[a.n]), dim3(kSelectThreads), smem, st, 1, a));
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
