// Selection by accumulated attention weight: of every scored window the top_k heaviest positions (the alternative to the
// score of Eq. 4-8).  One CTA per window.
#include "weight_select.h"

namespace lrsa {
namespace {

// (Eight CTAs on an SM: those of the call behind it start beside the last ones, 480 windows of 4096 tokens 13.3 to 14.3 us in a run of
// calls instead of 15.6 with six.)
__global__ void __launch_bounds__(kSelThreads, 8) weight_select_kernel(const __grid_constant__ WeightSelectArgs a) {
  extern __shared__ __align__(16) uint32_t key[];
  __shared__ SelectShared sh;
  int item = blockIdx.x, sq = 0;
  while (sq + 1 < a.n && item >= a.item0[sq + 1]) ++sq;
  item -= a.item0[sq];
  const int bh = item / a.windows[sq], w = item % a.windows[sq];
  select_clear(sh);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  select_window_by_weight(sh, key, a.L, a.K, a.weight + (size_t)bh * a.row + a.first[sq] + (long long)w * a.L, nullptr, 0,
                          a.idx + ((size_t)bh * a.Wtot + a.woff[sq] + w) * a.K, a.emit0[sq] + w * a.L);
}

}  // namespace

static int launch_weight_select(const WeightSelectArgs& a, cudaStream_t st) {
  if (a.n == 0 || a.item0[a.n] == 0) return LRSA_OK;
  const size_t smem = (size_t)a.L * 4;
  if (smem > kSelSmemFree)
    LRSA_CUDA_CHECK(cudaFuncSetAttribute(weight_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelSmemMax));
  LRSA_CUDA_CHECK(launch_dependent(weight_select_kernel, dim3((unsigned)a.item0[a.n]), dim3(kSelThreads), smem, st, 1, a));
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
