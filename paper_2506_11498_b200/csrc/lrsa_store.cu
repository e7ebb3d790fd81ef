// The store: a condensed KV cache like that of lrsa_infer.cu whose kept rows may be held in 8 bits and whose windows may be
// cut by accumulated attention weight, and decode attention over it.
//
// Per (batch, KV head):
//   list    [Wcap * Kp][d]  the top_k kept rows of every compressed window; a window starts a block of its own, Kp = top_k
//           rounded up to whole blocks (the rows behind the top_k are zero and never visible).  8 bits: one scale per block
//           of `block` rows for K and one for V; a block is written once, complete, so no row is ever rounded twice.
//   recent  [S + 2L][d]     bf16: the sinks, then the ring of uncompressed tokens (position p >= S at row S + (p - S) mod 2L)
//   weight  [2L]            fp32: the attention weight that the ring's tokens have gathered (keep by weight)
// A window leaves the ring when the first token of the chunk after the next one arrives, as in lrsa_infer.cu.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "infer_sm100.h"
#include "weight_select.h"

namespace lrsa {
namespace {

struct StoreGeom {
  int type, block, Kp, Wcap, rows_list, recent;
  bool by_weight;
};

int make_store_geom(const lrsa_params_t* params, const lrsa_store_t* s, Geom* g, StoreGeom* o) {
  const int rc = make_geom(params, g);
  if (rc != LRSA_OK) return rc;
  if (!s) return LRSA_ERR_INVALID_ARG;
  if (params->n_seqs > 0 || g->ndp != 1) return LRSA_ERR_UNSUPPORTED;
  if (s->list_type < LRSA_LIST_BF16 || s->list_type > LRSA_LIST_INT8) return LRSA_ERR_INVALID_ARG;
  if (s->keep != LRSA_KEEP_LAG && s->keep != LRSA_KEEP_WEIGHT) return LRSA_ERR_INVALID_ARG;
  if (s->block != 16 && s->block != 32 && s->block != 64 && s->block != 128) return LRSA_ERR_UNSUPPORTED;
  o->type = s->list_type; o->block = s->block; o->by_weight = s->keep == LRSA_KEEP_WEIGHT;
  const int c_last = g->N > g->S ? (g->N - 1 - g->S) / g->L : 0;
  o->Wcap = c_last >= 2 ? c_last - 1 : 0;
  o->Kp = (g->K + s->block - 1) / s->block * s->block;
  o->recent = g->S + 2 * g->L;
  // rows are numbered in 32 bits inside a head
  if ((long long)o->Wcap * o->Kp > 0x7fffffffLL || (long long)g->S + 2LL * g->L > 0x7fffffffLL) return LRSA_ERR_UNSUPPORTED;
  o->rows_list = o->Wcap * o->Kp;
  return LRSA_OK;
}

bool mis(const void* p, size_t al) { return reinterpret_cast<uintptr_t>(p) % al != 0; }

// Are the tensors of the store there, and aligned?
int check_store(const lrsa_store_t* s, const StoreGeom& o) {
  if (!s->k_recent || !s->v_recent || mis(s->k_recent, 16) || mis(s->v_recent, 16)) return LRSA_ERR_INVALID_ARG;
  if (o.by_weight && (!s->weight || mis(s->weight, 4))) return LRSA_ERR_INVALID_ARG;
  if (o.Wcap == 0) return LRSA_OK;
  if (!s->k_list || !s->v_list || !s->idx || mis(s->k_list, 16) || mis(s->v_list, 16) || mis(s->idx, 4)) return LRSA_ERR_INVALID_ARG;
  if (o.type != LRSA_LIST_BF16 && (!s->k_scale || !s->v_scale || mis(s->k_scale, 4) || mis(s->v_scale, 4))) return LRSA_ERR_INVALID_ARG;
  return LRSA_OK;
}

// ---- growing the store ----
constexpr int kRowThreads = 256;

struct StoreRows {
  const __nv_bfloat16 *k_new, *v_new;   // [BH][n_new][d], token p at row p - p_first
  const float* w_new;                   // [BH][n_new] or null (zero)
  __nv_bfloat16 *k_recent, *v_recent;
  float* weight;                        // null: not kept
  void *k_list, *v_list;
  float *k_scale, *v_scale;
  const int32_t* idx;                   // [BH][Wcap][K]
  int* status;                          // cleared when not null
  int n_new, p_first, S, L, K, Kp, Wcap, rows_list, recent, block;
  int n_sink, p0, n_ins;                // new tokens [p_first, + n_sink) and [p0, + n_ins) go to the recent rows
  int w0, n_win, from_ring;             // kept rows of windows [w0, + n_win), out of the ring or out of the new tokens
  int copy_blocks, list_blocks;         // thread blocks per (batch, KV head)
};

// The least bf16 that is not below x (finite, positive); infinities and NaN stay.  With eight bits in the scale the quotient
// of a bf16 value and the scale lies at least 2^-17 (relative) away from every rounding border of the codes that it does
// not hit exactly, so a correctly rounded fp32 quotient gives the code of the exact one.
__device__ __forceinline__ float scale_up(float x) {
  return x < INFINITY ? __uint_as_float((__float_as_uint(x) + 0xffffu) & 0xffff0000u) : x;
}

// Tokens into the recent rows, and blocks of kept rows into the list.  Bound by the rows it moves: a copied row is read and
// written once; a kept row is read once (gathered by position, whole lines), held in registers while the block's largest
// magnitude is found, and written once in 8 bits.
template <int D, int T>
__global__ void __launch_bounds__(kRowThreads) store_rows_kernel(const __grid_constant__ StoreRows a) {
  constexpr int CPR = D / 8;                // 16-byte chunks per bf16 row
  __shared__ uint32_t s_max[kRowThreads / 32];
  const int tid = threadIdx.x, per = a.copy_blocks + a.list_blocks;
  const int bh = blockIdx.x / per, blk = blockIdx.x % per;
  wait_for_front();
  if (a.status && blockIdx.x == 0 && tid == 0) *a.status = 0;
  if (blk < a.copy_blocks) {
    const int item = blk * (kRowThreads / CPR) + tid / CPR, ch = tid % CPR;
    if (item >= a.n_sink + a.n_ins) return;
    const int p = item < a.n_sink ? a.p_first + item : a.p0 + (item - a.n_sink);
    const int at = p < a.S ? p : a.S + (p - a.S) % (2 * a.L);
    const size_t src = ((size_t)bh * a.n_new + (p - a.p_first)) * CPR + ch, dst = ((size_t)bh * a.recent + at) * CPR + ch;
    const uint4 k = reinterpret_cast<const uint4*>(a.k_new)[src], v = reinterpret_cast<const uint4*>(a.v_new)[src];
    reinterpret_cast<uint4*>(a.k_recent)[dst] = k;
    reinterpret_cast<uint4*>(a.v_recent)[dst] = v;
    if (a.weight && ch == 0 && p >= a.S)
      a.weight[(size_t)bh * 2 * a.L + (at - a.S)] = a.w_new ? a.w_new[(size_t)bh * a.n_new + (p - a.p_first)] : 0.f;
    return;
  }
  // a block of K (even) or of V (odd)
  const int lb = (blk - a.copy_blocks) >> 1, row0 = lb * a.block;   // first row, from window w0's first on
  const bool is_v = (blk - a.copy_blocks) & 1;
  const int w = a.w0 + row0 / a.Kp, j0 = row0 % a.Kp;
  const int32_t* idx = a.idx + ((size_t)bh * a.Wcap + w) * a.K;
  const __nv_bfloat16* src = a.from_ring ? (is_v ? a.v_recent : a.k_recent) + (size_t)bh * a.recent * D
                                         : (is_v ? a.v_new : a.k_new) + (size_t)bh * a.n_new * D;
  constexpr int kMost = 128 * CPR / kRowThreads;   // chunks per thread of the largest block
  uint4 x[kMost];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int c = i * kRowThreads + tid, r = c / CPR;
    x[i] = make_uint4(0, 0, 0, 0);
    if (r < a.block && j0 + r < a.K) {
      const int pos = idx[j0 + r];
      const int at = a.from_ring ? a.S + (pos - a.S) % (2 * a.L) : pos - a.p_first;
      x[i] = *reinterpret_cast<const uint4*>(src + (size_t)at * D + (c % CPR) * 8);
    }
  }
  const size_t out_row = (size_t)bh * a.rows_list + (size_t)w * a.Kp + j0;
  if constexpr (T == LRSA_LIST_BF16) {
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(is_v ? a.v_list : a.k_list) + out_row * D;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int c = i * kRowThreads + tid;
      if (c / CPR < a.block) reinterpret_cast<uint4*>(dst)[c] = x[i];
    }
  } else {
    // largest magnitude: bits without the sign are ordered like the values, infinities and NaN above all
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) most = max(most, max(u[e] & 0x7fffu, (u[e] >> 16) & 0x7fffu));
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if ((tid & 31) == 0) s_max[tid >> 5] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRowThreads / 32; ++i) most = max(most, s_max[i]);
    const float limit = T == LRSA_LIST_E4M3 ? 448.f : 127.f;
    const float scale = most ? fmaxf(scale_up(__fdiv_rn(__uint_as_float(most << 16), limit)), 1.17549435e-38f) : 1.f;
    if (tid == 0) {
      // NaN in a block must not become the floor's 2^-126 (fmaxf drops it): its rows then all stand for NaN, as they do for an infinity
      const bool nan = most > 0x7f80u;
      (is_v ? a.v_scale : a.k_scale)[out_row / a.block] = nan ? NAN : scale;
    }
    unsigned char* dst = static_cast<unsigned char*>(is_v ? a.v_list : a.k_list) + out_row * D;
    const bool finite = most < 0x7f80u;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int c = i * kRowThreads + tid;
      if (c / CPR >= a.block) continue;
      const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
      uint32_t code[4];   // two codes each
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = __fdiv_rn(__uint_as_float(u[e] << 16), scale), hi = __fdiv_rn(__uint_as_float(u[e] & 0xffff0000u), scale);
        if constexpr (T == LRSA_LIST_E4M3)
          code[e] = __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
        else
          code[e] = (__float2int_rn(lo) & 0xff) | (__float2int_rn(hi) & 0xff) << 8;
        if (!finite) code[e] = 0;
      }
      reinterpret_cast<uint2*>(dst)[c] = make_uint2(code[0] | code[1] << 16, code[2] | code[3] << 16);
    }
  }
}

int launch_store_rows(StoreRows a, const StoreGeom& o, int BH, int d, cudaStream_t st) {
  const int rpb = kRowThreads / (d / 8);
  a.copy_blocks = (a.n_sink + a.n_ins + rpb - 1) / rpb;
  a.list_blocks = a.n_win * (o.Kp / o.block) * 2;
  const long long grid = (long long)BH * (a.copy_blocks + a.list_blocks);
  if (grid == 0) return LRSA_OK;
  if (grid > 0x7fffffffLL) return LRSA_ERR_UNSUPPORTED;
  auto kern = d == 128 ? (o.type == LRSA_LIST_E4M3 ? store_rows_kernel<128, LRSA_LIST_E4M3> : o.type == LRSA_LIST_INT8 ? store_rows_kernel<128, LRSA_LIST_INT8> : store_rows_kernel<128, LRSA_LIST_BF16>)
                       : (o.type == LRSA_LIST_E4M3 ? store_rows_kernel<64, LRSA_LIST_E4M3> : o.type == LRSA_LIST_INT8 ? store_rows_kernel<64, LRSA_LIST_INT8> : store_rows_kernel<64, LRSA_LIST_BF16>);
  LRSA_CUDA_CHECK(launch_dependent(kern, dim3((unsigned)grid), dim3(kRowThreads), 0, st, 1, a));
  launch_counter().n++;
  return LRSA_OK;
}

// ---- reading the list back ----
struct StoreReadArgs {
  const void *k_list, *v_list;
  const float *k_scale, *v_scale;
  float *k, *v;          // [BH][n][d]
  int n, K, Kp, rows_list, block;   // n = kept rows
};

// A thread takes 16 channels of a kept row (bound by the fp32 rows it writes).
template <int D, int T>
__global__ void __launch_bounds__(256) store_read_kernel(const StoreReadArgs a) {
  constexpr int CPR = D / 16;
  const int bh = blockIdx.y, r = blockIdx.x * (256 / CPR) + threadIdx.x / CPR, ch = threadIdx.x % CPR;
  const bool is_v = blockIdx.z;
  wait_for_front();
  if (r >= a.n) return;
  const size_t row = (size_t)bh * a.rows_list + (size_t)(r / a.K) * a.Kp + r % a.K;
  float4* out = reinterpret_cast<float4*>((is_v ? a.v : a.k) + ((size_t)bh * a.n + r) * D + ch * 16);
  const void* list = is_v ? a.v_list : a.k_list;
  float x[16];
  if constexpr (T == LRSA_LIST_BF16) {
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(list) + row * D + ch * 16);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint4 u = src[h];
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) { x[8 * h + 2 * e] = __uint_as_float(w[e] << 16); x[8 * h + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
    }
  } else {
    const float scale = (is_v ? a.v_scale : a.k_scale)[row / a.block];
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(list) + row * D + ch * 16);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint32_t c = w[e / 4] >> (8 * (e % 4)) & 0xffu;
      x[e] = scale * (T == LRSA_LIST_INT8 ? (float)(int8_t)c
                                          : __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)c, __NV_E4M3))));
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
}

// ---- decode attention ----
struct StoreDecodeArgs {
  const __nv_bfloat16 *q, *k_recent, *v_recent;
  const unsigned char *k_list, *v_list;
  const float *k_scale, *v_scale;
  float* part;          // [BHkv][n_group][G][D + 2]: unnormalised output, maximum (log2 domain), sum
  __nv_bfloat16* o;     // [B][Hq][D]
  float* lse;           // [B][Hq], optional
  float* weight;        // [BHkv][2L], receives the weights of the ring's keys; null: not kept
  float* scores;        // [BHkv][2L][Gp]: the ring's scores (log2 domain), when weight is not null
  int* status;
  int Hq, Hkv, G, Gp, L2, rows_list, recent, S;
  int K, Kp, gpw, n_groups, shift;      // 16-row groups per window and in all; log2 of the block
  int n_recent, n_front, ring0;         // recent keys: n_front sink rows, then the ring from ring row ring0 on (wrapping)
  int list_blocks, blocks, n_split, n_group;
  float scale_log2;
};

__device__ __forceinline__ uint2 ld_stream8(const void* p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ void mma_16816_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                              uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Four codes as two pairs of halves (exact): bytes 0, 1 and bytes 2, 3.  An int8 code is offset to 0 ... 255 and put behind
// the exponent byte of 1024, where a half counts in ones.
template <int T>
__device__ __forceinline__ void widen(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (T == LRSA_LIST_E4M3) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(w));
  } else {
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    asm("sub.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));   // 1152 = 1024 + 128
    asm("sub.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
  }
}

// Grid (n_group * n_split, BHkv), clusters of n_split CTAs: the plan, the lanes' places and the merge are those of
// decode_kernel (lrsa_infer.cu).  The work is the transfer of the rows, one byte an element in the list and two in the recent
// rows, so a warp takes 8 KB at a time in either: 256 / d groups of sixteen list rows, or half as many of recent rows,
// loaded straight into the registers in which the warp-level products want them.
//   List.  A code is widened to a half (exact) and multiplied as such.  Q is brought into the range of halves by a power of
//     two per head (exact but for elements below 2^-28 of the head's largest).  The K scale of a group multiplies its scores.
//     The V scale enters the exponent, p' = 2^(s + log2(scale) - m' + 7), with a running maximum m' of that sum: what is rounded
//     to a half is at most 2^15 and 2^7 or more for the key that counts most, whatever the scales are, so a half's
//     smallest step is 2^-31 of it; O is in units of 2^(m' - 7).  The sum of the weights has its own maximum m and is kept in fp32.
//   Recent rows.  bf16 products with the bf16 Q, scale 1.
// The maxima are raised only when they grew by more than 2^8 (then O is rescaled).  With `weight` the ring's scores are
// stored, and when the cluster has its maximum and sum, each CTA adds exp2(score - lse) over the heads to the weights of
// the keys that were its own: one owner per key, no atomics.  Several clusters per head: store_weight_kernel does it.
template <int D, int NH, int T>
__global__ void __launch_bounds__(dec_max_warps(NH) * 32, 1) store_decode_kernel(const __grid_constant__ StoreDecodeArgs a) {
  constexpr bool k8 = T != LRSA_LIST_BF16;
  constexpr int UR = 128 / D;               // 16-key groups per block of recent rows
  constexpr int UL = k8 ? 256 / D : UR;     // of list rows
  constexpr int KC = D / 32;                // 16-byte chunks of a bf16 row per lane
  constexpr int KC8 = D / 64;               // of an 8-bit row
  constexpr int VC = D / 64;                // 16-byte chunks of V per lane, bf16
  constexpr int MT = D / 16;                // channel tiles of the output: tile f holds channels g*D/8 + 2f, + 1
  constexpr int kSlots = dec_max_warps(NH) / 2;
  constexpr float kLift = 7.f;              // 8 + 7 < 16: no half overflows between two raises of the maxima
  __shared__ __align__(16) float sm_o[kSlots][8][D + 4];
  __shared__ float sm_m[kSlots][8], sm_l[kSlots][8], sm_r[kSlots][8];
  __shared__ __align__(16) uint4 sm_q[NH][KC][32];                    // bf16
  __shared__ __align__(16) uint4 sm_h[k8 ? NH : 1][k8 ? 2 * KC8 : 1][32];   // halves
  __shared__ float sm_qs[8 * NH];                                     // what the halves are multiplied by
  __shared__ float fin_o[8][D], fin_m[8], fin_l[8], fin_r[8];         // the CTA's result, read by the cluster
  __shared__ float sm_lse[8 * NH];                                    // of the pass, in the log2 domain
  const int bh = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int nw = blockDim.x >> 5, g = lane >> 2, t = lane & 3;
  const int b = bh / a.Hkv, hkv = bh % a.Hkv;
  const unsigned char* kl = a.k_list + (size_t)bh * a.rows_list * (k8 ? D : 2 * D);
  const unsigned char* vl = a.v_list + (size_t)bh * a.rows_list * (k8 ? D : 2 * D);
  const unsigned char* kr = reinterpret_cast<const unsigned char*>(a.k_recent) + (size_t)bh * a.recent * (D * 2);
  const unsigned char* vr = reinterpret_cast<const unsigned char*>(a.v_recent) + (size_t)bh * a.recent * (D * 2);
  const float* ks = a.k_scale + (size_t)bh * (a.rows_list >> a.shift);
  const float* vs = a.v_scale + (size_t)bh * (a.rows_list >> a.shift);
  // byte offset of recent key `key`'s row; beyond the end: the last one's (its probability is zero)
  auto recent_row = [&](int key) {
    key = min(key, a.n_recent - 1);
    int r = key;
    if (key >= a.n_front) {
      r = key - a.n_front + a.ring0;
      if (r >= a.L2) r -= a.L2;
      r += a.S;
    }
    return (size_t)r * (D * 2);
  };
  // first row and visible rows of 16-row group `gi` of the list
  auto group_row = [&](int gi, int& n) {
    const int w = gi / a.gpw, j = (gi - w * a.gpw) * 16;
    n = gi < a.n_groups ? min(16, a.K - j) : 0;
    return gi < a.n_groups ? w * a.Kp + j : 0;
  };
  const int nx = a.n_split * a.n_group;
  const int blk0 = (int)((long long)a.blocks * blockIdx.x / nx), blk1 = (int)((long long)a.blocks * (blockIdx.x + 1) / nx);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0 && bh == 0 && tid == 0) *a.status = 0;

  for (int g0 = 0; g0 < a.G; g0 += 8 * NH) {
    __syncthreads();
    // Q of the pass as the B operand: chunk t + 4j of a lane's head, as it takes the chunks of every key row
    for (int hd = warp; hd < 8 * NH; hd += nw) {
      constexpr int PL = D / 32;   // channels per lane
      const int c0 = lane * PL, li = (hd & 7) * 4;
      __nv_bfloat16 x[PL];
#pragma unroll
      for (int e = 0; e < PL; ++e)
        x[e] = g0 + hd < a.G ? a.q[((size_t)b * a.Hq + hkv * a.G + g0 + hd) * D + c0 + e] : __float2bfloat16(0.f);
      __nv_bfloat16* qb = reinterpret_cast<__nv_bfloat16*>(&sm_q[hd >> 3][c0 / 8 / 4][li + c0 / 8 % 4]) + c0 % 8;
#pragma unroll
      for (int e = 0; e < PL; ++e) qb[e] = x[e];
      if constexpr (k8) {
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < PL; ++e) most = max(most, (uint32_t)__bfloat16_as_ushort(x[e]) & 0x7fffu);
        most = __reduce_max_sync(0xffffffffu, most);
        // exponent of the largest element to 14; infinities, NaN and zero stay what they are
        const int e8 = (int)(most >> 7);
        const int up = most == 0 || most >= 0x7f80u ? 0 : 14 - (max(e8, 1) - 127);
        const float f1 = exp2f((float)(up / 2)), f2 = exp2f((float)(up - up / 2));   // 2^up may exceed the range
        __half* qh = reinterpret_cast<__half*>(&sm_h[hd >> 3][c0 / 64 * 2 + c0 % 16 / 8][li + c0 / 16 % 4]) + c0 % 8;
#pragma unroll
        for (int e = 0; e < PL; ++e) qh[e] = __float2half(__bfloat162float(x[e]) * f1 * f2);
        if (lane == 0) sm_qs[hd] = exp2f((float)(-up));
      }
    }
    __syncthreads();
    float o[NH][MT][4];         // tile f: channels g*D/8 + 2f, + 1 of heads 2t, 2t + 1
    float m[NH][2], l[NH][2];   // heads 2t, 2t + 1: maximum of the scores (the warp's), sum (this lane's keys)
    float r[NH][2];             // reference of O: maximum of score + log2(V scale); O is in units of 2^(r - kLift)
#pragma unroll
    for (int h = 0; h < NH; ++h) {
#pragma unroll
      for (int e = 0; e < 2; ++e) { m[h][e] = r[h][e] = -INFINITY; l[h][e] = 0.f; }
#pragma unroll
      for (int i = 0; i < MT; ++i) o[h][i][0] = o[h][i][1] = o[h][i][2] = o[h][i][3] = 0.f;
    }
    // raises the references of head group h where a score (mx) or a score with its scale (mr) has outgrown them
    auto raise = [&](int h, float (&mx)[2], float (&mr)[2]) {
      if (__any_sync(0xffffffffu, mx[0] > m[h][0] + 8.f || mx[1] > m[h][1] + 8.f || mr[0] > r[h][0] + 8.f || mr[1] > r[h][1] + 8.f)) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) {
            mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], x));
            mr[e] = fmaxf(mr[e], __shfl_xor_sync(0xffffffffu, mr[e], x));
          }
          const float mn = fmaxf(m[h][e], mx[e]), rn = fmaxf(r[h][e], mr[e]);   // -inf while every score has been
          l[h][e] *= m[h][e] == -INFINITY ? 0.f : exp2f(m[h][e] - mn);
          const float f = r[h][e] == -INFINITY ? 0.f : exp2f(r[h][e] - rn);
          m[h][e] = mn;
          r[h][e] = rn;
#pragma unroll
          for (int i = 0; i < MT; ++i) { o[h][i][e] *= f; o[h][i][e + 2] *= f; }
        }
      }
    };
    int blk = blk0 + warp;
    if constexpr (k8) {
      for (; blk < min(blk1, a.list_blocks); blk += nw) {
        uint4 kq[UL][2][KC8];
        uint32_t vq[UL][4][D / 32];   // D / 8 codes of a V row
        int nvis[UL];
        float fk[UL], lv[UL];
#pragma unroll
        for (int u = 0; u < UL; ++u) {
          const int row = group_row(blk * UL + u, nvis[u]);
          fk[u] = ks[row >> a.shift];
          lv[u] = vs[row >> a.shift];
          const unsigned char* p = kl + (size_t)row * D;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < KC8; ++j) kq[u][i][j] = ld_stream(p + (g + 8 * i) * D + (t + 4 * j) * 16);
          p = vl + (size_t)row * D;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const unsigned char* pv = p + (2 * t + (i & 1) + 8 * (i >> 1)) * D + g * (D / 8);
            if constexpr (D == 128) {
              const uint4 v = ld_stream(pv);
              vq[u][i][0] = v.x; vq[u][i][1] = v.y; vq[u][i][2] = v.z; vq[u][i][3] = v.w;
            } else {
              const uint2 v = ld_stream8(pv);
              vq[u][i][0] = v.x; vq[u][i][1] = v.y;
            }
          }
        }
#pragma unroll
        for (int u = 0; u < UL; ++u) lv[u] = __log2f(lv[u]);
        float s[NH][UL][4];
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int u = 0; u < UL; ++u) s[h][u][0] = s[h][u][1] = s[h][u][2] = s[h][u][3] = 0.f;
#pragma unroll
        for (int j = 0; j < KC8; ++j)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint4 q[NH];
#pragma unroll
            for (int h = 0; h < NH; ++h) q[h] = sm_h[h][2 * j + c][lane];
#pragma unroll
            for (int u = 0; u < UL; ++u) {
              const uint32_t w0 = c ? kq[u][0][j].z : kq[u][0][j].x, w1 = c ? kq[u][1][j].z : kq[u][1][j].x;
              const uint32_t w2 = c ? kq[u][0][j].w : kq[u][0][j].y, w3 = c ? kq[u][1][j].w : kq[u][1][j].y;
              uint32_t a0, a1, a2, a3;
              widen<T>(w0, a0, a2);
              widen<T>(w1, a1, a3);
#pragma unroll
              for (int h = 0; h < NH; ++h) mma_16816_f16(s[h][u], a0, a1, a2, a3, q[h].x, q[h].y);
              widen<T>(w2, a0, a2);
              widen<T>(w3, a1, a3);
#pragma unroll
              for (int h = 0; h < NH; ++h) mma_16816_f16(s[h][u], a0, a1, a2, a3, q[h].z, q[h].w);
            }
          }
        uint32_t pb[NH][UL][2];
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          const float c0 = sm_qs[8 * h + 2 * t] * a.scale_log2, c1 = sm_qs[8 * h + 2 * t + 1] * a.scale_log2;
          float mx[2] = {-INFINITY, -INFINITY}, mr[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int u = 0; u < UL; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              s[h][u][e] = g + 8 * (e >> 1) < nvis[u] ? s[h][u][e] * (fk[u] * (e & 1 ? c1 : c0)) : -INFINITY;
              mx[e & 1] = fmaxf(mx[e & 1], s[h][u][e]);
              mr[e & 1] = fmaxf(mr[e & 1], s[h][u][e] + lv[u]);
            }
          raise(h, mx, mr);
          const float rm[2] = {m[h][0] == -INFINITY ? 0.f : m[h][0], m[h][1] == -INFINITY ? 0.f : m[h][1]};
          const float rr[2] = {r[h][0] == -INFINITY ? 0.f : r[h][0] - kLift, r[h][1] == -INFINITY ? 0.f : r[h][1] - kLift};
#pragma unroll
          for (int u = 0; u < UL; ++u) {
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              l[h][e & 1] += ptx::ex2(s[h][u][e] - rm[e & 1]);
              p[e] = ptx::ex2(s[h][u][e] + (lv[u] - rr[e & 1]));
            }
            pb[h][u][0] = transpose_8x8(pack_f16(p[0], p[1]));
            pb[h][u][1] = transpose_8x8(pack_f16(p[2], p[3]));
          }
        }
#pragma unroll
        for (int u = 0; u < UL; ++u)
#pragma unroll
          for (int i = 0; i < D / 32; ++i) {   // four channels: tiles 2i, 2i + 1
            uint32_t x[2][4];                  // [rows 2t, 2t+1 | + 8][channel]: pairs of keys
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              widen<T>(__byte_perm(vq[u][2 * z][i], vq[u][2 * z + 1][i], 0x5140), x[z][0], x[z][1]);
              widen<T>(__byte_perm(vq[u][2 * z][i], vq[u][2 * z + 1][i], 0x7362), x[z][2], x[z][3]);
            }
#pragma unroll
            for (int h = 0; h < NH; ++h) {
              mma_16816_f16(o[h][2 * i], x[0][0], x[0][1], x[1][0], x[1][1], pb[h][u][0], pb[h][u][1]);
              mma_16816_f16(o[h][2 * i + 1], x[0][2], x[0][3], x[1][2], x[1][3], pb[h][u][0], pb[h][u][1]);
            }
          }
      }
    }
    for (; blk < blk1; blk += nw) {
      // bf16: recent rows, or rows of a bf16 list
      const bool in_list = !k8 && blk < a.list_blocks;
      uint4 kq[UR][2][KC], vq[UR][4][VC];
      int nvis[UR], key0[UR];
#pragma unroll
      for (int u = 0; u < UR; ++u) {
        int row = 0;
        if (in_list) {
          row = group_row(blk * UR + u, nvis[u]);
        } else {
          key0[u] = ((blk - a.list_blocks) * UR + u) * 16;
          nvis[u] = a.n_recent - key0[u];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const unsigned char* p = in_list ? kl + (size_t)(row + g + 8 * i) * (D * 2) : kr + recent_row(key0[u] + g + 8 * i);
#pragma unroll
          for (int j = 0; j < KC; ++j) kq[u][i][j] = ld_stream(p + (t + 4 * j) * 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 2 * t + (i & 1) + 8 * (i >> 1);
          const unsigned char* p = in_list ? vl + (size_t)(row + k) * (D * 2) : vr + recent_row(key0[u] + k);
#pragma unroll
          for (int j = 0; j < VC; ++j) vq[u][i][j] = ld_stream(p + g * (D / 4) + j * 16);
        }
      }
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        float s[UR][4], mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int u = 0; u < UR; ++u) {
          s[u][0] = s[u][1] = s[u][2] = s[u][3] = 0.f;
#pragma unroll
          for (int j = 0; j < KC; ++j) {
            const uint4 q = sm_q[h][j][lane];
            mma_16816(s[u], kq[u][0][j].x, kq[u][1][j].x, kq[u][0][j].y, kq[u][1][j].y, q.x, q.y);
            mma_16816(s[u], kq[u][0][j].z, kq[u][1][j].z, kq[u][0][j].w, kq[u][1][j].w, q.z, q.w);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[u][e] = g + 8 * (e >> 1) < nvis[u] ? s[u][e] * a.scale_log2 : -INFINITY;
            mx[e & 1] = fmaxf(mx[e & 1], s[u][e]);
          }
          if (a.weight && !in_list) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int key = key0[u] + g + 8 * i;
              if (key >= a.n_front && key < a.n_recent && g0 + 8 * h + 2 * t < a.Gp)
                *reinterpret_cast<float2*>(a.scores + ((size_t)bh * a.L2 + key - a.n_front) * a.Gp + g0 + 8 * h + 2 * t) =
                    make_float2(s[u][2 * i], s[u][2 * i + 1]);
            }
          }
        }
        float mr[2] = {mx[0], mx[1]};
        raise(h, mx, mr);
        const float rm[2] = {m[h][0] == -INFINITY ? 0.f : m[h][0], m[h][1] == -INFINITY ? 0.f : m[h][1]};
        const float rr[2] = {r[h][0] == -INFINITY ? 0.f : r[h][0] - kLift, r[h][1] == -INFINITY ? 0.f : r[h][1] - kLift};
#pragma unroll
        for (int u = 0; u < UR; ++u) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            l[h][e & 1] += ptx::ex2(s[u][e] - rm[e & 1]);
            p[e] = ptx::ex2(s[u][e] - rr[e & 1]);
          }
          const uint32_t b0 = transpose_8x8(ptx::pack_bf16(p[0], p[1])), b1 = transpose_8x8(ptx::pack_bf16(p[2], p[3]));
#pragma unroll
          for (int j = 0; j < VC; ++j)
#pragma unroll
            for (int f = 0; f < 4; ++f) {
              auto w = [&](int i) { return f == 0 ? vq[u][i][j].x : f == 1 ? vq[u][i][j].y : f == 2 ? vq[u][i][j].z : vq[u][i][j].w; };
              mma_16816(o[h][4 * j + f], __byte_perm(w(0), w(1), 0x5410), __byte_perm(w(0), w(1), 0x7632),
                        __byte_perm(w(2), w(3), 0x5410), __byte_perm(w(2), w(3), 0x7632), b0, b1);
            }
        }
      }
    }
    // Merge the warps: the upper half hands its state to the lower half, then all threads add what is left.
    const int half = nw / 2;
    const bool upper = warp >= half;
    const int slot = upper ? warp - half : warp;
    const int group = blockIdx.x / a.n_split, rank = blockIdx.x - group * a.n_split;
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      float lh[2], mh[2], rh[2];
      auto put = [&]() {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float* dst = sm_o[slot][2 * t + e] + g * (D / 8);
#pragma unroll
          for (int i = 0; i < MT; ++i) *reinterpret_cast<float2*>(dst + 2 * i) = make_float2(o[h][i][e], o[h][i][e + 2]);
          if (g == 0) { sm_m[slot][2 * t + e] = mh[e]; sm_l[slot][2 * t + e] = lh[e]; sm_r[slot][2 * t + e] = rh[e]; }
        }
      };
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        mh[e] = m[h][e];
        rh[e] = r[h][e] - kLift;
        lh[e] = l[h][e];
#pragma unroll
        for (int y = 4; y < 32; y <<= 1) lh[e] += __shfl_xor_sync(0xffffffffu, lh[e], y);
      }
      auto part_of = [](float from, float to) { return from == -INFINITY ? 0.f : exp2f(from - to); };
      __syncthreads();   // the buffer is free
      if (upper) put();
      __syncthreads();
      if (!upper) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float mo = sm_m[slot][2 * t + e], mn = fmaxf(mh[e], mo);
          const float ro = sm_r[slot][2 * t + e], rn = fmaxf(rh[e], ro);
          lh[e] = lh[e] * part_of(mh[e], mn) + sm_l[slot][2 * t + e] * part_of(mo, mn);
          const float f0 = part_of(rh[e], rn), f1 = part_of(ro, rn);
          mh[e] = mn;
          rh[e] = rn;
          const float* srcp = sm_o[slot][2 * t + e] + g * (D / 8);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const float2 v = *reinterpret_cast<const float2*>(srcp + 2 * i);
            o[h][i][e] = o[h][i][e] * f0 + v.x * f1;
            o[h][i][e + 2] = o[h][i][e + 2] * f0 + v.y * f1;
          }
        }
        __syncwarp();   // every lane has read the slot before it is overwritten
        put();
      }
      __syncthreads();
      const int ng = min(8, a.G - g0 - 8 * h);
      for (int i = tid; i < ng * D; i += blockDim.x) {
        const int hd = i / D, c = i % D;
        float M = -INFINITY, R = -INFINITY;
        for (int w = 0; w < half; ++w) { M = fmaxf(M, sm_m[w][hd]); R = fmaxf(R, sm_r[w][hd]); }
        float ov = 0.f, ls = 0.f;
        for (int w = 0; w < half; ++w) {
          ov = fmaf(sm_o[w][hd][c], part_of(sm_r[w][hd], R), ov);
          ls = fmaf(sm_l[w][hd], part_of(sm_m[w][hd], M), ls);
        }
        fin_o[hd][c] = ov;
        if (c == 0) { fin_m[hd] = M; fin_l[hd] = ls; fin_r[hd] = R; }
      }
      cluster_sync();
      // the CTAs of the cluster share the elements of the output; every CTA wants the log-sums of all heads for its weights
      auto total = [&](int hd, float& M, float& ls) {
        M = -INFINITY; ls = 0.f;
#pragma unroll 4
        for (int k = 0; k < a.n_split; ++k) M = fmaxf(M, ld_cluster(&fin_m[hd], k));
#pragma unroll 4
        for (int k = 0; k < a.n_split; ++k) ls = fmaf(ld_cluster(&fin_l[hd], k), M == -INFINITY ? 0.f : exp2f(ld_cluster(&fin_m[hd], k) - M), ls);
      };
      for (int i = rank * blockDim.x + tid; i < ng * D; i += a.n_split * blockDim.x) {
        const int hd = i / D, c = i % D;
        float M, ls, R = -INFINITY, ov = 0.f;
        total(hd, M, ls);
#pragma unroll 4
        for (int k = 0; k < a.n_split; ++k) R = fmaxf(R, ld_cluster(&fin_r[hd], k));
#pragma unroll 4
        for (int k = 0; k < a.n_split; ++k) ov = fmaf(ld_cluster(&fin_o[hd][c], k), R == -INFINITY ? 0.f : exp2f(ld_cluster(&fin_r[hd], k) - R), ov);
        // O in units of 2^M: R - M is the scale of the V rows that carry the weight
        ov *= R == -INFINITY ? 0.f : exp2f(R - M);
        if (a.n_group > 1) {
          float* dst = a.part + (((size_t)bh * a.n_group + group) * a.G + g0 + 8 * h + hd) * (D + 2);
          dst[c] = ov;
          if (c == 0) { dst[D] = M; dst[D + 1] = ls; }
          continue;
        }
        const size_t head = (size_t)b * a.Hq + hkv * a.G + g0 + 8 * h + hd;
        a.o[head * D + c] = __float2bfloat16(ov / ls);
        if (c == 0 && a.lse) a.lse[head] = (M + log2f(ls)) * 0.6931471805599453f;
      }
      if (a.weight && a.n_group == 1 && tid < ng) {
        float M, ls;
        total(tid, M, ls);
        sm_lse[8 * h + tid] = M + log2f(ls);
      }
      cluster_sync();   // the other CTAs have read this one's result: it may be overwritten, or the CTA may leave
    }
    if (a.weight && a.n_group == 1) {
      // (the barriers above have ordered the scores of the CTA's warps before these reads)
      const int ng = min(8 * NH, a.G - g0);
      const int k0 = max(a.n_front, (max(blk0, a.list_blocks) - a.list_blocks) * UR * 16), k1 = min(a.n_recent, (blk1 - a.list_blocks) * UR * 16);
      for (int key = k0 + tid; key < k1; key += blockDim.x) {
        const float* sc = a.scores + ((size_t)bh * a.L2 + key - a.n_front) * a.Gp + g0;
        float sum = 0.f;
        for (int hd = 0; hd < ng; ++hd) sum += ptx::ex2(sc[hd] - sm_lse[hd]);
        int at = key - a.n_front + a.ring0;
        if (at >= a.L2) at -= a.L2;
        a.weight[(size_t)bh * a.L2 + at] += sum;
      }
    }
  }
}

// The weights where a head has several clusters: log-sums are the merge kernel's.  A thread takes a key.
__global__ void __launch_bounds__(128) store_weight_kernel(const StoreDecodeArgs a, const float* lse) {
  const int bh = blockIdx.y, key = a.n_front + blockIdx.x * 128 + threadIdx.x;
  wait_for_front();
  if (key >= a.n_recent) return;
  const float* sc = a.scores + ((size_t)bh * a.L2 + key - a.n_front) * a.Gp;
  const float* ls = lse + (size_t)(bh / a.Hkv) * a.Hq + (bh % a.Hkv) * a.G;
  float sum = 0.f;
  for (int hd = 0; hd < a.G; ++hd) sum += ptx::ex2(sc[hd] - ls[hd] * 1.4426950408889634f);
  int at = key - a.n_front + a.ring0;
  if (at >= a.L2) at -= a.L2;
  a.weight[(size_t)bh * a.L2 + at] += sum;
}

template <int D, int NH, int T>
cudaError_t launch_store_decode_t(StoreDecodeArgs& a, const DecodePlan& pl, int BHkv, cudaStream_t st) {
  auto kern = store_decode_kernel<D, NH, T>;
  if (pl.splits > 8) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return launch_dependent(kern, dim3(pl.splits * pl.groups, BHkv), dim3(pl.warps * 32), 0, st, pl.splits, a);
}

template <int T>
cudaError_t launch_store_decode(const Geom& g, StoreDecodeArgs& a, const DecodePlan& pl, cudaStream_t st) {
  const int BHkv = g.B * g.Hkv;
  a.n_split = pl.splits; a.n_group = pl.groups; a.blocks = pl.blocks;
  if (g.d == 128) return pl.nh == 1 ? launch_store_decode_t<128, 1, T>(a, pl, BHkv, st) : launch_store_decode_t<128, 2, T>(a, pl, BHkv, st);
  return pl.nh == 1 ? launch_store_decode_t<64, 1, T>(a, pl, BHkv, st) : launch_store_decode_t<64, 2, T>(a, pl, BHkv, st);
}

// Parts of the workspace.
struct StoreWs { size_t part, lse, scores, total; };
StoreWs store_ws(const Geom& g, const StoreGeom& o) {
  StoreWs w;
  const size_t BH = (size_t)g.B * g.Hkv;
  size_t off = sizeof(WsHeader);
  // several clusters for a head only below 592 CTAs of 16 warps (deal_blocks)
  w.part = off; off += align_up(BH <= 4 * (size_t)kSms * 4 ? BH * kDecMaxGroups * g.G * (g.d + 2) * sizeof(float) : 0, 256);
  w.lse = off; off += align_up((size_t)g.B * g.Hq * sizeof(float), 256);
  w.scores = off; off += o.by_weight ? align_up(BH * 2 * g.L * ((g.G + 7) / 8 * 8) * sizeof(float), 256) : 0;
  w.total = off;
  return w;
}

size_t store_ws_bytes(const Geom& g, const StoreGeom& o) {
  size_t need = store_ws(g, o).total;
  if (!o.by_weight) {   // scoring scratch of the windows of a whole prompt
    Geom all = g;
    all.W = o.Wcap + 1 > 2 ? o.Wcap + 1 : 2; all.Wsel = all.W - 1;
    const size_t s = score_select_ws_bytes(all);
    if (s > need) need = s;
  }
  return need;
}

}  // namespace
}  // namespace lrsa

using namespace lrsa;

extern "C" {

int lrsa_store_shape(const lrsa_params_t* params, const lrsa_store_t* store, int32_t* w_cap, int32_t* rows_per_window,
                     size_t* workspace_bytes) {
  Geom g;
  StoreGeom o;
  const int rc = make_store_geom(params, store, &g, &o);
  if (rc != LRSA_OK) return rc;
  if (w_cap) *w_cap = o.Wcap;
  if (rows_per_window) *rows_per_window = o.Kp;
  if (workspace_bytes) *workspace_bytes = store_ws_bytes(g, o);
  return LRSA_OK;
}

int lrsa_store_append(const lrsa_params_t* params, const lrsa_store_t* store, const void* k_new, const void* v_new,
                      const float* w_new, int32_t n_prev, int32_t n_new, void* workspace, size_t workspace_bytes,
                      void* cuda_stream) {
  NvtxRange nvtx_range("lrsa_store_append");
  launch_counter().n = 0;
  Geom g;
  StoreGeom o;
  int rc = make_store_geom(params, store, &g, &o);
  if (rc != LRSA_OK) return rc;
  if (!k_new || !v_new || !workspace || n_prev < 0 || n_new < 1 || (long long)n_prev + n_new > g.N) return LRSA_ERR_INVALID_ARG;
  if (mis(workspace, 256) || mis(k_new, 16) || mis(v_new, 16) || mis(w_new, 4)) return LRSA_ERR_INVALID_ARG;
  if (w_new && !o.by_weight) return LRSA_ERR_INVALID_ARG;
  rc = check_store(store, o);
  if (rc != LRSA_OK) return rc;
  if (workspace_bytes < store_ws_bytes(g, o)) return LRSA_ERR_WORKSPACE_TOO_SMALL;
  const int end = n_prev + n_new;
  // Windows compressed by this call: cut by weight, a window that holds tokens of this call needs their weights.
  const int c_end = end > g.S ? (end - 1 - g.S) / g.L : 0, c_prev = n_prev > g.S ? (n_prev - 1 - g.S) / g.L : 0;
  if (o.by_weight && !w_new && c_end >= 2 && c_end > c_prev && (long long)g.S + (c_end - 1LL) * g.L > n_prev) return LRSA_ERR_INVALID_ARG;
  auto st = static_cast<cudaStream_t>(cuda_stream);
  const int BH = g.B * g.Hkv;
  StoreRows rows = {};
  rows.k_new = static_cast<const __nv_bfloat16*>(k_new); rows.v_new = static_cast<const __nv_bfloat16*>(v_new); rows.w_new = w_new;
  rows.k_recent = static_cast<__nv_bfloat16*>(store->k_recent); rows.v_recent = static_cast<__nv_bfloat16*>(store->v_recent);
  rows.weight = o.by_weight ? store->weight : nullptr;
  rows.k_list = store->k_list; rows.v_list = store->v_list; rows.k_scale = store->k_scale; rows.v_scale = store->v_scale;
  rows.idx = store->idx;
  rows.n_new = n_new; rows.p_first = n_prev; rows.S = g.S; rows.L = g.L; rows.K = g.K; rows.Kp = o.Kp; rows.Wcap = o.Wcap;
  rows.rows_list = o.rows_list; rows.recent = o.recent; rows.block = o.block;
  // The status word is cleared by the first kernel of the call (a memset in front of a scoring kernel that cannot).
  int* status = &static_cast<WsHeader*>(workspace)->status;
  bool cleared = false;
  // Selects windows [w0, + n): out of the ring (one window), or out of the new tokens.
  auto select = [&](int w0, int n, bool ring) -> int {
    const int tok0 = ring ? (w0 % 2) * g.L : g.S + w0 * g.L - n_prev;
    if (o.by_weight) {
      WeightSelectArgs a = {};
      a.weight = ring ? store->weight : w_new;
      a.row = ring ? 2 * g.L : n_new;
      a.idx = store->idx; a.status = cleared ? nullptr : status; a.L = g.L; a.K = g.K; a.Wtot = o.Wcap; a.n = 1;
      if ((long long)BH * n > 0x7fffffffLL) return LRSA_ERR_UNSUPPORTED;
      a.item0[1] = BH * n; a.windows[0] = n; a.first[0] = tok0; a.woff[0] = w0; a.emit0[0] = g.S + w0 * g.L;
      cleared = true;
      return launch_weight_select(a, st);
    }
    Geom s = g;
    s.S = 0; s.T = 0; s.W = n + 1; s.C = n + 1; s.Wsel = n; s.Wtot = o.Wcap; s.woff = w0; s.emit_off = g.S + w0 * g.L;
    s.N = s.Nrow = ring ? o.recent : n_new;
    s.tok0 = ring ? g.S + tok0 : tok0;
    s.win_stride = ring && w0 % 2 ? -g.L : g.L;
    const bool self = !cleared && score_select_clears_status(s);
    if (!cleared && !self) {
      LRSA_CUDA_CHECK(cudaMemsetAsync(workspace, 0, sizeof(WsHeader), st));
      launch_counter().n++;
    }
    cleared = true;
    return launch_score_select(&s, 1, ring ? rows.k_recent : rows.k_new, ring ? rows.v_recent : rows.v_new, store->idx, nullptr, workspace, st, self);
  };
  auto move_rows = [&]() -> int {
    if (rows.n_sink + rows.n_ins + rows.n_win == 0) return LRSA_OK;
    rows.status = cleared ? nullptr : status;
    cleared = true;
    return launch_store_rows(rows, o, BH, g.d, st);
  };
  int pos = n_prev;                                     // tokens before it are in the store
  int c = pos > g.S ? (pos - g.S + g.L - 1) / g.L : 0;  // next chunk whose first token has not arrived yet
  if (c < 2) c = 2;
  // Chunk start after chunk start while the window c-2 that leaves the ring holds tokens of earlier calls (at most two): the
  // tokens up to it enter the ring, the window is cut, its kept rows join the list before its half is overwritten.
  for (; (long long)g.S + (long long)c * g.L < end && g.S + (c - 2) * g.L < n_prev; ++c) {
    const int w = c - 2;
    rows.p0 = pos; rows.n_ins = g.S + c * g.L - pos; rows.n_win = 0;
    if ((rc = move_rows()) != LRSA_OK) return rc;
    if ((rc = select(w, 1, true)) != LRSA_OK) return rc;
    rows.n_ins = 0; rows.w0 = w; rows.n_win = 1; rows.from_ring = 1;
    if ((rc = move_rows()) != LRSA_OK) return rc;
    pos = g.S + c * g.L;
  }
  rows.n_win = 0;
  rows.p0 = pos; rows.n_ins = end - pos;
  if ((long long)g.S + (long long)c * g.L < end) {
    // Windows c-2 .. c_last-2 lie in the new tokens as a whole: one selection for all of them, then one launch for their
    // kept rows, the sinks and the tokens that stay in the ring.
    const int w0 = c - 2, nw = (end - 1 - g.S) / g.L - c + 1;
    if ((rc = select(w0, nw, false)) != LRSA_OK) return rc;
    rows.n_sink = pos < g.S ? g.S - pos : 0;
    rows.p0 = end - 2 * g.L > pos ? end - 2 * g.L : pos;
    rows.n_ins = end - rows.p0;
    rows.w0 = w0; rows.n_win = nw; rows.from_ring = 0;
  }
  return move_rows();
}

int lrsa_store_decode(const lrsa_params_t* params, const lrsa_store_t* store, const void* q, int32_t n_tokens, void* out_o,
                      float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  NvtxRange nvtx_range("lrsa_store_decode");
  launch_counter().n = 0;
  Geom g;
  StoreGeom o;
  int rc = make_store_geom(params, store, &g, &o);
  if (rc != LRSA_OK) return rc;
  if (!q || !out_o || !workspace || n_tokens < 1 || n_tokens > g.N) return LRSA_ERR_INVALID_ARG;
  if (mis(workspace, 256) || mis(q, 16) || mis(out_o, 16) || mis(lse, 4)) return LRSA_ERR_INVALID_ARG;
  rc = check_store(store, o);
  if (rc != LRSA_OK) return rc;
  if (workspace_bytes < store_ws_bytes(g, o)) return LRSA_ERR_WORKSPACE_TOO_SMALL;
  if ((long long)g.B * g.Hkv > 65535) return LRSA_ERR_UNSUPPORTED;   // grid rows
  auto st = static_cast<cudaStream_t>(cuda_stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  const StoreWs lay = store_ws(g, o);
  StoreDecodeArgs a = {};
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.k_recent = static_cast<const __nv_bfloat16*>(store->k_recent); a.v_recent = static_cast<const __nv_bfloat16*>(store->v_recent);
  a.k_list = static_cast<const unsigned char*>(store->k_list); a.v_list = static_cast<const unsigned char*>(store->v_list);
  a.k_scale = store->k_scale; a.v_scale = store->v_scale;
  a.part = reinterpret_cast<float*>(ws + lay.part);
  a.o = static_cast<__nv_bfloat16*>(out_o); a.lse = lse;
  a.weight = o.by_weight ? store->weight : nullptr;
  a.scores = reinterpret_cast<float*>(ws + lay.scores);
  a.status = &reinterpret_cast<WsHeader*>(ws)->status;
  a.Hq = g.Hq; a.Hkv = g.Hkv; a.G = g.G; a.Gp = (g.G + 7) / 8 * 8; a.L2 = 2 * g.L; a.rows_list = o.rows_list; a.recent = o.recent; a.S = g.S;
  a.K = g.K; a.Kp = o.Kp; a.gpw = (g.K + 15) / 16;
  while ((1 << a.shift) < o.block) ++a.shift;
  // the keys that the query at position t sees (Attn-Fill 1/2): a sink query its causal prefix; otherwise the kept rows of
  // windows 0..c-2, the sinks, and positions [S + (c-1)L, t] from the ring
  const int t = n_tokens - 1;
  if (t < g.S) {
    a.n_front = a.n_recent = t + 1;
  } else {
    const int c = (t - g.S) / g.L, nc = c >= 1 ? c - 1 : 0;
    a.n_groups = nc * a.gpw;
    a.n_front = g.S;
    a.n_recent = g.S + t - (g.S + nc * g.L) + 1;
    a.ring0 = (nc * g.L) % (2 * g.L);
  }
  a.scale_log2 = g.scale * 1.4426950408889634f;
  const int ul = o.type == LRSA_LIST_BF16 ? 128 / g.d : 256 / g.d, ur = 128 / g.d;
  a.list_blocks = (a.n_groups + ul - 1) / ul;
  const int blocks = a.list_blocks + (a.n_recent + 16 * ur - 1) / (16 * ur);
  DecodePlan pl = deal_blocks(g, blocks);
  auto launch = [&](const DecodePlan& p) {
    return o.type == LRSA_LIST_E4M3 ? launch_store_decode<LRSA_LIST_E4M3>(g, a, p, st)
           : o.type == LRSA_LIST_INT8 ? launch_store_decode<LRSA_LIST_INT8>(g, a, p, st)
                                      : launch_store_decode<LRSA_LIST_BF16>(g, a, p, st);
  };
  cudaError_t e = launch(pl);
  if (e != cudaSuccess && pl.splits > 8) {   // clusters of 16 are not portable: a part of a GPU may not have room for them
    (void)cudaGetLastError();
    pl = deal_blocks(g, blocks, 8);
    e = launch(pl);
  }
  LRSA_CUDA_CHECK(e);
  launch_counter().n++;
  if (pl.groups > 1) {
    float* ls = a.weight && !lse ? reinterpret_cast<float*>(ws + lay.lse) : lse;
    auto merge = g.d == 128 ? decode_merge_kernel<128, 1> : decode_merge_kernel<64, 1>;
    LRSA_CUDA_CHECK(launch_dependent(merge, dim3(g.B * g.Hq), dim3(g.d), 0, st, 1, (const float*)a.part, a.o, ls, g.Hq, g.Hkv, g.G, pl.groups));
    launch_counter().n++;
    if (a.weight && a.n_recent > a.n_front) {
      LRSA_CUDA_CHECK(launch_dependent(store_weight_kernel, dim3((a.n_recent - a.n_front + 127) / 128, g.B * g.Hkv), dim3(128), 0, st, 1, a, (const float*)ls));
      launch_counter().n++;
    }
  }
  return LRSA_OK;
}

int lrsa_store_rows(const lrsa_params_t* params, const lrsa_store_t* store, int32_t n_windows, float* k, float* v, void* cuda_stream) {
  NvtxRange nvtx_range("lrsa_store_rows");
  launch_counter().n = 0;
  Geom g;
  StoreGeom o;
  int rc = make_store_geom(params, store, &g, &o);
  if (rc != LRSA_OK) return rc;
  if (n_windows < 0 || n_windows > o.Wcap) return LRSA_ERR_INVALID_ARG;
  if (n_windows == 0) return LRSA_OK;
  if (!k || !v || mis(k, 16) || mis(v, 16)) return LRSA_ERR_INVALID_ARG;
  rc = check_store(store, o);
  if (rc != LRSA_OK) return rc;
  if ((long long)g.B * g.Hkv > 65535) return LRSA_ERR_UNSUPPORTED;   // grid rows
  StoreReadArgs a = {};
  a.k_list = store->k_list; a.v_list = store->v_list; a.k_scale = store->k_scale; a.v_scale = store->v_scale; a.k = k; a.v = v;
  a.n = n_windows * g.K; a.K = g.K; a.Kp = o.Kp; a.rows_list = o.rows_list; a.block = o.block;
  auto kern = g.d == 128 ? (o.type == LRSA_LIST_E4M3 ? store_read_kernel<128, LRSA_LIST_E4M3> : o.type == LRSA_LIST_INT8 ? store_read_kernel<128, LRSA_LIST_INT8> : store_read_kernel<128, LRSA_LIST_BF16>)
                         : (o.type == LRSA_LIST_E4M3 ? store_read_kernel<64, LRSA_LIST_E4M3> : o.type == LRSA_LIST_INT8 ? store_read_kernel<64, LRSA_LIST_INT8> : store_read_kernel<64, LRSA_LIST_BF16>);
  const int rpb = 256 / (g.d / 16);
  LRSA_CUDA_CHECK(launch_dependent(kern, dim3((unsigned)((a.n + rpb - 1) / rpb), g.B * g.Hkv, 2), dim3(256), 0,
                                   static_cast<cudaStream_t>(cuda_stream), 1, a));
  launch_counter().n++;
  return LRSA_OK;
}

}  // extern "C"
