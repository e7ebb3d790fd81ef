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
#include <limits.h>

#include <type_traits>

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
constexpr int kRowThreads = kSelThreads;

struct StoreRows {
  const __nv_bfloat16 *k_new, *v_new;   // [BH][n_new][d], token p at row p - p_first
  const float* w_new;                   // [BH][n_new] or null (zero)
  __nv_bfloat16 *k_recent, *v_recent;
  float* weight;                        // null: not kept
  void *k_list, *v_list;
  float *k_scale, *v_scale;
  int32_t* idx;                         // [BH][Wcap][K]
  int* status;                          // cleared when not null
  int n_new, p_first, S, L, K, Kp, Wcap, rows_list, recent, block;
  int n_sink, p0, n_ins;                // new tokens [p_first, + n_sink) and [p0, + n_ins) go to the recent rows
  int w0, n_win, ring_below;            // kept rows of windows [w0, + n_win): positions below ring_below are in the ring
  int BH, copy_blocks, list_blocks;     // thread blocks per (batch, KV head); store_cut_kernel: clusters that cut
  int lanes;                            // threads that share a block of the list: M 16-byte chunks each
  int split;                            // CTAs that share a window (store_cut_kernel)
};

// The least bf16 that is not below x (finite, positive); infinities and NaN stay.
__device__ __forceinline__ float scale_up(float x) {
  return x < INFINITY ? __uint_as_float((__float_as_uint(x) + 0xffffu) & 0xffff0000u) : x;
}
// value / scale as exactly as its code needs.  Value and scale have eight significant bits, a border between two codes at most
// eight: a quotient that is not on a border is at least 2^-16 (relative) away from it.  The product with the rounded
// reciprocal is within 2^-22 of the quotient, and rounded to 19 bits it is on the border exactly when the quotient is, and on its side
// otherwise.  (A division takes eight instructions more for every element.)
__device__ __forceinline__ float quotient(float x, float inv) {
  return __uint_as_float((__float_as_uint(x * inv) + 0x10u) & 0xffffffe0u);
}

// Token `item` of the copied ones into the recent rows: this thread's 16 bytes of K and of V, and its weight.
template <int D>
__device__ __forceinline__ void move_token(const StoreRows& a, int bh, int item, int ch) {
  constexpr int CPR = D / 8;                // 16-byte chunks per bf16 row
  if (item >= a.n_sink + a.n_ins) return;
  const int p = item < a.n_sink ? a.p_first + item : a.p0 + (item - a.n_sink);
  const int at = p < a.S ? p : a.S + (p - a.S) % (2 * a.L);
  const size_t src = ((size_t)bh * a.n_new + (p - a.p_first)) * CPR + ch, dst = ((size_t)bh * a.recent + at) * CPR + ch;
  const uint4 k = reinterpret_cast<const uint4*>(a.k_new)[src], v = reinterpret_cast<const uint4*>(a.v_new)[src];
  reinterpret_cast<uint4*>(a.k_recent)[dst] = k;
  reinterpret_cast<uint4*>(a.v_recent)[dst] = v;
  if (a.weight && ch == 0 && p >= a.S)
    a.weight[(size_t)bh * 2 * a.L + (at - a.S)] = a.w_new ? a.w_new[(size_t)bh * a.n_new + (p - a.p_first)] : 0.f;
}

// Blocks of kept rows of K (even items) or of V (odd) of window w into the list, each by a.lanes threads: block item / 2 of the
// window.  A row is read once (gathered by position, whole lines), held in registers while the block's largest magnitude
// is found, and written once.  s_max: a word for every warp.  All threads come here; there: this one has a block.
template <int D, int T, int M>
__device__ __forceinline__ void cut_block(const StoreRows& a, int bh, int w, int item, bool there, uint32_t* s_max) {
  constexpr int CPR = D / 8;
  const int tid = threadIdx.x, in = tid & (a.lanes - 1), j0 = there ? (item >> 1) * a.block : 0;
  const bool is_v = item & 1;
  const int32_t* idx = a.idx + ((size_t)bh * a.Wcap + w) * a.K;
  const __nv_bfloat16 *ring = (is_v ? a.v_recent : a.k_recent) + (size_t)bh * a.recent * D, *fresh = (is_v ? a.v_new : a.k_new) + (size_t)bh * a.n_new * D;
  // (all positions, then all rows: one behind the other they are M round trips, a 65K prompt of 8 heads with half of it kept 131 us
  // with its read-back instead of 108)
  int pos[M];
  uint4 x[M];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < M; ++i) pos[i] = __ldcg(idx + min(j0 + (i * a.lanes + in) / CPR, a.K - 1));   // (may be another CTA's of this kernel)
  const int ring0 = a.S + (w & 1) * a.L - (a.S + w * a.L);   // from a position to its ring row
#pragma unroll
  for (int i = 0; i < M; ++i) {
    // (clamped: where a scoring kernel's wait ran out, the positions are what was there before)
    const __nv_bfloat16* row = pos[i] < a.ring_below ? ring + (size_t)min((unsigned)(pos[i] + ring0), (unsigned)(a.recent - 1)) * D
                                                     : fresh + (size_t)min((unsigned)(pos[i] - a.p_first), (unsigned)(a.n_new - 1)) * D;
    x[i] = *reinterpret_cast<const uint4*>(row + (i * a.lanes + in) % CPR * 8);
  }
#pragma unroll
  for (int i = 0; i < M; ++i)
    if (j0 + (i * a.lanes + in) / CPR >= a.K) x[i] = make_uint4(0, 0, 0, 0);
  const size_t out_row = (size_t)bh * a.rows_list + (size_t)w * a.Kp + j0;
  if constexpr (T == LRSA_LIST_BF16) {
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(is_v ? a.v_list : a.k_list) + out_row * D;
#pragma unroll
    for (int i = 0; i < M; ++i)
      if (there) reinterpret_cast<uint4*>(dst)[i * a.lanes + in] = x[i];
  } else {
    // largest magnitude: bits without the sign are ordered like the values, infinities and NaN above all
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) most = max(most, max(u[e] & 0x7fffu, (u[e] >> 16) & 0x7fffu));
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if ((tid & 31) == 0) s_max[tid >> 5] = most;
    __syncthreads();
    if (!there) return;
    const int warps = a.lanes / 32;   // share the block (one to eight)
    most = __reduce_max_sync(0xffffffffu, s_max[tid / a.lanes * warps + (tid & (warps - 1))]);
    const float limit = T == LRSA_LIST_E4M3 ? 448.f : 127.f;
    const float scale = most ? fmaxf(scale_up(__fdiv_rn(__uint_as_float(most << 16), limit)), 1.17549435e-38f) : 1.f;
    if (in == 0) {
      // NaN in a block must not become the floor's 2^-126 (fmaxf drops it): its rows then all stand for NaN, as they do for an infinity
      const bool nan = most > 0x7f80u;
      (is_v ? a.v_scale : a.k_scale)[out_row / a.block] = nan ? NAN : scale;
    }
    unsigned char* dst = static_cast<unsigned char*>(is_v ? a.v_list : a.k_list) + out_row * D;
    const bool finite = most < 0x7f80u;
    const float inv = __frcp_rn(scale);
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const int c = i * a.lanes + in;
      const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
      uint32_t code[4];   // two codes each
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = quotient(__uint_as_float(u[e] << 16), inv), hi = quotient(__uint_as_float(u[e] & 0xffff0000u), inv);
        if constexpr (T == LRSA_LIST_E4M3) {
          code[e] = __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
        } else {   // rounded to whole numbers in the low bits of the sum
          code[e] = __byte_perm(__float_as_uint(lo + 12582912.f), __float_as_uint(hi + 12582912.f), 0x0040);
        }
      }
      const uint2 y = make_uint2(__byte_perm(code[0], code[1], 0x5410), __byte_perm(code[2], code[3], 0x5410));
      reinterpret_cast<uint2*>(dst)[c] = finite ? y : make_uint2(0, 0);
    }
  }
}

// Tokens into the recent rows, and kept rows into the list.  Bound by the rows it moves.
template <int D, int T, int M>
__global__ void __launch_bounds__(kRowThreads) store_rows_kernel(const __grid_constant__ StoreRows a) {
  constexpr int CPR = D / 8;
  __shared__ uint32_t s_max[kRowThreads / 32];
  const int tid = threadIdx.x, per = a.copy_blocks + a.list_blocks;
  const int bh = blockIdx.x / per, blk = blockIdx.x % per;
  wait_for_front();
  if (a.status && blockIdx.x == 0 && tid == 0) *a.status = 0;
  if (blk < a.copy_blocks) {
    move_token<D>(a, bh, blk * (blockDim.x / CPR) + tid / CPR, tid % CPR);
    return;
  }
  const int item = (blk - a.copy_blocks) * (blockDim.x / a.lanes) + tid / a.lanes, per_win = a.Kp / a.block * 2;
  const bool there = item < a.n_win * per_win;
  const int win = there ? item / per_win : 0;
  cut_block<D, T, M>(a, bh, a.w0 + win, item - win * per_win, there, s_max);
}

// By weight: selects windows [w0, + n_win) and moves their kept rows, a cluster of a.split CTAs a window (one selects, all move),
// beside the tokens that enter the recent rows.  A chain of latencies where windows are few (512 tokens, of which 128 are kept: weights
// 1.2 us, two digits 1.1, positions 0.7, cluster 0.5, rows and codes 2), the rows it moves where they are many.  (A 32K
// prompt and its read-back took 26.3 us as two kernels, one behind the other, and 23.9 in this form, a 9K prompt in five pieces
// 76 and 65; 19.8 and 56.5 since the loads of a thread go out together.)
template <int D, int T, int M>
__global__ void __launch_bounds__(kRowThreads) store_cut_kernel(const __grid_constant__ StoreRows a) {
  constexpr int CPR = D / 8;
  extern __shared__ __align__(16) uint32_t cut_key[];
  __shared__ SelectShared sh;
  __shared__ uint32_t s_max[kRowThreads / 32];
  const int tid = threadIdx.x, cluster = blockIdx.x / a.split, rank = blockIdx.x - cluster * a.split;
  const int n_cut = a.list_blocks;                       // clusters that cut: one for each window of each (batch, KV head)
  if (cluster < n_cut && rank == 0) select_clear(sh);
  wait_for_front();
  if (a.status && blockIdx.x == 0 && tid == 0) *a.status = 0;
  if (cluster >= n_cut) {
    const int blk = blockIdx.x - n_cut * a.split, bh = blk / a.copy_blocks;
    if (bh < a.BH) move_token<D>(a, bh, (blk - bh * a.copy_blocks) * (kRowThreads / CPR) + tid / CPR, tid % CPR);
    return;
  }
  const int bh = cluster / a.n_win, w = a.w0 + cluster - bh * a.n_win;
  if (rank == 0) {
    const int pos0 = a.S + w * a.L, in_ring = min(a.L, max(a.ring_below - pos0, 0));
    select_window_by_weight(sh, cut_key, a.L, a.K, a.w_new + (size_t)bh * a.n_new + (pos0 - a.p_first), a.weight + ((size_t)bh * 2 + w % 2) * a.L,
                            in_ring, a.idx + ((size_t)bh * a.Wcap + w) * a.K, pos0);
  }
  cluster_sync();   // the positions are in global memory for the CTAs of the cluster
  const int at_once = kRowThreads / a.lanes, per_win = a.Kp / a.block * 2;
  for (int i = rank * at_once; i < per_win; i += a.split * at_once) {
    const int item = i + tid / a.lanes;
    cut_block<D, T, M>(a, bh, w, item, item < per_win, s_max);
    __syncthreads();   // the words of the warps are written again
  }
}

template <int D, int T, int M>
int launch_rows_t(const StoreRows& a, int threads, long long grid, size_t smem, cudaStream_t st, bool cut) {
  auto rows = store_rows_kernel<D, T, M>;
  auto cuts = store_cut_kernel<D, T, M>;
  if (smem > kSelSmemFree) LRSA_CUDA_CHECK(cudaFuncSetAttribute(cuts, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelSmemMax));
  LRSA_CUDA_CHECK(cut ? launch_dependent(cuts, dim3((unsigned)grid), dim3(threads), smem, st, a.split, a)
                      : launch_dependent(rows, dim3((unsigned)grid), dim3(threads), 0, st, 1, a));
  launch_counter().n++;
  return LRSA_OK;
}

// `cut`: the windows are selected, by weight, in the same launch.
int launch_store_rows(StoreRows a, const StoreGeom& o, int BH, int d, cudaStream_t st, bool cut) {
  const int chunks = o.block * (d / 8);   // 16-byte chunks of a block: 128 ... 2048
  const bool wide = chunks > 4 * kRowThreads;
  a.lanes = chunks / (wide ? 8 : 4);      // 32 ... 256
  a.BH = BH;
  const int per_win = o.Kp / o.block * 2;
  long long grid;
  int threads = kRowThreads;
  if (cut) {
    // A CTA more for a window while its rows take several turns and the CTAs are few.  us of a prompt and its read-back, 1 | 2 | 4 | 8, * taken: 32K of
    // 28/4 heads, windows of 1024 28.1 | 21.0 | 20.1* | 23.8; 65K of 32/8, half kept 107.5* | 106.6 | 114 | 132; 60K of 8/8, d = 64, windows of
    // 2048 39.9 | 34.1* | 38.3 | 49; 30K of 28/4, windows of 4096 68.5 | 42.8 | 30.0 | 24.2*; 9K in five pieces 65 | 57* | 57 | 63.
    const int at_once = kRowThreads / a.lanes, turns = (per_win + at_once - 1) / at_once;
    a.split = 1;
    while (a.split < 8 && a.split < turns && (long long)BH * a.n_win * a.split * 2 <= 4LL * kSms) a.split *= 2;
    const int rpb = kRowThreads / (d / 8);
    a.copy_blocks = (a.n_sink + a.n_ins + rpb - 1) / rpb;
    if ((long long)BH * a.n_win > 0x7fffffffLL / 8) return LRSA_ERR_UNSUPPORTED;
    a.list_blocks = BH * a.n_win;
    grid = (long long)a.list_blocks * a.split + ((long long)BH * a.copy_blocks + a.split - 1) / a.split * a.split;
  } else {
    // few blocks: one a thread block (a window of 512 out of the ring, 16 pairs: 4.7 us instead of 6.7)
    if ((long long)BH * a.n_win * per_win * a.lanes < 2LL * kSms * kRowThreads) threads = a.lanes > 64 ? a.lanes : 64;
    const int rpb = threads / (d / 8), bpb = threads / a.lanes;
    a.copy_blocks = (a.n_sink + a.n_ins + rpb - 1) / rpb;
    a.list_blocks = (a.n_win * per_win + bpb - 1) / bpb;
    grid = (long long)BH * (a.copy_blocks + a.list_blocks);
  }
  if (grid == 0) return LRSA_OK;
  if (grid > 0x7fffffffLL) return LRSA_ERR_UNSUPPORTED;
  const size_t smem = cut ? (size_t)a.L * 4 : 0;
  auto launch = [&](auto type) -> int {
    constexpr int T = decltype(type)::value;
    if (d == 64) return launch_rows_t<64, T, 4>(a, threads, grid, smem, st, cut);
    return wide ? launch_rows_t<128, T, 8>(a, threads, grid, smem, st, cut) : launch_rows_t<128, T, 4>(a, threads, grid, smem, st, cut);
  };
  return o.type == LRSA_LIST_E4M3   ? launch(std::integral_constant<int, LRSA_LIST_E4M3>())
         : o.type == LRSA_LIST_INT8 ? launch(std::integral_constant<int, LRSA_LIST_INT8>())
                                    : launch(std::integral_constant<int, LRSA_LIST_BF16>());
}

// ---- reading the list back ----
struct StoreReadArgs {
  const void *k_list, *v_list;
  const float *k_scale, *v_scale;
  float *k, *v;          // [BH][n_windows * K][d]
  int n_windows, chunks, K, Kp, rows_list, shift;   // thread blocks per window; log2 of the block
};

// A thread takes four channels of each of four rows, so that a warp writes whole lines: bound by the fp32 rows it writes.
template <int D, int T>
__global__ void __launch_bounds__(256) store_read_kernel(const __grid_constant__ StoreReadArgs a) {
  constexpr int LPR = D / 4, RPS = 256 / LPR;   // lanes a row, rows a step
  const int w = blockIdx.x / a.chunks, chunk = blockIdx.x - w * a.chunks, bh = blockIdx.y >> 1, ch = threadIdx.x % LPR * 4;
  const bool is_v = blockIdx.y & 1;
  const int j0 = chunk * (4 * RPS) + threadIdx.x / LPR;   // row of the window
  const size_t row0 = (size_t)bh * a.rows_list + (size_t)w * a.Kp;
  float* out = (is_v ? a.v : a.k) + (((size_t)bh * a.n_windows + w) * a.K) * D + ch;
  const void* list = is_v ? a.v_list : a.k_list;
  wait_for_front();
  uint2 u[4];
  float scale[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = min(j0 + i * RPS, a.K - 1);
    if constexpr (T == LRSA_LIST_BF16) {
      u[i] = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(list) + (row0 + j) * D + ch);
      scale[i] = 1.f;
    } else {
      u[i] = make_uint2(*reinterpret_cast<const uint32_t*>(static_cast<const unsigned char*>(list) + (row0 + j) * D + ch), 0);
      scale[i] = (is_v ? a.v_scale : a.k_scale)[(row0 + j) >> a.shift];
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = j0 + i * RPS;
    if (j >= a.K) break;
    float x[4];
    if constexpr (T == LRSA_LIST_BF16) {
      x[0] = __uint_as_float(u[i].x << 16); x[1] = __uint_as_float(u[i].x & 0xffff0000u);
      x[2] = __uint_as_float(u[i].y << 16); x[3] = __uint_as_float(u[i].y & 0xffff0000u);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t c = u[i].x >> (8 * e) & 0xffu;
        x[e] = scale[i] * (T == LRSA_LIST_INT8 ? (float)(int8_t)c
                                               : __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)c, __NV_E4M3))));
      }
    }
    *reinterpret_cast<float4*>(out + (size_t)j * D) = make_float4(x[0], x[1], x[2], x[3]);
  }
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
  int list_share, list_rest, recent_share, recent_rest;   // blocks of a CTA; so many CTAs have one more
  int n_split, n_group;
  float scale_log2;
};

// Rows reach a warp through a ring of its own in shared memory, filled by asynchronous 16-byte copies: kRing stages of kStage bytes.
// The 16-byte chunks of every 128 bytes lie in an order in which neither the lanes' reads of K nor those of V meet in a bank
// (kBytes: of a row; row counts from the start of the stage).
constexpr int kRing = 3, kStage = 4096;
template <int kBytes>
__device__ __forceinline__ uint32_t swizzled(int row, int byte) {   // byte within the row, a multiple of 8
  const uint32_t at = row * kBytes + byte;
  if constexpr (kBytes == 64) return at ^ (at >> 7 & 3) << 5;
  if constexpr (kBytes == 128) return at ^ ((row & 1) << 6 ^ (row >> 1 & 3) << 5);
  return at ^ (((row ^ row >> 1) & 1) << 6 | (row >> 2 & 1) << 4);
}
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// zeros unless `there` (src is an address that may be read, but is not)
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint2 lds8(uint32_t p) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint4 lds16(uint32_t p) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(p) : "memory");
  return v;
}
__device__ __forceinline__ void mma_16816_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                              uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// this CTA's variable at `p` as CTA `rank` of the cluster has it
__device__ __forceinline__ void st_cluster(const float* p, int rank, float v) {
  uint32_t addr;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(ptx::smem_u32(p)), "r"(rank));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
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

// Grid (n_group * n_split, BHkv), clusters of n_split CTAs of eight warps (four with two groups of heads).  One query token per
// (batch, head): the work is the transfer of the rows, one byte an element in the list and two in the recent rows, so a
// warp takes 8 KB of K and V at a time of either, 256 / d groups of sixteen list rows or half as many of recent rows.  They come by
// asynchronous copies into a ring of three stages per warp: two of them are on their way while the third is used, 128 KB an SM with
// two CTAs.  (Loaded straight into registers, as in decode_kernel, the next ones have no room on their way: sixteen sequences of 28/4
// heads at 32K took 44.7 us instead of 37.8 then, four of 32/8 at 120K 134.6 instead of 111.4.)  The warp-level products take
// the rows from there; as in decode_kernel (lrsa_infer.cu) which channel or key a lane's chunk stands for is the same on
// both sides of a product, so that a lane reads 8 or 16 bytes at a time.
//   List.  A code is widened to a half (exact) and multiplied as such.  Q is brought into the range of halves by a power of
//     two per head (exact but for elements below 2^-28 of the head's largest).  The K scale of a group multiplies its scores.
//     The V scale enters the exponent, p' = 2^(s + log2(scale) - m' + 7), with a running maximum m' of that sum: what is rounded
//     to a half is at most 2^15 and 2^7 or more for the key that counts most, whatever the scales are, so a half's
//     smallest step is 2^-31 of it; O is in units of 2^(m' - 7).  The sum of the weights has its own maximum m and is kept in fp32.
//   Recent rows, and a bf16 list.  bf16 products with the bf16 Q, scale 1; the probabilities are bf16 there, as the product asks for.
//   Rounding.  The sums of the probabilities, and the weights, are formed before they are rounded.  A term of O is off by half a step of its
//     probability, 2^-11 (halves) or 2^-8 (bf16) at most, either way: o is 1.8e-3 to 2.0e-3 (root mean square, relative) from the exact
//     one where probabilities of 32 bits leave 1.65e-3, the rounding of o itself.  Two bf16 for a probability would be twice the products
//     with V.  decode_kernel rounds alike.
// The maxima are raised only when they grew by more than 2^8 (then O is rescaled).  Every CTA takes an even share of the list's
// blocks and one of the recent rows'.  The CTAs of a cluster write their maxima, sums and parts of O into one another's
// shared memory, then meet once (reading from one another between two meetings: one sequence of 28/4 heads at 32K, by weight and with its
// host time, 16.8 us instead of 15.4).  With `weight` the ring's scores are stored, and when the cluster has its maximum and sum, each CTA
// adds exp2(score - lse) over the heads to the weights of the keys that were its own: one owner per key, no atomics.  Several
// clusters per head: store_finish_kernel does both.
// Bound by the rows it reads where there are many (sixteen sequences at 32K, 189 MB: 33.8 us, 5.6 TB/s; four at 120K, 623 MB: 107 us in short
// runs, 117 in long ones, 5.8 and 5.3 TB/s); where there are few by its start, two or three round trips to memory and the merge (one of 28/4
// heads at 32K 8.6 us in a graph, of 8/8, d = 64, at 4K 5.0, by weight 9.4 and 5.4).
template <int D, int NH, int T>
__global__ void __launch_bounds__(dec_max_warps(NH) * 16, 2) store_decode_kernel(const __grid_constant__ StoreDecodeArgs a) {
  constexpr bool k8 = T != LRSA_LIST_BF16;
  constexpr int UL = 128 / D;               // 16-row groups per block
  constexpr int KC = D / 32;                // 16-byte chunks of a bf16 row per lane
  constexpr int KC8 = D / 64;               // of an 8-bit row
  constexpr int VC = D / 64;                // 16-byte chunks of V per lane, bf16
  constexpr int MT = D / 16;                // channel tiles of the output: tile f holds channels g*D/8 + 2f, + 1
  constexpr int kSlot = 8 * (D + 4);        // floats of a warp's O in the merge
  constexpr float kLift = 7.f;              // 8 + 7 < 16: no half overflows between two raises of the maxima
  constexpr int kWarps = dec_max_warps(NH) / 2;
  // The rings; behind the loops, in the same place, the O of the warps [8 heads][D + 4] each.
  extern __shared__ __align__(128) unsigned char dec_smem[];
  float* sm_o = reinterpret_cast<float*>(dec_smem);
  __shared__ float sm_m[kWarps][8], sm_l[kWarps][8], sm_r[kWarps][8], sm_f[kWarps][8];
  // What the CTAs of the cluster write here: their maxima and sums, and their part of the outputs that are this one's.  The head groups
  // take turns (a CTA writes those of group h + 1 when all have read those of group h - 1).
  __shared__ float in_mlr[NH][kDecMaxSplits][3][8], in_o[NH][8 * D + kDecMaxSplits];
  __shared__ __align__(16) uint4 sm_q[NH][KC][32];                    // bf16
  __shared__ __align__(16) uint4 sm_h[k8 ? NH : 1][k8 ? 2 * KC8 : 1][32];   // halves
  __shared__ __align__(8) float sm_scale[k8 ? kWarps : 1][kRing * 2 * UL];   // of the groups of a stage: K, V
  __shared__ float sm_qs[8 * NH];                                     // what the halves are multiplied by
  __shared__ float all_f[kDecMaxSplits][8], sum_m[8], sum_l[8];       // factor of a CTA's O, maximum and sum of the cluster
  __shared__ float sm_lse[8 * NH];                                    // of the pass, in the log2 domain
  const int bh = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int nw = kWarps, kThreads = 32 * kWarps;
  const int g = lane >> 2, t = lane & 3;
  const int b = bh / a.Hkv, hkv = bh % a.Hkv;
  const unsigned char* kl = a.k_list + (size_t)bh * a.rows_list * (k8 ? D : 2 * D);
  const unsigned char* vl = a.v_list + (size_t)bh * a.rows_list * (k8 ? D : 2 * D);
  const unsigned char* kr = reinterpret_cast<const unsigned char*>(a.k_recent) + (size_t)bh * a.recent * (D * 2);
  const unsigned char* vr = reinterpret_cast<const unsigned char*>(a.v_recent) + (size_t)bh * a.recent * (D * 2);
  const float* ks = a.k_scale + (size_t)bh * (a.rows_list >> a.shift);
  const float* vs = a.v_scale + (size_t)bh * (a.rows_list >> a.shift);
  // byte offset of recent key `key`'s row; beyond the end: the last one's
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
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // (waited for before anything is written to another CTA)
  // This CTA's blocks: an even share of the list's (l0 ...) and of the recent rows' (r0 ...), which are twice the bytes.  Block v
  // of the CTA is list block l0 + v for v < nl, then recent block r0 + v - nl.
  const int x = blockIdx.x, l0 = a.list_share * x + min(x, a.list_rest), nl = a.list_share + (x < a.list_rest);
  const int r0 = a.recent_share * x + min(x, a.recent_rest), nr = a.recent_share + (x < a.recent_rest);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0 && bh == 0 && tid == 0) *a.status = 0;

  // The warp takes the CTA's blocks warp, warp + nw, ...  The first n_list of them are 8-bit blocks of the list, a stage each (K and
  // V), the others bf16 rows (first of a bf16 list), a stage for K and one for V.
  const int n_blk = max(0, (nl + nr - warp + nw - 1) / nw), n_list = k8 ? max(0, (nl - warp + nw - 1) / nw) : 0;
  const int n_stages = n_list + 2 * (n_blk - n_list);
  // Place of a 16-row group in the list: group j of a window.  A cursor goes from block to block without a division.
  struct Cursor { int w, j; };
  const int step = nw * UL, step_w = step / a.gpw, step_j = step - step_w * a.gpw;
  auto cursor_at = [&](int group) {
    Cursor c;
    c.w = group / a.gpw;
    c.j = group - c.w * a.gpw;
    return c;
  };
  auto advance = [&](Cursor& c) {
    c.w += step_w;
    c.j += step_j;
    if (c.j >= a.gpw) { c.j -= a.gpw; ++c.w; }
  };
  // first row of the group `u` places behind the cursor; beyond the last group `last`: of the first
  auto group_row = [&](Cursor c, int u, bool there) {
    c.j += u;
    if (c.j >= a.gpw) { c.j -= a.gpw; ++c.w; }   // (UL <= 2 and a window has a group at least)
    return there ? c.w * a.Kp + c.j * 16 : 0;
  };
  auto group_rows = [&](Cursor c, int u, bool there) {   // its visible rows
    c.j += u;
    if (c.j >= a.gpw) c.j -= a.gpw;
    return there ? min(16, a.K - c.j * 16) : 0;
  };
  const uint32_t ring = ptx::smem_u32(dec_smem) + warp * (kRing * kStage), meta = ptx::smem_u32(sm_scale[k8 ? warp : 0]);
  int f_stage = 0, f_slot = 0, f_v = warp;   // the next stage to ask for, its slot, its block
  Cursor f_at = cursor_at((l0 + warp) * UL);
  // what this lane copies of a stage: 16 bytes of rows lane / chunks-per-row, ...
  const uint32_t own8 = swizzled<D>(lane / (D / 16), lane % (D / 16) * 16);
  auto fetch = [&]() {
    const uint32_t dst = ring + f_slot * kStage;
    if (f_stage < n_list) {
#pragma unroll
      for (int u = 0; u < UL; ++u) {
        const int row = group_row(f_at, u, (l0 + f_v) * UL + u < a.n_groups);
        const unsigned char *pk = kl + (size_t)row * D + lane * 16, *pv = vl + (size_t)row * D + lane * 16;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {   // 512 bytes each: 4 rows (d = 128), 8 rows (64)
          const uint32_t to = dst + u * 16 * D + ((D == 128 && (k & 1)) ? own8 ^ 64 : own8) + k * 512;
          copy_async16(to, pk + k * 512);
          copy_async16(to + kStage / 2, pv + k * 512);
        }
        if (lane < 2) copy_async4(meta + (f_slot * 2 * UL + 2 * u + lane) * 4, (lane ? vs : ks) + (row >> a.shift));
      }
      advance(f_at);
      f_v += nw;
    } else if (f_stage < n_stages) {
      const bool is_v = (f_stage - n_list) & 1, in_list = !k8 && f_v < nl;
      constexpr int kRows = 512 / (2 * D);   // rows per 512 bytes
      const int key0 = (r0 + f_v - nl) * (16 * UL);
      const unsigned char* src = in_list ? (is_v ? vl : kl) : (is_v ? vr : kr);
      // the block's rows one behind the other?
      int first = key0 - a.n_front + a.ring0;
      if (first >= a.L2) first -= a.L2;
      const bool run = !in_list && key0 >= a.n_front && key0 + 16 * UL <= a.n_recent && first + 16 * UL <= a.L2;
      const unsigned char* base = src + (size_t)(a.S + first) * (2 * D) + lane * 16;
      if (run) {
#pragma unroll
        for (int k = 0; k < kStage / 512; ++k)
          copy_async16(dst + swizzled<2 * D>(lane / (D / 8) + kRows * k, lane % (D / 8) * 16), base + k * 512);
      } else {
        // Rows behind the last one are zeros: their probability is zero, which an infinity must not meet.
#pragma unroll
        for (int k = 0; k < kStage / 512; ++k) {
          const int r = lane / (D / 8) + kRows * k;
          const bool there = in_list ? (l0 + f_v) * UL + (r >> 4) < a.n_groups : key0 + r < a.n_recent;
          const size_t at = in_list ? (size_t)(group_row(f_at, r >> 4, there) + (r & 15)) * (2 * D) : recent_row(key0 + r);
          copy_async16(dst + swizzled<2 * D>(r, lane % (D / 8) * 16), src + at + lane % (D / 8) * 16, there);
        }
      }
      if (is_v) { f_v += nw; advance(f_at); }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    ++f_stage;
    f_slot = f_slot == kRing - 1 ? 0 : f_slot + 1;
  };
  int slot = 0;   // of the stage that is read next
  // waits for the next stage, asks for the one kRing - 1 behind it
  auto stage = [&]() {
    __syncwarp();   // every lane has read the stage in front, whose place is filled now
    fetch();
    asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
    __syncwarp();   // the stage is there for all lanes
    const int at = slot;
    slot = slot == kRing - 1 ? 0 : slot + 1;
    return at;
  };

  for (int g0 = 0; g0 < a.G; g0 += 8 * NH) {
    __syncthreads();   // the rings are idle: what the merge left there has been read
    f_stage = f_slot = slot = 0;
    f_v = warp;
    f_at = cursor_at((l0 + warp) * UL);
    for (int i = 0; i < kRing - 1; ++i) fetch();
    // Q of the pass as the B operand: chunk t + 4j of a lane's head, as it takes the chunks of every key row
    for (int hd = warp; hd < 8 * NH; hd += nw) {
      constexpr int PL = D / 32;   // channels per lane
      const int c0 = lane * PL, li = (hd & 7) * 4;
      uint32_t x[PL / 2] = {};   // pairs of channels
      if (g0 + hd < a.G) {
        const uint32_t* src = reinterpret_cast<const uint32_t*>(a.q + ((size_t)b * a.Hq + hkv * a.G + g0 + hd) * D + c0);
#pragma unroll
        for (int e = 0; e < PL / 2; ++e) x[e] = src[e];
      }
      uint32_t* qb = reinterpret_cast<uint32_t*>(&sm_q[hd >> 3][c0 / 8 / 4][li + c0 / 8 % 4]) + c0 % 8 / 2;
#pragma unroll
      for (int e = 0; e < PL / 2; ++e) qb[e] = x[e];
      if constexpr (k8) {
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < PL / 2; ++e) most = max(most, max(x[e] & 0x7fffu, x[e] >> 16 & 0x7fffu));
        most = __reduce_max_sync(0xffffffffu, most);
        // exponent of the largest element to 14; infinities, NaN and zero stay what they are
        const int e8 = (int)(most >> 7);
        const int up = most == 0 || most >= 0x7f80u ? 0 : 14 - (max(e8, 1) - 127);
        auto two_to = [](int n) { return __int_as_float((n + 127) << 23); };   // n in [-126, 127]
        const float f1 = two_to(up / 2), f2 = two_to(up - up / 2);   // 2^up may exceed the range
        uint32_t* qh = reinterpret_cast<uint32_t*>(&sm_h[hd >> 3][c0 / 64 * 2 + c0 % 16 / 8][li + c0 / 16 % 4]) + c0 % 8 / 2;
#pragma unroll
        for (int e = 0; e < PL / 2; ++e)
          qh[e] = pack_f16(__uint_as_float(x[e] << 16) * f1 * f2, __uint_as_float(x[e] & 0xffff0000u) * f1 * f2);
        if (lane == 0) sm_qs[hd] = two_to(-(up / 2)) * two_to(-(up - up / 2));
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
    int v = warp;
    Cursor at = cursor_at((l0 + warp) * UL);
    if constexpr (k8) {
      float qc[NH][2];   // what takes a product of halves to the log2 domain, but for the scale
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) qc[h][e] = sm_qs[8 * h + 2 * t + e] * a.scale_log2;
      // this lane's places in a stage: K row g, chunk t; V row 2t, its D / 8 channels
      const uint32_t k_at = swizzled<D>(g, t * 16), v_at = swizzled<D>(2 * t, g * (D / 8)) + kStage / 2;
      for (int i = 0; i < n_list; ++i, v += nw) {
        int nvis[UL];
        float fk[UL], lv[UL];
        const int sl = stage();
        const uint32_t buf = ring + sl * kStage;
#pragma unroll
        for (int u = 0; u < UL; ++u) {
          nvis[u] = group_rows(at, u, (l0 + v) * UL + u < a.n_groups);
          const uint2 f = lds8(meta + (sl * 2 * UL + 2 * u) * 4);
          fk[u] = __uint_as_float(f.x);
          lv[u] = __uint_as_float(f.y);
        }
        advance(at);
        float s[NH][UL][4];
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int u = 0; u < UL; ++u) s[h][u][0] = s[h][u][1] = s[h][u][2] = s[h][u][3] = 0.f;
#pragma unroll
        for (int j = 0; j < KC8; ++j) {
          uint4 kq[UL][2];
#pragma unroll
          for (int u = 0; u < UL; ++u)
#pragma unroll
            for (int z = 0; z < 2; ++z) kq[u][z] = lds16(buf + u * 16 * D + (j ? k_at ^ 64 : k_at) + 8 * D * z);   // (d = 64: one chunk)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint4 q[NH];
#pragma unroll
            for (int h = 0; h < NH; ++h) q[h] = sm_h[h][2 * j + c][lane];
#pragma unroll
            for (int u = 0; u < UL; ++u) {
              const uint32_t w0 = c ? kq[u][0].z : kq[u][0].x, w1 = c ? kq[u][1].z : kq[u][1].x;
              const uint32_t w2 = c ? kq[u][0].w : kq[u][0].y, w3 = c ? kq[u][1].w : kq[u][1].y;
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
        }
#pragma unroll
        for (int h = 0; h < NH; ++h) {
#pragma unroll
          for (int u = 0; u < UL; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s[h][u][e] = g + 8 * (e >> 1) < nvis[u] ? s[h][u][e] * (fk[u] * qc[h][e & 1]) : -INFINITY;
        }
        uint32_t pb[NH][UL][2];
        uint32_t vq[UL][4][D / 32];   // D / 8 codes of a V row
#pragma unroll
        for (int u = 0; u < UL; ++u) {
          lv[u] = __log2f(lv[u]);
#pragma unroll
          for (int i2 = 0; i2 < 4; ++i2) {
            const uint32_t pv = buf + u * 16 * D + (i2 & 1 ? (v_at ^ 64) + (D == 128 ? 128 : 0) : v_at) + (i2 >> 1) * 8 * D;   // (d = 64: two rows in 128 bytes)
            if constexpr (D == 128) {
              const uint4 v = lds16(pv);
              vq[u][i2][0] = v.x; vq[u][i2][1] = v.y; vq[u][i2][2] = v.z; vq[u][i2][3] = v.w;
            } else {
              const uint2 v = lds8(pv);
              vq[u][i2][0] = v.x; vq[u][i2][1] = v.y;
            }
          }
        }
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          float mx[2] = {-INFINITY, -INFINITY}, mr[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int u = 0; u < UL; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
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
          for (int f = 0; f < D / 32; ++f) {   // four channels: tiles 2f, 2f + 1
            uint32_t x[2][4];                  // [rows 2t, 2t+1 | + 8][channel]: pairs of keys
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              widen<T>(__byte_perm(vq[u][2 * z][f], vq[u][2 * z + 1][f], 0x5140), x[z][0], x[z][1]);
              widen<T>(__byte_perm(vq[u][2 * z][f], vq[u][2 * z + 1][f], 0x7362), x[z][2], x[z][3]);
            }
#pragma unroll
            for (int h = 0; h < NH; ++h) {
              mma_16816_f16(o[h][2 * f], x[0][0], x[0][1], x[1][0], x[1][1], pb[h][u][0], pb[h][u][1]);
              mma_16816_f16(o[h][2 * f + 1], x[0][2], x[0][3], x[1][2], x[1][3], pb[h][u][0], pb[h][u][1]);
            }
          }
      }
    }
    for (; v < nl + nr; v += nw) {
      // bf16: recent rows, or rows of a bf16 list
      const bool in_list = !k8 && v < nl;
      int nvis[UL], key0[UL];
#pragma unroll
      for (int u = 0; u < UL; ++u) {
        key0[u] = ((r0 + v - nl) * UL + u) * 16;
        nvis[u] = a.n_recent - key0[u];
        if (in_list) nvis[u] = group_rows(at, u, (l0 + v) * UL + u < a.n_groups);
      }
      if (!k8) advance(at);
      float s[NH][UL][4];
      {
        const uint32_t buf = ring + stage() * kStage;
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int u = 0; u < UL; ++u) s[h][u][0] = s[h][u][1] = s[h][u][2] = s[h][u][3] = 0.f;
#pragma unroll
        for (int j = 0; j < KC; ++j) {
          uint4 q[NH];
#pragma unroll
          for (int h = 0; h < NH; ++h) q[h] = sm_q[h][j][lane];
#pragma unroll
          for (int u = 0; u < UL; ++u) {
            const uint4 k0 = lds16(buf + swizzled<D * 2>(16 * u + g, (t + 4 * j) * 16));
            const uint4 k1 = lds16(buf + swizzled<D * 2>(16 * u + g + 8, (t + 4 * j) * 16));
#pragma unroll
            for (int h = 0; h < NH; ++h) {
              mma_16816(s[h][u], k0.x, k1.x, k0.y, k1.y, q[h].x, q[h].y);
              mma_16816(s[h][u], k0.z, k1.z, k0.w, k1.w, q[h].z, q[h].w);
            }
          }
        }
      }
      uint32_t pb[NH][UL][2];
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int u = 0; u < UL; ++u) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[h][u][e] = g + 8 * (e >> 1) < nvis[u] ? s[h][u][e] * a.scale_log2 : -INFINITY;
            mx[e & 1] = fmaxf(mx[e & 1], s[h][u][e]);
          }
          if (a.weight && !in_list) {
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const int key = key0[u] + g + 8 * z;
              if (key >= a.n_front && key < a.n_recent && g0 + 8 * h + 2 * t < a.Gp)
                *reinterpret_cast<float2*>(a.scores + ((size_t)bh * a.L2 + key - a.n_front) * a.Gp + g0 + 8 * h + 2 * t) =
                    make_float2(s[h][u][2 * z], s[h][u][2 * z + 1]);
            }
          }
        }
        float mr[2] = {mx[0], mx[1]};
        raise(h, mx, mr);
        const float rm[2] = {m[h][0] == -INFINITY ? 0.f : m[h][0], m[h][1] == -INFINITY ? 0.f : m[h][1]};
        const float rr[2] = {r[h][0] == -INFINITY ? 0.f : r[h][0] - kLift, r[h][1] == -INFINITY ? 0.f : r[h][1] - kLift};
#pragma unroll
        for (int u = 0; u < UL; ++u) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            l[h][e & 1] += ptx::ex2(s[h][u][e] - rm[e & 1]);
            p[e] = ptx::ex2(s[h][u][e] - rr[e & 1]);
          }
          pb[h][u][0] = transpose_8x8(ptx::pack_bf16(p[0], p[1]));
          pb[h][u][1] = transpose_8x8(ptx::pack_bf16(p[2], p[3]));
        }
      }
      const uint32_t buf = ring + stage() * kStage;
#pragma unroll
      for (int u = 0; u < UL; ++u)
#pragma unroll
        for (int j = 0; j < VC; ++j) {
          uint4 vr4[4];
#pragma unroll
          for (int z = 0; z < 4; ++z) vr4[z] = lds16(buf + swizzled<D * 2>(16 * u + 2 * t + (z & 1) + 8 * (z >> 1), g * (D / 4) + j * 16));
#pragma unroll
          for (int f = 0; f < 4; ++f) {
            auto w = [&](int z) { return f == 0 ? vr4[z].x : f == 1 ? vr4[z].y : f == 2 ? vr4[z].z : vr4[z].w; };
#pragma unroll
            for (int h = 0; h < NH; ++h)
              mma_16816(o[h][4 * j + f], __byte_perm(w(0), w(1), 0x5410), __byte_perm(w(0), w(1), 0x7632),
                        __byte_perm(w(2), w(3), 0x5410), __byte_perm(w(2), w(3), 0x7632), pb[h][u][0], pb[h][u][1]);
          }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    // Merge: the warps through shared memory, the CTAs by writing into one another's.
    const int group = blockIdx.x / a.n_split, rank = blockIdx.x - group * a.n_split;
    const int share = (8 * D + a.n_split - 1) / a.n_split;   // elements of the output that are a CTA's
    // The keys of the ring whose scores this CTA has stored: k0 + tid, + blockDim.x, ... below k1.  What the first of them needs is on
    // its way while the cluster meets.
    const bool weigh = a.weight && a.n_group == 1;
    const int k0 = max(a.n_front, r0 * UL * 16), k1 = weigh ? min(a.n_recent, (r0 + nr) * UL * 16) : 0, n_heads = min(8 * NH, a.G - g0);
    float4 sc[2 * NH];
    float gathered = 0.f;
    auto weight_of = [&](int key) {
      int at = key - a.n_front + a.ring0;
      if (at >= a.L2) at -= a.L2;
      return a.weight + (size_t)bh * a.L2 + at;
    };
    auto load_scores = [&](int key) {
      const float4* src = reinterpret_cast<const float4*>(a.scores + ((size_t)bh * a.L2 + key - a.n_front) * a.Gp + g0);
#pragma unroll
      for (int i = 0; i < 2 * NH; ++i) sc[i] = 4 * i < n_heads ? src[i] : make_float4(0.f, 0.f, 0.f, 0.f);
      gathered = *weight_of(key);
    };
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      auto part_of = [](float from, float to) { return from == -INFINITY ? 0.f : exp2f(from - to); };
      const int ng = min(8, a.G - g0 - 8 * h);
      __syncthreads();   // the rings, or the last group's O, have been read
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float* dst = sm_o + warp * kSlot + (2 * t + e) * (D + 4) + g * (D / 8);
#pragma unroll
        for (int i = 0; i < MT; ++i) *reinterpret_cast<float2*>(dst + 2 * i) = make_float2(o[h][i][e], o[h][i][e + 2]);
        float lh = l[h][e];
#pragma unroll
        for (int y = 4; y < 32; y <<= 1) lh += __shfl_xor_sync(0xffffffffu, lh, y);
        if (g == 0) { sm_m[warp][2 * t + e] = m[h][e]; sm_l[warp][2 * t + e] = lh; sm_r[warp][2 * t + e] = r[h][e] - kLift; }
      }
      if (h == 0 && g0 == 0) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");   // every CTA of the cluster has started
      __syncthreads();
      if (h == NH - 1 && k0 + tid < k1) load_scores(k0 + tid);   // (stored ahead of the barriers above)
      if (tid < 8 * nw) {
        const int hd = tid & 7, w = tid >> 3;
        float M = -INFINITY, R = -INFINITY, ls = 0.f;
#pragma unroll
        for (int k = 0; k < nw; ++k) { M = fmaxf(M, sm_m[k][hd]); R = fmaxf(R, sm_r[k][hd]); }
#pragma unroll
        for (int k = 0; k < nw; ++k) ls = fmaf(sm_l[k][hd], part_of(sm_m[k][hd], M), ls);
        sm_f[w][hd] = part_of(sm_r[w][hd], R);
        for (int k = w; k < a.n_split; k += nw) {
          st_cluster(&in_mlr[h][rank][0][hd], k, M);
          st_cluster(&in_mlr[h][rank][1][hd], k, ls);
          st_cluster(&in_mlr[h][rank][2][hd], k, R);
        }
      }
      __syncthreads();
      for (int i = tid; i < ng * D; i += kThreads) {
        const int hd = i / D, c = i % D, owner = i / share;
        float ov = 0.f;
#pragma unroll
        for (int w = 0; w < nw; ++w) ov = fmaf(sm_o[w * kSlot + hd * (D + 4) + c], sm_f[w][hd], ov);
        st_cluster(&in_o[h][rank * share + i - owner * share], owner, ov);
      }
      cluster_sync();
      for (int hd = warp; hd < ng; hd += nw) {   // a warp per head, a lane per CTA
        const bool there = lane < a.n_split;
        const float mk = there ? in_mlr[h][lane][0][hd] : -INFINITY, rk = there ? in_mlr[h][lane][2][hd] : -INFINITY;
        float M = mk, R = rk;
#pragma unroll
        for (int y = 8; y; y >>= 1) {
          M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, y));
          R = fmaxf(R, __shfl_xor_sync(0xffffffffu, R, y));
        }
        float ls = there ? in_mlr[h][lane][1][hd] * part_of(mk, M) : 0.f;
#pragma unroll
        for (int y = 8; y; y >>= 1) ls += __shfl_xor_sync(0xffffffffu, ls, y);
        // O in units of 2^M: R - M is the scale of the V rows that carry the weight
        if (there) all_f[lane][hd] = R == -INFINITY ? 0.f : part_of(rk, R) * exp2f(R - M);
        if (lane == 0) { sum_m[hd] = M; sum_l[hd] = ls; sm_lse[8 * h + hd] = M + log2f(ls); }
      }
      __syncthreads();
      for (int j = tid; j < share && rank * share + j < ng * D; j += kThreads) {
        const int i = rank * share + j, hd = i / D, c = i % D;
        float ov = 0.f;
#pragma unroll 4
        for (int k = 0; k < a.n_split; ++k) ov = fmaf(in_o[h][k * share + j], all_f[k][hd], ov);
        if (a.n_group > 1) {
          float* dst = a.part + (((size_t)bh * a.n_group + group) * a.G + g0 + 8 * h + hd) * (D + 2);
          dst[c] = ov;
          if (c == 0) { dst[D] = sum_m[hd]; dst[D + 1] = sum_l[hd]; }
          continue;
        }
        const size_t head = (size_t)b * a.Hq + hkv * a.G + g0 + 8 * h + hd;
        a.o[head * D + c] = __float2bfloat16(ov / sum_l[hd]);
        if (c == 0 && a.lse) a.lse[head] = sm_lse[8 * h + hd] * 0.6931471805599453f;
      }
      if (h == NH - 1) {
        for (int key = k0 + tid; key < k1; key += kThreads) {
          if (key != k0 + tid) load_scores(key);
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * NH; ++i) {
            const float y[4] = {sc[i].x, sc[i].y, sc[i].z, sc[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (4 * i + e < n_heads) sum += ptx::ex2(y[e] - sm_lse[4 * i + e]);
          }
          *weight_of(key) = gathered + sum;
        }
      }
    }
  }
}

// Where a head has several clusters: their results are merged, and the weights formed with the log-sums.  Grid (chunks of the ring's
// keys, BHkv); every CTA forms the log-sums of the group's heads, and the CTAs share the elements of the output and the keys.
template <int D>
__global__ void __launch_bounds__(128) store_finish_kernel(const __grid_constant__ StoreDecodeArgs a) {
  extern __shared__ float fin_smem[];
  float *lse2 = fin_smem, *inv = lse2 + a.G, *f = inv + a.G;   // per head: log-sum (log2 domain), 1 / sum; factor of every cluster
  const int bh = blockIdx.y, tid = threadIdx.x, b = bh / a.Hkv, hkv = bh % a.Hkv;
  const size_t head0 = (size_t)b * a.Hq + hkv * a.G;
  const float* part = a.part + (size_t)bh * a.n_group * a.G * (D + 2);
  wait_for_front();
  for (int hd = tid; hd < a.G; hd += 128) {
    float M = -INFINITY, ls = 0.f;
    for (int k = 0; k < a.n_group; ++k) M = fmaxf(M, __ldcg(part + ((size_t)k * a.G + hd) * (D + 2) + D));
    for (int k = 0; k < a.n_group; ++k) {
      const float* p = part + ((size_t)k * a.G + hd) * (D + 2) + D;
      const float m = __ldcg(p), x = m == -INFINITY ? 0.f : exp2f(m - M);
      f[k * a.G + hd] = x;
      ls = fmaf(__ldcg(p + 1), x, ls);
    }
    lse2[hd] = M + log2f(ls);
    inv[hd] = 1.f / ls;
    if (a.lse && blockIdx.x == 0) a.lse[head0 + hd] = lse2[hd] * 0.6931471805599453f;
  }
  __syncthreads();
  for (int i = blockIdx.x * 128 + tid; i < a.G * D; i += gridDim.x * 128) {
    const int hd = i / D, c = i % D;
    float ov = 0.f;
#pragma unroll 4
    for (int k = 0; k < a.n_group; ++k) ov = fmaf(__ldcg(part + ((size_t)k * a.G + hd) * (D + 2) + c), f[k * a.G + hd], ov);
    a.o[head0 * D + i] = __float2bfloat16(ov * inv[hd]);
  }
  const int key = a.n_front + blockIdx.x * 128 + tid;
  if (!a.weight || key >= a.n_recent) return;
  const float4* sc = reinterpret_cast<const float4*>(a.scores + ((size_t)bh * a.L2 + key - a.n_front) * a.Gp);
  int at = key - a.n_front + a.ring0;
  if (at >= a.L2) at -= a.L2;
  float* w = a.weight + (size_t)bh * a.L2 + at;
  float sum = *w;
  for (int i = 0; 4 * i < a.G; ++i) {
    const float4 x = __ldcg(sc + i);
    const float y[4] = {x.x, x.y, x.z, x.w};
    for (int e = 0; e < 4 && 4 * i + e < a.G; ++e) sum += ptx::ex2(y[e] - lse2[4 * i + e]);
  }
  *w = sum;
}

// Heads of a group whose factors store_finish_kernel has room for; where there are more, a pair has one cluster.
constexpr int kFinishHeads = 48 * 1024 / (4 * (2 + kDecMaxGroups));

// How the blocks are dealt out: `groups` clusters of `splits` CTAs a (batch, KV head) pair, two CTAs on an SM (of 8 warps, 4 with two head
// groups), by a model of the time in cycles: a warp takes about 2400 for a block, with all warps of the SM at work 170 for each (the
// memory's rate and about the issue rate); start and merge take 4000, the kernel behind several clusters and their traffic 20 000.
// us, splits x groups, * the plan that is taken: sixteen sequences of 28/4 heads at 32K (e4m3) 4x1* 34.0, 2x1 34.7, 3x1 37.2, 8x1 38.1, 6x1
// 44.7, 1x1 57; one of them 16x1* 10.0, 12x1 10.8, 8x1 12.6, 8x2 17.8, 16x2 17.3, 4x4 19.3; four of 32/8 at 120K (int8) 8x1* 107, 2x4 113,
// 1x9 117, 4x1 119, 16x1 127, 9x1 (two waves of clusters) 138; four of 8/8, d = 64, at 66K 8x1* 21.1, 4x1 26.2, 9x1 29.2, 16x1 31.0, 16x2 44.6.
// Where one pair's list is long the model takes several clusters too early: one sequence of 28/4 at 127K 12x5* 27.7, 16x1 19.3, 16x2 25.8.
DecodePlan store_plan(const Geom& g, int blocks, int max_splits = kDecMaxSplits) {
  const int nh = g.G > 8 ? 2 : 1, warps = dec_max_warps(nh) / 2;
  DecodePlan best = {nh, warps, blocks, 1, 1};
  const unsigned BH = (unsigned)g.B * g.Hkv;
  const ClusterRoom& room = cluster_room();
  unsigned long long least = ~0ull;
  for (int s = 1; s <= max_splits; ++s) {
    const unsigned at_once = room.at_once(2, s);
    // one cluster for a pair, or as many as run at a time
    const unsigned fit = BH > 2 * kSms || g.G > kFinishHeads ? 1 : at_once / BH < kDecMaxGroups ? at_once / BH : kDecMaxGroups;
    for (unsigned grp = 1; grp == 1 || grp <= fit; grp = grp == 1 && fit > 1 ? fit : kDecMaxGroups + 1) {
      const unsigned n = s * grp;
      if (n > 1 && (n - 1) * warps >= (unsigned)blocks) break;
      const unsigned clusters = BH * grp, waves = (clusters + at_once - 1) / at_once;
      const unsigned on_sm = ((clusters < at_once ? clusters : at_once) * s + kSms - 1) / kSms;
      const unsigned rounds = (blocks + n * warps - 1) / (n * warps), busy = 170 * on_sm * warps;
      const unsigned long long cost = (unsigned long long)waves * (rounds * (busy > 2400 ? busy : 2400) + 4000) + (grp > 1 ? 20000 : 0);
      if (cost <= least) { least = cost; best.splits = s; best.groups = grp; }
    }
  }
  return best;
}

template <int D, int NH, int T>
cudaError_t launch_store_decode_t(StoreDecodeArgs& a, const DecodePlan& pl, int BHkv, cudaStream_t st) {
  auto kern = store_decode_kernel<D, NH, T>;
  const int merge = pl.warps * 8 * (D + 4) * 4, rings = pl.warps * kRing * kStage, smem = merge > rings ? merge : rings;
  const cudaError_t es = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (es != cudaSuccess) return es;
  if (pl.splits > 8) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return launch_dependent(kern, dim3(pl.splits * pl.groups, BHkv), dim3(pl.warps * 32), smem, st, pl.splits, a);
}

template <int T>
cudaError_t launch_store_decode(const Geom& g, StoreDecodeArgs a, const DecodePlan& pl, int list_blocks, int recent_blocks, int bh0, int BHkv,
                                cudaStream_t st) {
  // pairs [bh0, + BHkv): the heads of a pair are G behind one another in q, o and lse
  const size_t at = bh0, row = (size_t)g.d * (T == LRSA_LIST_BF16 ? 2 : 1);
  a.q += at * g.G * g.d; a.o += at * g.G * g.d;
  if (a.lse) a.lse += at * g.G;
  a.k_list += at * a.rows_list * row; a.v_list += at * a.rows_list * row;
  a.k_scale += at * (a.rows_list >> a.shift); a.v_scale += at * (a.rows_list >> a.shift);
  a.k_recent += at * a.recent * g.d; a.v_recent += at * a.recent * g.d;
  if (a.weight) { a.weight += at * a.L2; a.scores += at * a.L2 * a.Gp; }
  a.n_split = pl.splits; a.n_group = pl.groups;
  const int n = pl.splits * pl.groups;
  a.list_share = list_blocks / n; a.list_rest = list_blocks % n;
  a.recent_share = recent_blocks / n; a.recent_rest = recent_blocks % n;
  if (g.d == 128) return pl.nh == 1 ? launch_store_decode_t<128, 1, T>(a, pl, BHkv, st) : launch_store_decode_t<128, 2, T>(a, pl, BHkv, st);
  return pl.nh == 1 ? launch_store_decode_t<64, 1, T>(a, pl, BHkv, st) : launch_store_decode_t<64, 2, T>(a, pl, BHkv, st);
}

constexpr int kGridRows = 65535;

// Parts of the workspace.
struct StoreWs { size_t part, scores, total; };
StoreWs store_ws(const Geom& g, const StoreGeom& o) {
  StoreWs w;
  const size_t BH = (size_t)g.B * g.Hkv;
  size_t off = sizeof(WsHeader);
  // several clusters for a head only where they run at a time (store_plan)
  w.part = off; off += align_up(BH <= 2 * (size_t)kSms ? BH * kDecMaxGroups * g.G * (g.d + 2) * sizeof(float) : 0, 256);
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
  // Lag rule: selects windows [w0, + n), out of the ring (one window) or out of the new tokens.
  auto score = [&](int w0, int n, bool ring) -> int {
    Geom s = g;
    s.S = 0; s.T = 0; s.W = n + 1; s.C = n + 1; s.Wsel = n; s.Wtot = o.Wcap; s.woff = w0; s.emit_off = g.S + w0 * g.L;
    s.N = s.Nrow = ring ? o.recent : n_new;
    s.tok0 = ring ? g.S + (w0 % 2) * g.L : g.S + w0 * g.L - n_prev;
    s.win_stride = ring && w0 % 2 ? -g.L : g.L;
    const bool self = !cleared && score_select_clears_status(s);
    if (!cleared && !self) {
      LRSA_CUDA_CHECK(cudaMemsetAsync(workspace, 0, sizeof(WsHeader), st));
      launch_counter().n++;
    }
    cleared = true;
    return launch_score_select(&s, 1, ring ? rows.k_recent : rows.k_new, ring ? rows.v_recent : rows.v_new, store->idx, nullptr, workspace, st, self);
  };
  auto move_rows = [&](bool cut = false) -> int {   // cut: windows are selected, by weight, in the same launch
    if (rows.n_sink + rows.n_ins + rows.n_win == 0) return LRSA_OK;
    rows.status = cleared ? nullptr : status;
    cleared = true;
    return launch_store_rows(rows, o, BH, g.d, st, cut);
  };
  int pos = n_prev;                                     // tokens before it are in the store
  int c = pos > g.S ? (pos - g.S - 1) / g.L + 1 : 0;    // next chunk whose first token has not arrived yet
  if (c < 2) c = 2;
  // Lag rule: chunk start after chunk start while the window c-2 that leaves the ring holds tokens of earlier calls (at most two).
  // The tokens up to it enter the ring, the window is scored with its successor there, its kept rows join the list before its
  // half is overwritten.
  for (; !o.by_weight && (long long)g.S + (long long)c * g.L < end && g.S + (c - 2) * g.L < n_prev; ++c) {
    const int w = c - 2;
    rows.p0 = pos; rows.n_ins = g.S + c * g.L - pos; rows.n_win = 0;
    if ((rc = move_rows()) != LRSA_OK) return rc;
    if ((rc = score(w, 1, true)) != LRSA_OK) return rc;
    rows.n_ins = 0; rows.w0 = w; rows.n_win = 1; rows.ring_below = INT_MAX;
    if ((rc = move_rows()) != LRSA_OK) return rc;
    pos = g.S + c * g.L;
  }
  rows.n_win = 0;
  rows.p0 = pos; rows.n_ins = end - pos;
  if ((long long)g.S + (long long)c * g.L < end) {
    // Windows c-2 .. c_last-2, one selection for all of them, then their kept rows, the sinks and the tokens that stay in the ring.
    // By the lag rule they lie in the new tokens as a whole, by weight the first ones may be in the ring.
    const int w0 = c - 2, nw = (end - 1 - g.S) / g.L - c + 1;
    if (!o.by_weight && (rc = score(w0, nw, false)) != LRSA_OK) return rc;
    rows.w0 = w0; rows.n_win = nw; rows.ring_below = n_prev;
    if (g.S + w0 * g.L < n_prev) {   // rows of the ring have to be read before tokens take their places
      rows.n_ins = 0;
      if ((rc = move_rows(o.by_weight)) != LRSA_OK) return rc;
      rows.n_win = 0;
    }
    rows.n_sink = pos < g.S ? g.S - pos : 0;
    rows.p0 = end - 2 * g.L > pos ? end - 2 * g.L : pos;
    rows.n_ins = end - rows.p0;
  }
  return move_rows(o.by_weight && rows.n_win > 0);
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
  const int ur = 128 / g.d;   // 16-row groups per block
  const int list_blocks = (a.n_groups + ur - 1) / ur, recent_blocks = (a.n_recent + 16 * ur - 1) / (16 * ur);
  DecodePlan pl = store_plan(g, list_blocks + recent_blocks);
  const int BH = g.B * g.Hkv;
  // A grid has 65535 rows: more pairs take turns.  (Folded into another dimension, the pair's number costs every CTA a division, sixteen
  // sequences of 28/4 heads at 32K 34.8 us instead of 34.5, or registers, 35.7.)
  for (int bh0 = 0; bh0 < BH; bh0 += kGridRows) {
    const int n = BH - bh0 < kGridRows ? BH - bh0 : kGridRows;
    auto launch = [&](const DecodePlan& p) {
      return o.type == LRSA_LIST_E4M3 ? launch_store_decode<LRSA_LIST_E4M3>(g, a, p, list_blocks, recent_blocks, bh0, n, st)
             : o.type == LRSA_LIST_INT8 ? launch_store_decode<LRSA_LIST_INT8>(g, a, p, list_blocks, recent_blocks, bh0, n, st)
                                        : launch_store_decode<LRSA_LIST_BF16>(g, a, p, list_blocks, recent_blocks, bh0, n, st);
    };
    cudaError_t e = launch(pl);
    if (e != cudaSuccess && pl.splits > 8) {   // clusters of 16 are not portable: a part of a GPU may not have room for them
      (void)cudaGetLastError();
      pl = store_plan(g, list_blocks + recent_blocks, 8);
      e = launch(pl);
    }
    LRSA_CUDA_CHECK(e);
    launch_counter().n++;
  }
  if (pl.groups > 1) {
    a.n_group = pl.groups;
    const int keys = a.weight ? a.n_recent - a.n_front : 0, chunks = keys > 128 ? (keys + 127) / 128 : 1;
    const size_t smem = (size_t)(2 + pl.groups) * g.G * sizeof(float);
    auto finish = g.d == 128 ? store_finish_kernel<128> : store_finish_kernel<64>;
    LRSA_CUDA_CHECK(launch_dependent(finish, dim3(chunks, g.B * g.Hkv), dim3(128), smem, st, 1, a));
    launch_counter().n++;
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
  StoreReadArgs a = {};
  a.k_list = store->k_list; a.v_list = store->v_list; a.k_scale = store->k_scale; a.v_scale = store->v_scale; a.k = k; a.v = v;
  const int rows = 4 * 256 / (g.d / 4);   // of a thread block
  a.n_windows = n_windows; a.chunks = (g.K + rows - 1) / rows; a.K = g.K; a.Kp = o.Kp; a.rows_list = o.rows_list;
  while ((1 << a.shift) < o.block) ++a.shift;
  if ((long long)n_windows * a.chunks > 0x7fffffffLL) return LRSA_ERR_UNSUPPORTED;
  auto kern = g.d == 128 ? (o.type == LRSA_LIST_E4M3 ? store_read_kernel<128, LRSA_LIST_E4M3> : o.type == LRSA_LIST_INT8 ? store_read_kernel<128, LRSA_LIST_INT8> : store_read_kernel<128, LRSA_LIST_BF16>)
                         : (o.type == LRSA_LIST_E4M3 ? store_read_kernel<64, LRSA_LIST_E4M3> : o.type == LRSA_LIST_INT8 ? store_read_kernel<64, LRSA_LIST_INT8> : store_read_kernel<64, LRSA_LIST_BF16>);
  const size_t BH = (size_t)g.B * g.Hkv, row = (size_t)g.d * (o.type == LRSA_LIST_BF16 ? 2 : 1);
  for (size_t bh0 = 0; bh0 < BH; bh0 += kGridRows / 2) {   // K and V of a pair are two rows of a grid
    const size_t n = BH - bh0 < kGridRows / 2 ? BH - bh0 : kGridRows / 2;
    StoreReadArgs b = a;
    b.k_list = static_cast<const unsigned char*>(a.k_list) + bh0 * a.rows_list * row;
    b.v_list = static_cast<const unsigned char*>(a.v_list) + bh0 * a.rows_list * row;
    b.k_scale += bh0 * (a.rows_list >> a.shift); b.v_scale += bh0 * (a.rows_list >> a.shift);
    b.k += bh0 * a.n_windows * a.K * g.d; b.v += bh0 * a.n_windows * a.K * g.d;
    LRSA_CUDA_CHECK(launch_dependent(kern, dim3((unsigned)n_windows * a.chunks, (unsigned)n * 2), dim3(256), 0,
                                     static_cast<cudaStream_t>(cuda_stream), 1, b));
    launch_counter().n++;
  }
  return LRSA_OK;
}

}  // extern "C"
