// Accumulated attention weight of every position over a whole prompt, on tcgen05 tensor cores (key-outer).
//
//   weight[j] = sum over the query heads of the KV group and the queries t that see position j uncompressed of
//               P_tj = exp(scale * q_t k_j - LSE_t)
//
// Position j of window w is seen uncompressed by the queries t >= j up to the end of the last chunk that does not see the
// window through its kept tokens, so the work is about 1.5 L queries a key whatever the length of the sequence.  A CTA
// takes a tile of 128 keys and walks the (128-query tile, query head) pairs that see it:
//   S^T = K_j Q_i^T   (smem x smem -> TMEM, keys on lanes)     acc_key += exp2(S^T*c - LSE_i*log2e)
// With keys on the lanes a thread owns a key row, so the sum over the queries stays in its registers; nothing is exchanged
// until the end.  Where there are few tiles a cluster of CTAs shares one, each takes a run of its pairs, and rank 0 adds
// the partial sums in the order of the ranks (no atomics: repeats are equal bit by bit).
// Bound by the unit that forms the exponentials, one a pair (32K tokens of 28/4 heads, d = 128, windows of 1024: 1.4e9 of them take
// 297 us at 1965 MHz, the products 213; measured 480 to 503, at 1.68 GHz, that unit 78 % and the issue slots 40 % busy by their
// counters); shorter prompts by tiles of unequal length on few places (4K tokens of 8 heads, d = 64: 14 us, 256 tiles on 296 places,
// of which 5 are exponentials).
// Rounding: the exponent is one fma of the score with -LSE * log2(e), itself rounded to fp32, and goes to ex2.approx (2^-22 relative):
// an exponential costs one instruction of the unit that bounds the kernel.  A weight is within 1.1e-7 of its exact value
// (32-bit torch operations: 4.6e-8), relative, at 32K.
#include <math.h>

#include <type_traits>

#include "attn_common_sm100.h"
#include "infer_sm100.h"

namespace lrsa {
namespace {

using namespace ptx;

template <int D>
struct WgtCfg {
  static constexpr int kSub = D / 64;
  static constexpr int kSubBytes = kTile * 128;
  static constexpr int kTileBytes = kSub * kSubBytes;      // K_j or Q_i
  static constexpr int kStages = D == 128 ? 2 : 4;         // Q tiles in flight: 96 KB a CTA, two CTAs an SM
  static constexpr int kOffQ = kTileBytes;
  static constexpr int kOffStats = kOffQ + kStages * kTileBytes;   // two slots of 128 x -LSE*log2(e)
  static constexpr int kOffCtl = kOffStats + 2 * kTile * 4;
  static constexpr int kSmem = kOffCtl + 1280;
  static constexpr int kSoftWarps = 8;                     // two warpgroups of 64 query columns each
  static constexpr int kThreads = 128 + 32 * kSoftWarps;   // TMA producer, issuer, (idle), statistics; exponentials
  static constexpr uint32_t kCols = 256;                   // two buffers of S^T
};

// Key tiles of one sequence: the windows and the tail (sink positions are never candidates and get weight zero).
struct WgtPlan {
  int S, L, N, W, C, Wsel, ndp, per_win, n_tiles;
};

inline WgtPlan make_wgt_plan(const Geom& g) {
  WgtPlan p;
  p.S = g.S; p.L = g.L; p.N = g.N; p.W = g.W; p.C = g.C; p.Wsel = g.Wsel; p.ndp = g.ndp;
  p.per_win = (g.L + kTile - 1) / kTile;
  p.n_tiles = g.W * p.per_win + (g.T + kTile - 1) / kTile;
  if (p.n_tiles == 0) p.n_tiles = 1;   // nothing but sinks: one tile without queries
  return p;
}

template <int NSEQ>
struct WgtMaps { CUtensorMap q[NSEQ], k[NSEQ]; };

template <int NSEQ>
struct WgtArgs {
  WgtPlan plan[NSEQ];
  int tok0[NSEQ], item0[NSEQ + 1];   // first token; (head, tile) pairs of the sequences before
  int n_seqs, BHkv, Hq, Hkv, G, Nrow, split;
  const float* LSE;    // [B*Hq][Nrow]
  float* weight;       // [BHkv][Nrow]
  float scale_log2;
  int* status;
  int clear;           // the status word, by the first launch of a call
};

// Behind the statistics in shared memory (nothing is static, so that the tiles start on 1024 bytes).
struct WgtCtl {
  uint64_t k_full, q_full[4], q_empty[4];
  uint64_t s_full[2], s_empty[2];   // S^T of the step is in tensor memory and its statistics are staged; both have been read
  float part[2][kTile];             // [warpgroup][key]; [0] then holds the CTA's sums
  uint32_t tmem_base;
  int abort;
};
static_assert(sizeof(WgtCtl) <= 1280, "control block fits");

template <int D, int NSEQ>
__global__ void __launch_bounds__(WgtCfg<D>::kThreads, 2)
lrsa_weights_kernel(const __grid_constant__ WgtMaps<NSEQ> maps, const __grid_constant__ WgtArgs<NSEQ> a) {
  using Cfg = WgtCfg<D>;
  constexpr int NQ = Cfg::kStages;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const uint32_t smem0 = smem_u32(smem_raw), sK = smem0, sQ = smem0 + Cfg::kOffQ;
  float* st_nl2 = reinterpret_cast<float*>(smem_raw + Cfg::kOffStats);
  WgtCtl& ctl = *reinterpret_cast<WgtCtl*>(smem_raw + Cfg::kOffCtl);
  const uint32_t k_full = smem_u32(&ctl.k_full), q_full = smem_u32(ctl.q_full), q_empty = smem_u32(ctl.q_empty),
                 s_full = smem_u32(ctl.s_full), s_empty = smem_u32(ctl.s_empty);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort = &ctl.abort;

  // ---- which tile, which part of its pairs ----
  const int rank = blockIdx.x % a.split;
  int item = blockIdx.x / a.split, sq = 0;
  if constexpr (NSEQ > 1) {
    while (sq + 1 < a.n_seqs && item >= a.item0[sq + 1]) ++sq;
    item -= a.item0[sq];
  }
  const WgtPlan& p = a.plan[sq];
  const int bh = item / p.n_tiles, tile = item % p.n_tiles, tok0 = a.tok0[sq];
  const int w = min(tile / p.per_win, p.W);
  const int row0 = p.S + w * p.L + (tile - w * p.per_win) * kTile;
  const int key_end = min(p.N, p.S + (w + 1) * p.L);
  const int cc = first_compressed_chunk(w, p.ndp, p.Wsel, p.C);
  const int qend = cc >= p.C ? p.N : min(p.N, p.S + cc * p.L);
  const int nq = qend > row0 ? (qend - row0 + kTile - 1) / kTile : 0;
  const int all = a.G * nq, per = all / a.split, rest = all - per * a.split;
  const int it0 = per * rank + min(rank, rest), n = per + (rank < rest);
  const int hq0 = (bh / a.Hkv) * a.Hq + (bh % a.Hkv) * a.G;
  // pair i: query tile nq-1 - i/G (from the last query backwards) of head i % G of the group
  const int qt0 = nq - 1 - it0 / a.G, hd0 = it0 % a.G;
  auto load_q = [&](int slot, int qt, int hd) {
    mbar_expect_tx(q_full + 8 * slot, Cfg::kTileBytes);
    for (int h = 0; h < Cfg::kSub; ++h)
      tma_load_3d(sQ + slot * Cfg::kTileBytes + h * Cfg::kSubBytes, &maps.q[sq], h * 64, row0 + qt * kTile, hq0 + hd, q_full + 8 * slot);
  };
  if (tid == 0) {
    prefetch_tensormap(&maps.q[sq]); prefetch_tensormap(&maps.k[sq]);
    ctl.abort = (smem0 & 1023u) ? 1 : 0;   // the swizzled tiles need the alignment
    mbar_init(k_full, 1);
    for (int i = 0; i < NQ; ++i) { mbar_init(q_full + 8 * i, 1); mbar_init(q_empty + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 2);   // the product and the statistics
      mbar_init(s_empty + 8 * i, 32 * Cfg::kSoftWarps);
    }
    fence_barrier_init();
    // K_j and the first Q are on their way while the other warps get their tensor memory
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (n > 0 && !ctl.abort) {
      mbar_expect_tx(k_full, Cfg::kTileBytes);
      for (int h = 0; h < Cfg::kSub; ++h) tma_load_3d(sK + h * Cfg::kSubBytes, &maps.k[sq], h * 64, row0, bh, k_full);
      load_q(0, qt0, hd0);
    }
  }
  if (warp == 1) { tmem_alloc(smem_u32(&ctl.tmem_base), Cfg::kCols); tmem_relinquish(); }

  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = ctl.tmem_base;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (a.clear && blockIdx.x == 0 && tid == 0) *a.status = 0;   // (written again only by a wait that has run out, seconds later)

  if (*abort) {
  } else if (warp == 0) {
    // ---------------- TMA producer ----------------
    if (lane == 0 && n > 0) {
      int qt = qt0, hd = hd0, sl = 1, ph = 0, issued = 1;   // (the first step's loads are on their way)
      bool ok = true;
      for (int it = 1; it < n; ++it) {
        if (++hd == a.G) { hd = 0; --qt; }
        if (it >= NQ) ok = mbar_wait(q_empty + 8 * sl, ph ^ 1, abort);
        if (!ok) break;
        load_q(sl, qt, hd);
        ++issued;
        if (++sl == NQ) { sl = 0; ph ^= 1; }
      }
      if (!ok) {   // give the loads in flight a bounded chance to land before shared memory is released
        for (int back = 0; back <= NQ && back <= issued; ++back) {
          const int i = issued - back;
          const uint32_t bar = back == 0 ? k_full : q_full + 8 * (i % NQ);
          const long long t0 = clock64();
          while (!mbar_try_wait(bar, back == 0 ? 0 : (i / NQ) & 1) && clock64() - t0 < 2000000) {}
        }
      }
    }
  } else if (warp == 1) {
    // ---------------- issuer ----------------
    constexpr uint32_t idesc = make_idesc_bf16(kTile, kTile, 0, 0);
    const uint64_t descK = make_smem_desc_sw128(sK, 16, 1024), descQ = make_smem_desc_sw128(sQ, 16, 1024);
    const uint32_t leader = elect_one();
    bool ok = n > 0 && mbar_wait_warp(k_full, 0, abort);
    int sl = 0, ph = 0;
    for (int it = 0; it < n && ok; ++it) {
      const int b = it & 1;
      if (it >= 2) ok = mbar_wait_warp(s_empty + 8 * b, ((it >> 1) - 1) & 1, abort);
      if (ok) ok = mbar_wait_warp(q_full + 8 * sl, ph, abort);
      if (!ok) break;
      tc_fence_after_sync();
#pragma unroll
      for (int h = 0; h < Cfg::kSub; ++h)
        umma_ss4(tmem + b * kTile, desc_advance(descK, h * Cfg::kSubBytes), desc_advance(descQ, sl * Cfg::kTileBytes + h * Cfg::kSubBytes),
                 idesc, h > 0 ? 1u : 0u, leader);
      umma_commit(s_full + 8 * b, leader);
      umma_commit(q_empty + 8 * sl, leader);
      if (++sl == NQ) { sl = 0; ph ^= 1; }
    }
  } else if (warp == 3) {
    // ---------------- -LSE*log2(e) of every step, fetched one step ahead ----------------
    int qt = qt0, hd = hd0;
    auto fetch = [&](int qt_, int hd_, float (&v)[kTile / 32]) {
#pragma unroll
      for (int k = 0; k < kTile / 32; ++k) {
        const int q = row0 + qt_ * kTile + lane + 32 * k;
        v[k] = q < qend ? a.LSE[(size_t)(hq0 + hd_) * a.Nrow + tok0 + q] * -1.4426950408889634f : -INFINITY;
      }
    };
    float cur[kTile / 32], nxt[kTile / 32];
    bool ok = true;
    if (n > 0) fetch(qt, hd, cur);
    for (int it = 0; it < n; ++it) {
      const int b = it & 1;
      if (++hd == a.G) { hd = 0; --qt; }
      if (it + 1 < n) fetch(qt, hd, nxt);
      if (it >= 2) ok = mbar_wait_warp(s_empty + 8 * b, ((it >> 1) - 1) & 1, abort);
      if (!ok) break;
#pragma unroll
      for (int k = 0; k < kTile / 32; ++k) { st_nl2[b * kTile + lane + 32 * k] = cur[k]; cur[k] = nxt[k]; }
      __syncwarp();
      if (lane == 0) mbar_arrive(s_full + 8 * b);
    }
  } else if (warp >= 4) {
    // ---------------- exponentials: warpgroup `wg` takes query columns [64*wg, 64*wg+64) of every step ----------------
    const int wg = (warp - 4) >> 2, quad = warp & 3;
    const uint32_t S_addr = tmem + ((uint32_t)(quad * 32) << 16) + wg * 64;
    const float c = a.scale_log2;
    const uint64_t c2 = f2_pack(c, c);
    uint64_t acc[2] = {0ull, 0ull};
    int qt = qt0, hd = hd0;
    bool ok = true;
    for (int it = 0; it < n; ++it) {
      const int b = it & 1;
      const int q0 = row0 + qt * kTile + wg * 64;         // query of this warpgroup's first column
      const int lo = row0 + quad * 32 + lane - q0;        // columns below it do not see the key
      const int hi = qend - q0;                           // columns from it on do not exist, or see the key compressed
      const bool masked = row0 + quad * 32 + 31 > q0 || hi < 64;   // the same for the warp
      ok = mbar_wait_warp(s_full + 8 * b, (it >> 1) & 1, abort);
      if (!ok) break;
      tc_fence_after_sync();
      const float4* nl2 = reinterpret_cast<const float4*>(st_nl2 + b * kTile + wg * 64);
      // columns [first, first + n) of scores in s; where some of them are hidden from some lanes, by a selection: what a hidden query
      // holds, NaN or infinity, does not enter
      auto columns = [&](const auto& s, int first, int n, auto hidden) {
#pragma unroll
        for (int v = 0; v < n / 4; ++v) {
          const float4 nl = nl2[first / 4 + v];
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const int i = 4 * v + 2 * z;
            const uint64_t x = f2_fma(f2_pack(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), c2, z ? f2_pack(nl.z, nl.w) : f2_pack(nl.x, nl.y));
            float e0, e1;
            f2_unpack(x, e0, e1);
            e0 = ex2(e0);
            e1 = ex2(e1);
            if (decltype(hidden)::value && (first + i < lo || first + i >= hi)) e0 = 0.f;
            if (decltype(hidden)::value && (first + i + 1 < lo || first + i + 1 >= hi)) e1 = 0.f;
            acc[z] = f2_add(acc[z], f2_pack(e0, e1));
          }
        }
      };
      // A step that every lane sees whole goes straight through (a test per element costs more than the exponentials: with a branch for every
      // four, 32K took a seventh longer); in the others sixteen columns at a time are left out, taken whole or tested.
      if (!masked) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t s[32];
          tmem_ld32(S_addr + b * kTile + h * 32, s);
          tmem_wait_ld();
          columns(s, 32 * h, 32, std::false_type());
        }
      } else {
        const int lo0 = row0 + quad * 32 - q0;   // of lane 0
#pragma unroll 1
        for (int k = 0; k < 64; k += 16) {
          if (k + 16 <= lo0 || k >= hi) continue;
          uint32_t s[16];
          tmem_ld16(S_addr + b * kTile + k, s);
          tmem_wait_ld();
          if (k >= lo0 + 31 && k + 16 <= hi) columns(s, k, 16, std::false_type());
          else columns(s, k, 16, std::true_type());
        }
      }
      tc_fence_before_sync();
      mbar_arrive(s_empty + 8 * b);
      if (++hd == a.G) { hd = 0; --qt; }
    }
    float x0, x1, x2, x3;
    f2_unpack(acc[0], x0, x1);
    f2_unpack(acc[1], x2, x3);
    ctl.part[wg][quad * 32 + lane] = (x0 + x1) + (x2 + x3);
  }

  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, Cfg::kCols);
  if (tid < kTile) ctl.part[0][tid] += ctl.part[1][tid];
  if (a.split > 1) cluster_sync();
  if (rank == 0) {
    float* out = a.weight + (size_t)bh * a.Nrow + tok0;
    if (tid < kTile && row0 + tid < key_end) {
      float sum = ctl.part[0][tid];
      for (int r = 1; r < a.split; ++r) sum += ld_cluster(&ctl.part[0][tid], r);
      out[row0 + tid] = sum;
    }
    if (tile == 0)
      for (int i = tid; i < p.S; i += Cfg::kThreads) out[i] = 0.f;
  }
  if (a.split > 1) cluster_sync();   // rank 0 has read the other CTAs' sums: they may leave
  if (tid == 0 && ctl.abort) atomicExch(a.status, (int)LRSA_ERR_TIMEOUT);
}

// CTAs that share a key tile, by the time in steps (two CTAs on an SM; start and end of a CTA cost about five): the work spread over
// the slots, and half of the last CTA.  us at 1 | 2 | 4 | 8: 8/8 heads, d = 64, 4K tokens 14 | 17 | 25 | 44; 28/4, d = 128: 1777 (windows of 512)
// 48 | 31 | 25 | 25, 4K 51 | 47 | 47 | 53, 8K (1024) 168 | 135 | 131 | 149, 16K 271 | 240 | 250 | 292, 32K 503 | 482 | 508 | 581; 16/2, d = 64, two
// sequences of 11K (windows of 333) 54 | 54 | 63 | 91; 32/8, 20K (512) 183 | 189 | 231 | 343.
int weights_split(long long items, long long pairs) {
  const double n = (double)pairs / items, slots = 2 * kSms;
  int best = 1;
  double least = -1;
  for (int c = 1; c <= 8; c *= 2) {
    const double cost = items * (n + 5.0 * c) / slots + 0.5 * (n / c + 5.0);
    if (least < 0 || cost < least) { least = cost; best = c; }
  }
  return best;
}

template <int D, int NSEQ>
int launch_weights_t(const Geom& whole, const SeqBatch& b, const __nv_bfloat16* Q, const __nv_bfloat16* K, const float* LSE,
                     float* weight, int* status, bool clear, cudaStream_t st) {
  using Cfg = WgtCfg<D>;
  WgtMaps<NSEQ> m;
  WgtArgs<NSEQ> a;
  const long long BHq = (long long)whole.B * whole.Hq, BHkv = (long long)whole.B * whole.Hkv;
  long long items = 0, pairs = 0;
  for (int s = 0; s < b.n; ++s) {
    const Geom& g = b.g[s];
    const size_t sh = (size_t)g.tok0 * D;
    int r = make_tmap_bf16(&m.q[s], Q + sh, D, g.N, BHq, kTile, g.Nrow);
    if (r == LRSA_OK) r = make_tmap_bf16(&m.k[s], K + sh, D, g.N, BHkv, kTile, g.Nrow);
    if (r != LRSA_OK) return r;
    a.plan[s] = make_wgt_plan(g);
    a.tok0[s] = g.tok0;
    a.item0[s] = (int)items;
    items += BHkv * a.plan[s].n_tiles;
    const long long L = g.N - g.S < g.L ? g.N - g.S : g.L;   // a tile is seen by half a window's queries, and by the next window's
    pairs += BHkv * a.plan[s].n_tiles * (((g.ndp ? 3 : 1) * L / (2 * kTile) + 1) * g.G);
    a.item0[s + 1] = (int)items;
  }
  a.n_seqs = b.n;
  a.BHkv = (int)BHkv; a.Hq = whole.Hq; a.Hkv = whole.Hkv; a.G = whole.G; a.Nrow = whole.Nrow;
  a.split = weights_split(items, pairs);
  a.LSE = LSE; a.weight = weight; a.scale_log2 = whole.scale * 1.4426950408889634f; a.status = status; a.clear = clear;
  auto kern = lrsa_weights_kernel<D, NSEQ>;
  LRSA_CUDA_CHECK(allow_smem<Cfg::kSmem>(kern));
  LRSA_CUDA_CHECK(launch_dependent(kern, dim3((unsigned)(items * a.split)), dim3(Cfg::kThreads), Cfg::kSmem, st, a.split, m, a));
  launch_counter().n++;
  return LRSA_OK;
}

int launch_weights(const Geom& whole, const __nv_bfloat16* Q, const __nv_bfloat16* K, const float* LSE, float* weight, int* status,
                   cudaStream_t st) {
  SeqBatch b;
  bool clear = true;
  for (SeqBatches it(whole); it.next(&b);) {   // (windows of a few tokens can be too many tiles: found before anything is launched)
    long long items = 0;
    for (int s = 0; s < b.n; ++s) items += (long long)whole.B * whole.Hkv * make_wgt_plan(b.g[s]).n_tiles;
    if (items > 0x7fffffffLL / 8) return LRSA_ERR_UNSUPPORTED;
  }
  for (SeqBatches it(whole); it.next(&b); clear = false) {
    int rc;
    if (whole.d == 128)
      rc = b.n == 1 ? launch_weights_t<128, 1>(whole, b, Q, K, LSE, weight, status, clear, st)
                    : launch_weights_t<128, kMaxSeqs>(whole, b, Q, K, LSE, weight, status, clear, st);
    else
      rc = b.n == 1 ? launch_weights_t<64, 1>(whole, b, Q, K, LSE, weight, status, clear, st)
                    : launch_weights_t<64, kMaxSeqs>(whole, b, Q, K, LSE, weight, status, clear, st);
    if (rc != LRSA_OK) return rc;
  }
  return LRSA_OK;
}

}  // namespace
}  // namespace lrsa

using namespace lrsa;

extern "C" {

int lrsa_attn_weights(const lrsa_params_t* params, const void* Q, const void* K, const float* LSE, float* weight,
                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
  NvtxRange nvtx_range("lrsa_attn_weights");
  launch_counter().n = 0;
  Geom g;
  const int rc = make_geom(params, &g);
  if (rc != LRSA_OK) return rc;
  if (!Q || !K || !LSE || !weight || !workspace) return LRSA_ERR_INVALID_ARG;
  auto mis = [](const void* p, size_t al) { return reinterpret_cast<uintptr_t>(p) % al != 0; };
  if (mis(Q, 16) || mis(K, 16) || mis(LSE, 4) || mis(weight, 4) || mis(workspace, 256)) return LRSA_ERR_INVALID_ARG;
  if (workspace_bytes < sizeof(WsHeader)) return LRSA_ERR_WORKSPACE_TOO_SMALL;
  return launch_weights(g, static_cast<const __nv_bfloat16*>(Q), static_cast<const __nv_bfloat16*>(K), LSE, weight,
                        &static_cast<WsHeader*>(workspace)->status, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
