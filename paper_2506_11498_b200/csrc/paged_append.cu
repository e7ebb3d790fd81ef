// New tokens into the paged cache: K rotated on the way, windows that lie far enough back cut to their kept rows.
//
// The cache is condensed for its next token (paged_sm100.h), so tokens n .. n + m - 1 of a sequence cut the windows cut(n) ..
// cut(n + m) - 1: window w is scored with window w + 1 as its reference (Eq. 4-8, the arithmetic and the order of the sums of lrsa_score_select),
// and its top_k rows go to the window's own pages.  Rows of either window come from the pages (positions below n) or from the new
// tokens, so a prompt's windows never enter the pages as a whole.  Tokens from S + cut(n + m) L on, and the sinks, are written to their place.
//
// A cluster of CTAs cuts one window at a time: channel ranges of window w + 1, exchanged through shared memory; spreads of the rows
// of window w into the first CTA's shared memory; that one scores and selects; all of them move kept rows.  Two forms:
//   one launch (every step of a server: a token or some drafts a sequence, as far as the host can tell, one_launch below): a cluster per (sequence,
//     KV head) cuts what there is to cut, mostly nothing, one window after the other, then writes the new rows.  A token of 16 sequences
//     (4 heads, d = 128) 2.6 us in a graph; bound by the launch and four round trips (counts, page number, row, store).
//   several launches (prompts): the new keys rotated into the workspace; a cluster per window, and the rows of sequences that begin; the rows of
//     those that go on.  Bound by reading the windows twice (32K: 9 and 8 of the 33 us of a cut, 7.4 TB/s, mostly L2), and by the chain between:
//     finding the window 1, selecting 4, moving rows 2.5, barriers.
// The counts are on the device: a cluster finds its sequence and window by running over the sequences' counts.
#include "infer_sm100.h"
#include "paged_sm100.h"
#include "weight_select.h"

namespace lrsa {

int make_pages(const lrsa_params_t* params, const lrsa_paged_t* paged, Geom* g, PageGeom* out) {
  const int rc = make_geom(params, g);
  if (rc != LRSA_OK) return rc;
  if (!paged) return LRSA_ERR_INVALID_ARG;
  if (params->n_dense_prev != 1 || params->n_seqs != 0) return LRSA_ERR_UNSUPPORTED;
  const int page = paged->page;
  if (page != 16 && page != 32 && page != 64 && page != 128) return LRSA_ERR_UNSUPPORTED;
  PageGeom a = {};
  a.S = g->S; a.L = g->L; a.K = g->K; a.N = g->N; a.Hkv = g->Hkv;
  a.shift = page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7;
  auto pages = [page](int rows) { return (int)(((long long)rows + page - 1) / page); };
  a.sp = pages(g->S); a.lp = pages(g->L); a.kp = pages(g->K);
  a.w_cap = g->W > 1 ? g->W - 1 : 0;
  const long long width = a.sp + 2LL * a.lp + (long long)a.w_cap * a.kp;
  if (width > 0x7fffff) return LRSA_ERR_UNSUPPORTED;
  a.width = (int)width;
  a.n_pages = paged->n_pages; a.n_seqs = paged->n_seqs;
  a.table = paged->table; a.n_tokens = paged->n_tokens;
  *out = a;
  return LRSA_OK;
}

namespace {

constexpr int kAppThreads = 256;
constexpr int kAppMaxL = 25448;     // spreads of a window in shared memory: 204 KB (and the longest window that lrsa_score_select takes)

struct AppendArgs {
  PageGeom p;
  RopeArgs rope;
  const __nv_bfloat16 *k, *v;
  __nv_bfloat16* turned;                    // two launches and more: [Hkv][n_new][D], the new tokens' keys rotated (null: they come rotated)
  long long k_head, k_tok, v_head, v_tok;   // strides
  int n_rows;                               // rows of k and v
  const int32_t* rows;                      // optional: row of every new token
  __nv_bfloat16 *k_pages, *v_pages;
  int32_t* kept;                            // optional
  WsHeader* head;                           // its status is written by the cluster that checks
  int most, limit;                          // bounds of the counts
  int ddof;
  int clusters;                             // clusters that cut; the one behind them checks, those behind that write the rows of fresh sequences
  int row_blocks;                           // blocks that share the rows of a sequence
};

// What a CTA works on: sequence, head, its counts.
struct Seq {
  int s, h, n, m, tok0;
};

__device__ __forceinline__ int page_of(const AppendArgs& a, int s, int col) { return a.p.table[(size_t)s * a.p.width + col]; }
// (a page number or row that is not usable is reported by the checking cluster; here it becomes one that is)
__device__ __forceinline__ int usable(int i, int n) { return (unsigned)i < (unsigned)n ? i : 0; }

__device__ __forceinline__ int new_row(const AppendArgs& a, const Seq& q, int i) {   // of new token i
  const int t = q.tok0 + i;
  return a.rows ? usable(a.rows[t], a.n_rows) : t;
}

// The row of the token at position p, of K (z = 0) or V.  `turn` (TURN only): K of a new token, still to be rotated.
template <int D, bool TURN>
__device__ __forceinline__ const __nv_bfloat16* token_row(const AppendArgs& a, const Seq& q, int p, int z, bool& turn) {
  turn = false;
  if (p >= q.n) {
    if (!TURN && z == 0 && a.turned) return a.turned + ((size_t)q.h * a.p.n_new + q.tok0 + (p - q.n)) * D;
    const int r = new_row(a, q, p - q.n);
    turn = TURN && z == 0 && a.rope.half > 0;
    return z == 0 ? a.k + q.h * a.k_head + r * a.k_tok : a.v + q.h * a.v_head + r * a.v_tok;
  }
  int row;
  const int col = token_column(a.p, p, row);
  const size_t at = (((size_t)usable(page_of(a, q.s, col), a.p.n_pages) * a.p.Hkv + q.h) << a.p.shift) + row;
  return (z == 0 ? a.k_pages : a.v_pages) + at * D;
}

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmin2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t in_cluster(const void* p, int rank) {
  uint32_t addr;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(ptx::smem_u32(p)), "r"(rank));
  return addr;
}

template <int D>
struct AppendShared {
  float4 sasb[D];                    // [K, V][chunk][pair of channels]: scale, scale, offset, offset
  uint32_t stat[4][D / 2];           // [K, V][min, max]: channel pairs of this CTA's tokens
  uint32_t part[8][2][D / 2];        // of its warps
  float red[4][8];
  SelectShared sel;
};

// Two chunks that make pairs (x, y) with the eight angles of pair i0 on.
__device__ __forceinline__ void turn_chunks(uint4& x, uint4& y, const float* cs, const float* sn) {
  uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float4 c4 = *reinterpret_cast<const float4*>(cs + 4 * h), s4 = *reinterpret_cast<const float4*>(sn + 4 * h);
    const float cc[4] = {c4.x, c4.y, c4.z, c4.w}, ss[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int k = 2 * h + e;
      const float a0 = bf16_lo(xs[k]), a1 = bf16_hi(xs[k]), b0 = bf16_lo(ys[k]), b1 = bf16_hi(ys[k]);
      xs[k] = ptx::pack_bf16(turn(a0, b0, cc[2 * e], -ss[2 * e]), turn(a1, b1, cc[2 * e + 1], -ss[2 * e + 1]));
      ys[k] = ptx::pack_bf16(turn(b0, a0, cc[2 * e], ss[2 * e]), turn(b1, a1, cc[2 * e + 1], ss[2 * e + 1]));
    }
  }
  x = make_uint4(xs[0], xs[1], xs[2], xs[3]);
  y = make_uint4(ys[0], ys[1], ys[2], ys[3]);
}
// The chunks t, t + 4, ... of a row that a lane holds, rotated where they are: a pair's partners are in the same lane when half is a multiple of
// 32 channels.  (Otherwise they are loaded again, with their partners.)
template <int D>
__device__ __forceinline__ void rotate_held(uint4 (&x)[D / 32], const __nv_bfloat16* row, int t, int pos, const RopeArgs& r) {
  constexpr int KC = D / 32;
  if (!r.interleaved && (r.half & 31) == 0) {
    const float *cs = r.cos + (size_t)pos * r.half + 8 * t, *sn = r.sin + (size_t)pos * r.half + 8 * t;
    if (KC == 2 || r.half == 32) {
      turn_chunks(x[0], x[1], cs, sn);
    } else {
      turn_chunks(x[0], x[KC / 2], cs, sn);
      turn_chunks(x[1], x[KC - 1], cs + 32, sn + 32);
    }
  } else {
#pragma unroll
    for (int j = 0; j < KC; ++j) x[j] = rotated_chunk(row, t + 4 * j, pos, r);
  }
}

// Rows of a round: each warp takes eight tokens at a time, four such groups; four lanes share a row.
// What a window's rows are for: their channels' ranges, or their spreads.
template <int D, bool TURN, class F>
__device__ __forceinline__ void walk_window(const AppendArgs& a, const Seq& q, int w, int i0, int i1, F use) {
  constexpr int KC = D / 32, T = 4;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, z = warp & 1, wz = warp >> 1;
  const int p0 = a.p.S + w * a.p.L;
  for (int r0 = i0 + wz * 8 * T; r0 < i1; r0 += 4 * 8 * T) {
    uint4 x[T][KC];
    bool turn[T];
    const __nv_bfloat16* row[T];
#pragma unroll
    for (int s = 0; s < T; ++s) row[s] = token_row<D, TURN>(a, q, p0 + min(r0 + 8 * s + g, i1 - 1), z, turn[s]);
#pragma unroll
    for (int s = 0; s < T; ++s)
#pragma unroll
      for (int j = 0; j < KC; ++j) x[s][j] = *reinterpret_cast<const uint4*>(row[s] + (t + 4 * j) * 8);
    if (TURN && z == 0 && a.rope.half > 0) {
#pragma unroll
      for (int s = 0; s < T; ++s)
        if (turn[s])
          rotate_held<D>(x[s], row[s], t, p0 + min(r0 + 8 * s + g, i1 - 1), a.rope);
    }
    use(r0, x);
  }
}

// Cuts window w of the sequence (all CTAs of the cluster).
template <int D, bool TURN>
__device__ void cut_window(const AppendArgs& a, const Seq& q, int w, int rank, int C, AppendShared<D>& sh, float* spread) {
  constexpr int KC = D / 32, T = 4;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, z = warp & 1;
  const int L = a.p.L, K = a.p.K, per = (L + C - 1) / C, i0 = min(L, rank * per), i1 = min(L, i0 + per);
  if (rank == 0) select_clear(sh.sel);
  // Eq. 4, 5: ranges of window w + 1
  uint32_t mn[KC][4], mx[KC][4];
#pragma unroll
  for (int j = 0; j < KC; ++j)
#pragma unroll
    for (int p = 0; p < 4; ++p) { mn[j][p] = 0x7F807F80u; mx[j][p] = 0xFF80FF80u; }
  walk_window<D, TURN>(a, q, w + 1, i0, i1, [&](int, uint4 (&x)[T][KC]) {
#pragma unroll
    for (int s = 0; s < T; ++s)
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        const uint32_t v[4] = {x[s][j].x, x[s][j].y, x[s][j].z, x[s][j].w};
#pragma unroll
        for (int p = 0; p < 4; ++p) { mn[j][p] = min2(mn[j][p], v[p]); mx[j][p] = max2(mx[j][p], v[p]); }
      }
  });
#pragma unroll
  for (int o = 16; o >= 4; o >>= 1)
#pragma unroll
    for (int j = 0; j < KC; ++j)
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        mn[j][p] = min2(mn[j][p], __shfl_xor_sync(0xffffffffu, mn[j][p], o));
        mx[j][p] = max2(mx[j][p], __shfl_xor_sync(0xffffffffu, mx[j][p], o));
      }
  if (g == 0) {
#pragma unroll
    for (int j = 0; j < KC; ++j) {
      *reinterpret_cast<uint4*>(&sh.part[warp][0][(t + 4 * j) * 4]) = make_uint4(mn[j][0], mn[j][1], mn[j][2], mn[j][3]);
      *reinterpret_cast<uint4*>(&sh.part[warp][1][(t + 4 * j) * 4]) = make_uint4(mx[j][0], mx[j][1], mx[j][2], mx[j][3]);
    }
  }
  __syncthreads();
  for (int v = tid; v < 2 * D; v += kAppThreads) {
    const int zm = v / (D / 2), ch = v % (D / 2), m = zm & 1, zz = zm >> 1;
    uint32_t r = sh.part[zz][m][ch];
#pragma unroll
    for (int k = 1; k < 4; ++k) r = m ? max2(r, sh.part[2 * k + zz][m][ch]) : min2(r, sh.part[2 * k + zz][m][ch]);
    sh.stat[zm][ch] = r;
  }
  cluster_sync();
  for (int v = tid; v < D; v += kAppThreads) {   // channel pairs of K, then of V
    const int zz = v / (D / 2), ch = v % (D / 2);
    uint32_t lo = 0x7F807F80u, hi = 0xFF80FF80u;
    for (int r = 0; r < C; ++r) {
      uint32_t x, y;
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(in_cluster(&sh.stat[2 * zz][ch], r)) : "memory");
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(y) : "r"(in_cluster(&sh.stat[2 * zz + 1][ch], r)) : "memory");
      lo = min2(lo, x);
      hi = max2(hi, y);
    }
    float f[4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {   // a channel with zero range has zbar = 0, i.e. z' = -1/2
      const float a0 = e ? bf16_hi(lo) : bf16_lo(lo), a1 = e ? bf16_hi(hi) : bf16_lo(hi), range = a1 - a0;
      const float inv = range > 0.f ? 1.0f / range : 0.f;
      f[e] = inv;
      f[2 + e] = range > 0.f ? -(0.5f * (a0 + a1)) * inv : -0.5f;
    }
    const int chunk = ch >> 2, p = ch & 3;
    sh.sasb[((zz * KC + (chunk >> 2)) * 4 + p) * 4 + (chunk & 3)] = make_float4(f[0], f[1], f[2], f[3]);
  }
  __syncthreads();
  // Eq. 6, 7: spreads of window w, to the first CTA.  The sums are formed chunk by chunk and the chunks added in a tree over the
  // distances 8, 4, 2, 1, as in lrsa_score_select: equal scores fall on the same side.
  const float inv_dof = 1.0f / (float)(D - a.ddof);
  walk_window<D, TURN>(a, q, w, i0, i1, [&](int r0, uint4 (&x)[T][KC]) {
    float v[T][2], first2[T][2];
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      const int j = KC == 4 ? (k & 1) * 2 + (k >> 1) : k;   // 0, 2, 1, 3
      uint64_t sum2[T], sq2[T];
#pragma unroll
      for (int s = 0; s < T; ++s) sum2[s] = sq2[s] = 0ull;
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const float4 f = sh.sasb[((z * KC + j) * 4 + p) * 4 + t];
        const uint64_t sa = ptx::f2_pack(f.x, f.y), sb = ptx::f2_pack(f.z, f.w);
#pragma unroll
        for (int s = 0; s < T; ++s) {
          const uint32_t u = p == 0 ? x[s][j].x : p == 1 ? x[s][j].y : p == 2 ? x[s][j].z : x[s][j].w;
          const uint64_t z2 = ptx::f2_fma(ptx::f2_pack(bf16_lo(u), bf16_hi(u)), sa, sb);
          sum2[s] = ptx::f2_add(sum2[s], z2);
          sq2[s] = ptx::f2_fma(z2, z2, sq2[s]);
        }
      }
#pragma unroll
      for (int s = 0; s < T; ++s) {
        float x0, x1, y0, y1;
        ptx::f2_unpack(sum2[s], x0, x1);
        ptx::f2_unpack(sq2[s], y0, y1);
        const float a0 = x0 + x1, a1 = y0 + y1;
        if (k == 0) { v[s][0] = a0; v[s][1] = a1; }
        else if (k == 1) { v[s][0] += a0; v[s][1] += a1; }
        else if (k == 2) { first2[s][0] = a0; first2[s][1] = a1; }
        else { v[s][0] += first2[s][0] + a0; v[s][1] += first2[s][1] + a1; }
      }
    }
    // over the four lanes of a row, halving: a lane hands half of its rows to its partner at each level
    const bool up2 = (t & 2) != 0, up1 = (t & 1) != 0;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float send = up2 ? v[s][e] : v[s + 2][e], keep = up2 ? v[s + 2][e] : v[s][e];
        v[s][e] = keep + __shfl_xor_sync(0xffffffffu, send, 2);
      }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float send = up1 ? v[0][e] : v[1][e], keep = up1 ? v[1][e] : v[0][e];
      v[0][e] = keep + __shfl_xor_sync(0xffffffffu, send, 1);
    }
    const int tok = r0 + 8 * ((up2 ? 2 : 0) + (up1 ? 1 : 0)) + g;
    if (tok < i1) {
      const float var = (v[0][1] - v[0][0] * v[0][0] * (1.0f / D)) * inv_dof;
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(in_cluster(spread + (size_t)z * L + tok, 0)), "f"(sqrtf(fmaxf(var, 0.f))) : "memory");
    }
  });
  cluster_sync();   // every spread is in the first CTA
  int32_t* list = reinterpret_cast<int32_t*>(spread + L);   // of the first CTA, over the spreads of V: the kept tokens of the window
  if (rank == 0) {
    // Eq. 7, 8: softmax over the window's tokens, for K and V, added
    float *sk = spread, *sv = spread + L;
    float mk = -INFINITY, mv = -INFINITY;
    for (int i = tid; i < L; i += kAppThreads) { mk = fmaxf(mk, sk[i]); mv = fmaxf(mv, sv[i]); }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      mk = fmaxf(mk, __shfl_xor_sync(0xffffffffu, mk, o));
      mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, o));
    }
    if (lane == 0) { sh.red[0][warp] = mk; sh.red[1][warp] = mv; }
    __syncthreads();
    mk = sh.red[0][0]; mv = sh.red[1][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) { mk = fmaxf(mk, sh.red[0][i]); mv = fmaxf(mv, sh.red[1][i]); }
    float ek = 0.f, ev = 0.f;
    for (int i = tid; i < L; i += kAppThreads) {
      const float x = expf(sk[i] - mk), y = expf(sv[i] - mv);
      sk[i] = x; sv[i] = y;
      ek += x; ev += y;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      ek += __shfl_xor_sync(0xffffffffu, ek, o);
      ev += __shfl_xor_sync(0xffffffffu, ev, o);
    }
    if (lane == 0) { sh.red[2][warp] = ek; sh.red[3][warp] = ev; }
    __syncthreads();
    ek = ev = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) { ek += sh.red[2][i]; ev += sh.red[3][i]; }
    for (int i = tid; i < L; i += kAppThreads) sk[i] = sk[i] / ek + sv[i] / ev;   // (a thread reads back its own only, below)
    __syncthreads();   // the spreads of V are no longer needed
    select_window_by_weight(sh.sel, reinterpret_cast<uint32_t*>(sk), L, K, nullptr, sk, L, list, 0);
  }
  cluster_sync();   // the positions are there
  // kept rows into the window's pages, positions into `kept`
  const int warps = C * (kAppThreads / 32), me = rank * (kAppThreads / 32) + warp;
  constexpr int CPR = D / 8, ROWS = 32 / CPR;   // 16-byte chunks of a row, rows of a warp's access
  const int ch = lane % CPR;
  const uint32_t from = in_cluster(list, 0);
  const int col0 = a.p.sp + 2 * a.p.lp + w * a.p.kp;
  // (four rows a thread at a time: positions, then rows: one by one each is a chain of round trips)
  constexpr int kAhead = 4;
  for (int j0 = me * ROWS + lane / CPR; j0 < K; j0 += kAhead * warps * ROWS) {
    int pos[kAhead], page[kAhead];
    uint4 kx[kAhead], vx[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = min(j0 + u * warps * ROWS, K - 1);
      int i;
      asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(i) : "r"(from + 4 * j) : "memory");
      pos[u] = a.p.S + w * L + min(max(i, 0), L - 1);
      page[u] = page_of(a, q.s, col0 + (j >> a.p.shift));
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      bool turn, none;
      const __nv_bfloat16 *kr = token_row<D, TURN>(a, q, pos[u], 0, turn), *vr = token_row<D, TURN>(a, q, pos[u], 1, none);
      kx[u] = TURN && turn ? rotated_chunk(kr, ch, pos[u], a.rope) : *reinterpret_cast<const uint4*>(kr + 8 * ch);
      vx[u] = *reinterpret_cast<const uint4*>(vr + 8 * ch);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + u * warps * ROWS;
      if (j >= K) break;
      if ((unsigned)page[u] < (unsigned)a.p.n_pages) {
        const size_t at = ((((size_t)page[u] * a.p.Hkv + q.h) << a.p.shift) + (j & ((1 << a.p.shift) - 1))) * CPR + ch;
        reinterpret_cast<uint4*>(a.k_pages)[at] = kx[u];
        reinterpret_cast<uint4*>(a.v_pages)[at] = vx[u];
      }
      if (a.kept && ch == 0) a.kept[(((size_t)q.s * a.p.Hkv + q.h) * a.p.w_cap + w) * K + j] = pos[u];
    }
  }
}

// New tokens that stay: the sinks, and those from position S + cut(n + m) L on.
struct Staying { int sinks, first, count; };
__device__ __forceinline__ Staying staying(const PageGeom& p, int n, int m) {
  Staying r;
  const int end = n + m, whole = p.S + cut_windows(p, end) * p.L;
  r.sinks = max(0, min(end, p.S) - n);
  r.first = max(n, whole);
  r.count = r.sinks + max(0, end - r.first);
  return r;
}
__device__ __forceinline__ int stay_pos(const Staying& r, int n, int j) { return j < r.sinks ? n + j : r.first + (j - r.sinks); }

// A sequence of which no window that may be cut is in the pages: its rows can be written while its windows are cut.
__device__ __forceinline__ bool fresh(const PageGeom& p, int n) { return n <= p.S; }

// Row j of the staying ones of head q.h: chunk ch.
template <int D, bool TURN>
__device__ __forceinline__ void put_row(const AppendArgs& a, const Seq& q, const Staying& r, int j, int ch) {
  constexpr int CPR = D / 8;
  const int p = stay_pos(r, q.n, j), src = new_row(a, q, p - q.n);
  int row;
  const int page = page_of(a, q.s, token_column(a.p, p, row));
  const __nv_bfloat16* vr = a.v + q.h * a.v_head + src * a.v_tok;
  const __nv_bfloat16* kr = !TURN && a.turned ? a.turned + ((size_t)q.h * a.p.n_new + q.tok0 + (p - q.n)) * D : a.k + q.h * a.k_head + src * a.k_tok;
  const uint4 vx = *reinterpret_cast<const uint4*>(vr + 8 * ch);
  const uint4 kx = TURN && a.rope.half > 0 ? rotated_chunk(kr, ch, p, a.rope) : *reinterpret_cast<const uint4*>(kr + 8 * ch);
  if ((unsigned)page >= (unsigned)a.p.n_pages) return;
  const size_t at = ((((size_t)page * a.p.Hkv + q.h) << a.p.shift) + row) * CPR + ch;
  reinterpret_cast<uint4*>(a.k_pages)[at] = kx;
  reinterpret_cast<uint4*>(a.v_pages)[at] = vx;
}

// The staying rows of a sequence, all heads of them, by the blocks first, first + step, ...
template <int D, bool TURN>
__device__ __forceinline__ void put_rows(const AppendArgs& a, Seq& q, int first, int step) {
  constexpr int CPR = D / 8;
  const Staying r = staying(a.p, q.n, q.m);
  const int per_row = a.p.Hkv * CPR;
  const long long items = (long long)r.count * per_row;
#pragma unroll 2
  for (long long i = (long long)first * kAppThreads + threadIdx.x; i < items; i += (long long)step * kAppThreads) {
    const int j = (int)(i / per_row), e = (int)(i - (long long)j * per_row);
    q.h = e / CPR;
    put_row<D, TURN>(a, q, r, j, e % CPR);
  }
}

// One CTA looks at everything that the others take from the device, and writes the status word.  A thread looks at the few pages of
// a sequence with few new tokens, a warp at those of the others.
__device__ void check_append(const AppendArgs& a) {
  const PageGeom& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  bool bad = false;
  if (a.rows) {
    const int end = min(p.cu[p.n_seqs], p.n_new);
    for (int i = tid; i < end; i += kAppThreads) bad |= (unsigned)a.rows[i] >= (unsigned)a.n_rows;
  }
  for (int s0 = warp * 32; s0 < p.n_seqs; s0 += kAppThreads) {
    SeqCounts mine = {0, 0, 0, true};
    if (s0 + lane < p.n_seqs) mine = seq_counts(p, s0 + lane, a.most, a.limit);
    bad |= !mine.ok;
    const bool cuts = cut_windows(p, mine.n + mine.m) > cut_windows(p, mine.n);
    const unsigned many = __ballot_sync(0xffffffffu, mine.m > 64 || cuts);
    // the pages of sequence s, from page `first` of every run on in steps
    auto look = [&](int s, const SeqCounts& c, int first, int step) {
      const int32_t* row = p.table + (size_t)s * p.width;
      auto run = [&](int col, int r0, int r1) {   // rows [r0, r1) of the pages from column col on
        for (int i = (r0 >> p.shift) + first; r0 < r1 && i <= (r1 - 1) >> p.shift; i += step) bad |= (unsigned)row[col + i] >= (unsigned)p.n_pages;
      };
      auto window = [&](int w, int p0, int p1) {   // its tokens among positions [p0, p1)
        const int at = p.S + w * p.L;
        run(p.sp + (w & 1) * p.lp, max(p0 - at, 0), min(p1 - at, p.L));
      };
      const int end = c.n + c.m, w0 = cut_windows(p, c.n), w1 = cut_windows(p, end);
      run(0, c.n, min(end, p.S));
      window(w1, c.n, end);
      window(w1 + 1, c.n, end);
      if (w1 > w0) {
        run(p.sp + 2 * p.lp + w0 * p.kp, 0, ((w1 - w0) * p.kp) << p.shift);
        window(w0, p.S, c.n);
        window(w0 + 1, p.S, c.n);
      }
    };
    if (mine.m > 0 && !(many >> lane & 1u)) look(s0 + lane, mine, 0, 1);
    for (unsigned left = many; left; left &= left - 1) {
      const int l = __ffs(left) - 1;
      SeqCounts c;
      c.n = __shfl_sync(0xffffffffu, mine.n, l);
      c.m = __shfl_sync(0xffffffffu, mine.m, l);
      look(s0 + l, c, lane, 32);
    }
  }
  bad = __syncthreads_or(bad);
  if (tid != 0) return;
  a.head->status = bad ? LRSA_ERR_INVALID_ARG : LRSA_OK;
  if (bad) keep_status(a.head, LRSA_ERR_INVALID_ARG);
}

// The keys of all new tokens rotated, for the forms with several launches: a window's rows are read twice there (for its own scores, and as the
// reference of the one in front), and rotating them each time, in four of eight warps, made the cuts of a 32K prompt of 4 heads, d = 128, take
// 72 us.  This takes 15 (50 MB read, 34 written) and the cuts 38 with the rows beside them; the call 80 before, 51 now.  As in
// lrsa_rotate a thread takes two chunks of a token for all heads, with the angles loaded once.  (Finding the windows' ranges here too, so that a cut
// reads its rows once: 47 us for this and 33 for the cuts.)
template <int D>
__global__ void __launch_bounds__(256) paged_turn_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int UNITS = D / 16, TOK = 256 / UNITS, kAhead = 4;
  const int unit = threadIdx.x % UNITS, mine = blockIdx.x * TOK + threadIdx.x / UNITS;
  const int tok = min(mine, a.p.n_new - 1);   // (the lanes of a warp stay together)
  wait_front();
  const int src = a.rows ? usable(a.rows[tok], a.n_rows) : tok;
  const __nv_bfloat16* row = a.k + src * a.k_tok;
  RotUnit u;
  place_unit(u, unit, a.rope);
  uint4 x[kAhead], y[kAhead];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const __nv_bfloat16* r = row + min(h0 + i, a.p.Hkv - 1) * a.k_head;
      x[i] = __ldcs(reinterpret_cast<const uint4*>(r + 8 * u.c0));
      y[i] = __ldcs(reinterpret_cast<const uint4*>(r + 8 * u.c1));
    }
  };
  load(0);                       // on their way while the token's sequence is looked for
  bool back = false;             // boundaries that go back
  for (int i = threadIdx.x & 31; i < a.p.n_seqs && a.p.n_seqs > 1; i += 32) back |= a.p.cu[i + 1] < a.p.cu[i];
  int lo = 0, hi = a.p.n_seqs;   // the last sequence that begins at or before the token
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.p.cu[mid] <= tok) lo = mid; else hi = mid;
  }
  SeqCounts c;
  auto place = [&](int behind) {   // false: behind the last one, or a sequence with bad counts
    c = seq_counts(a.p, lo, a.most, a.limit, behind);
    const bool there = mine == tok && tok >= c.tok0 && tok < c.tok0 + c.m;
    if (there) load_angles(u, unit, c.n + tok - c.tok0, a.rope);
    return there;
  };
  bool there = place(0);
  if (__any_sync(0xffffffffu, back)) {   // (asked when the angles are on their way)  Then: the last sequence up to which all begin there
    int behind = 0;
    lo = 0;
    for (int s = 0, top = 0; s < a.p.n_seqs && max(top, a.p.cu[s]) <= tok; ++s) {
      lo = s;
      behind = top;
      top = max(top, a.p.cu[s]);
    }
    there = place(behind);
  }
  if (!there) return;
  for (int h0 = 0; h0 < a.p.Hkv; h0 += kAhead) {
    if (h0 > 0) load(h0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (h0 + i >= a.p.Hkv) break;
      u.x = x[i]; u.y = y[i];
      uint4 hi2[2], lo2[2];
      turn_unit(u, hi2, lo2);
      uint4* dst = reinterpret_cast<uint4*>(a.turned + ((size_t)(h0 + i) * a.p.n_new + tok) * D);
      dst[u.c0] = hi2[0];
      dst[u.c1] = hi2[1];
    }
  }
}

// Clusters of C CTAs: ROWS: one for each (sequence, head); otherwise one for each (window to be cut, head).
template <int D, bool ROWS, int PER_SM>
__global__ void __launch_bounds__(kAppThreads, PER_SM) paged_cut_kernel(const __grid_constant__ AppendArgs a, int C) {
  extern __shared__ __align__(16) float app_spread[];   // [2][L]
  __shared__ __align__(16) AppendShared<D> sh;
  const int cluster = blockIdx.x / C, rank = blockIdx.x - cluster * C;
  wait_front();
  Seq q;
  if (cluster >= a.clusters) {
    if (cluster == a.clusters) {
      if (rank == 0) check_append(a);
      return;
    }
    if constexpr (!ROWS) {   // the rows of fresh sequences
      const int blk = blockIdx.x - (a.clusters + 1) * C;
      q.s = blk / a.row_blocks;
      if (q.s >= a.p.n_seqs) return;
      const int first = first_boundary(a.p, q.s);
      const SeqCounts c = seq_counts(a.p, q.s, a.most, a.limit);
      if (!fresh(a.p, c.n) || begins_early(a.p, q.s, first)) return;
      q.n = c.n; q.m = c.m; q.tok0 = c.tok0;
      put_rows<D, false>(a, q, blk - q.s * a.row_blocks, a.row_blocks);
    }
    return;
  }
  int w0, w1;
  if (ROWS) {
    q.s = cluster / a.p.Hkv;
    q.h = cluster - q.s * a.p.Hkv;
    const SeqCounts c = seq_counts(a.p, q.s, a.most, a.limit);   // (should ranges overlap, each sequence has its own rows all the same)
    q.n = c.n; q.m = c.m; q.tok0 = c.tok0;
    w0 = cut_windows(a.p, q.n);
    w1 = cut_windows(a.p, q.n + q.m);
  } else {
    // the cluster's window: every warp runs over the sequences, 32 at a time
    const int unit = cluster / a.p.Hkv, lane = threadIdx.x & 31;
    q.h = cluster - unit * a.p.Hkv;
    q.m = 0;
    int before = 0, behind = 0;
    for (int s0 = 0; s0 < a.p.n_seqs; s0 += 32) {
      SeqCounts c = {};
      if (s0 + lane < a.p.n_seqs) c = seq_counts(a.p, s0 + lane, a.most, a.limit);
      if (c.tok0 < largest_in_front(a.p, s0, lane, behind)) c = SeqCounts{};
      const int cuts = cut_windows(a.p, c.n + c.m) - cut_windows(a.p, c.n);
      int incl = cuts;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, unit < before + incl);
      if (hit) {
        const int l = __ffs(hit) - 1;
        q.s = s0 + l;
        q.n = __shfl_sync(0xffffffffu, c.n, l);
        q.m = __shfl_sync(0xffffffffu, c.m, l);
        q.tok0 = __shfl_sync(0xffffffffu, c.tok0, l);
        w0 = cut_windows(a.p, q.n) + unit - before - __shfl_sync(0xffffffffu, incl - cuts, l);
        break;
      }
      before += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (q.m == 0) return;   // fewer windows than there could have been (the whole cluster)
    w1 = w0 + 1;
  }
  for (int w = w0; w < w1; ++w) {
    cut_window<D, ROWS>(a, q, w, rank, C, sh, app_spread);
    cluster_sync();   // the first CTA's positions have been read
  }
  if (!ROWS) return;
  constexpr int CPR = D / 8;
  const Staying r = staying(a.p, q.n, q.m);
  for (int i = rank * kAppThreads + threadIdx.x; i < r.count * CPR; i += C * kAppThreads) put_row<D, true>(a, q, r, i / CPR, i % CPR);
}

// The rows of prompts that go on from what is in the cache.  Grid: row_blocks for every sequence.
template <int D>
__global__ void __launch_bounds__(kAppThreads) paged_rows_kernel(const __grid_constant__ AppendArgs a) {
  const int blocks = a.row_blocks;
  Seq q;
  q.s = blockIdx.x / blocks;
  wait_front();
  const int first = first_boundary(a.p, q.s);
  const SeqCounts c = seq_counts(a.p, q.s, a.most, a.limit);
  if (fresh(a.p, c.n) || begins_early(a.p, q.s, first)) return;
  q.n = c.n; q.m = c.m; q.tok0 = c.tok0;
  put_rows<D, false>(a, q, blockIdx.x % blocks, blocks);
}

// One launch where the sequences get a few tokens each.  The host knows their sum only, and a sequence that gets most of it has its windows cut one
// after the other by one cluster a head: so neither more than drafts on average, nor so many that one sequence could have more than eight cuts.
// us in a graph, one launch | several, 4 heads, d = 128: drafts, 8 for each of 64 sequences, windows of 128 16.8 | 21.4, of 512 28 | 36; of 256, of 512
// 55 | 97; 60 for each of 8, of 128 18.5 | 18.7.  63 tokens beside a prompt of 500, of 128 63 | 20, of 1024 48 | 53; of 1000 95 | 18 and 23 | 22; of
// 4000 406 | 23 and 127 | 51.  (d = 64, 8 heads: 60 for each of 8 sequences 12.5 | 18; 8 for each of 256, of 128 41 | 67: the price of the rule.)
bool one_launch(const Geom& g, long long n_seqs, long long n_new) { return n_new <= n_seqs || (n_new <= 16 * n_seqs && n_new <= 8LL * g.L); }

bool rows_ok(const lrsa_rows_t* r) {
  return r && r->data && !(reinterpret_cast<uintptr_t>(r->data) & 15u) && r->head_stride % 8 == 0 && r->token_stride % 8 == 0;
}

}  // namespace

size_t append_ws_bytes(const Geom& g, long long n_seqs, long long n_new) {
  return sizeof(WsHeader) + (one_launch(g, n_seqs, n_new) ? 0 : (size_t)n_new * g.Hkv * g.d * sizeof(__nv_bfloat16));
}

}  // namespace lrsa

using namespace lrsa;

extern "C" int lrsa_paged_append(const lrsa_params_t* params, const lrsa_paged_t* paged, const lrsa_rows_t* k_new, const lrsa_rows_t* v_new,
                                 int32_t n_rows, const int32_t* cu_new, int32_t n_new, const int32_t* rows, const lrsa_rope_t* rope,
                                 int32_t* kept, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  NvtxRange nvtx_range("lrsa_paged_append");
  launch_counter().n = 0;
  Geom g;
  AppendArgs a = {};
  int rc = make_pages(params, paged, &g, &a.p);
  if (rc != LRSA_OK) return rc;
  rc = make_rope(rope, g.d, &a.rope);
  if (rc != LRSA_OK) return rc;
  if (paged->n_pages < 1 || paged->n_seqs < 1 || paged->table_width != a.p.width || !paged->k_pages || !paged->v_pages || !paged->n_tokens ||
      !cu_new || !workspace || n_rows < 0 || n_new < 0 || (!rows && n_new > n_rows) || (a.p.width > 0 && !paged->table))
    return LRSA_ERR_INVALID_ARG;
  if (n_new == 0 ? false : !rows_ok(k_new) || !rows_ok(v_new) || n_rows < 1) return LRSA_ERR_INVALID_ARG;
  auto bits = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if (((bits(paged->k_pages) | bits(paged->v_pages)) & 15u) ||
      ((bits(paged->table) | bits(paged->n_tokens) | bits(cu_new) | bits(rows) | bits(kept)) & 3u) || (bits(workspace) & 255u))
    return LRSA_ERR_INVALID_ARG;
  if (workspace_bytes < append_ws_bytes(g, paged->n_seqs, n_new)) return LRSA_ERR_WORKSPACE_TOO_SMALL;
  if (g.L > kAppMaxL) return LRSA_ERR_UNSUPPORTED;
  auto st = static_cast<cudaStream_t>(cuda_stream);
  a.p.cu = cu_new; a.p.n_new = n_new;
  if (n_new > 0) {
    a.k = static_cast<const __nv_bfloat16*>(k_new->data); a.v = static_cast<const __nv_bfloat16*>(v_new->data);
    a.k_head = k_new->head_stride; a.k_tok = k_new->token_stride; a.v_head = v_new->head_stride; a.v_tok = v_new->token_stride;
  }
  a.n_rows = n_rows; a.rows = rows; a.kept = kept;
  a.k_pages = static_cast<__nv_bfloat16*>(paged->k_pages); a.v_pages = static_cast<__nv_bfloat16*>(paged->v_pages);
  a.head = static_cast<WsHeader*>(workspace);
  a.most = n_new;
  a.limit = a.rope.half > 0 && a.rope.n_pos < g.N ? a.rope.n_pos : g.N;
  a.ddof = g.ddof;
  const int n_seqs = paged->n_seqs;
  const bool one = one_launch(g, n_seqs, n_new);
  if (!one && a.rope.half > 0) {
    a.turned = reinterpret_cast<__nv_bfloat16*>(static_cast<unsigned char*>(workspace) + sizeof(WsHeader));
    const int tok = 256 / (g.d / 16);
    LRSA_CUDA_CHECK(launch_dependent(g.d == 128 ? paged_turn_kernel<128> : paged_turn_kernel<64>, dim3((unsigned)((n_new + tok - 1) / tok)), dim3(256), 0,
                                     st, 1, a));
    launch_counter().n++;
  }
  const long long windows = one ? n_seqs : (long long)n_new / g.L + (n_seqs < n_new ? n_seqs : n_new);
  // A window's rows are read by C CTAs, as many as find room at a time; of drafts, where few clusters have a window to cut and the others are soon
  // gone, twice as many.  us, C = 1 | 2 | 4 | 8: 32K prompt, 4 heads, windows of 1024 64 | 51 | 57 | 80; eight prompts of 0.7 to 9K, 8 heads, of 512
  // 50 (40 with three CTAs an SM, below) | 60 | 83 | 140; one of 2295, 4 heads, of 512 22 | 18.5 | 16.3 | 16.0; a token of 16 sequences, 4 heads, of 1024 2.5 | 2.5 | 2.6 | 4.2; up to 16 drafts
  // of 40 sequences, 4 heads, of 512 30 | 24 | 19.6 | 20.8, up to 6 of nine, 8 heads, of 333 27.6 | 22.9 | 19.9 | 21.0.
  const bool drafts = one && n_new > n_seqs;
  // Prompts may fill three CTAs an SM: 208 cuts (13K, 8 heads, windows of 512, d = 64) 27.2 us with one CTA each, 25.6 with two; 100 (25K, 4 heads, of
  // 1024, d = 128) 44.5 with two, 43.4 with four; two prompts of 15 to 20K, 4 heads, of 1024, d = 64, 45.1 and 38.7.
  const size_t smem = (size_t)2 * g.L * sizeof(float);
  const bool fit3 = 3 * (smem + 17 * 1024) <= 227 * 1024;   // three windows' spreads in an SM's shared memory
  const long long room = (drafts ? 4 : !one && fit3 ? 3 : 2) * kSms;
  int C = 1;
  while (C < 8 && windows * g.Hkv * 2 * C <= room && g.L / (2 * C) >= (drafts ? 80 : 128)) C *= 2;
  // The rows of a sequence that stay, in blocks of four rounds: where the cuts leave room, beside them.
  const long long stay = (long long)g.S + 2 * g.L < n_new ? (long long)g.S + 2 * g.L : n_new;
  const int per_block = kAppThreads / (g.d / 8) * 4;
  a.row_blocks = (int)((stay * g.Hkv + per_block - 1) / per_block);
  if (a.row_blocks < 1) a.row_blocks = 1;
  const long long clusters = windows * g.Hkv, row_clusters = one ? 0 : ((long long)a.row_blocks * n_seqs + C - 1) / C;
  const long long grid = (clusters + 1 + row_clusters) * C;
  if (grid > 0x7fffffffLL) return LRSA_ERR_UNSUPPORTED;
  a.clusters = (int)clusters;
  // CTAs of an SM: a cut is a chain of round trips, so where more of them wait than two an SM can hold, three take turns (80 registers instead of
  // 100 and 126, fewer rows on their way in each).  us, two | three: eight prompts of 0.7 to 9K, 8 heads, windows of 512, d = 64 49.6 | 39.4,
  // d = 128 75 | 67; 48 of 0.2 to 0.7K, windows of 128, 72 | 66 and 89 | 82.  Where all are held at once: 32K prompt, 4 heads, d = 128
  // 50 | 57, four of 3 to 8K, 2 heads, windows of 1000, d = 64 20 | 23.
  const bool three = !one && fit3 && clusters * C > 2 * kSms;
  auto cut = g.d == 128 ? (one ? paged_cut_kernel<128, true, 2> : three ? paged_cut_kernel<128, false, 3> : paged_cut_kernel<128, false, 2>)
                        : (one ? paged_cut_kernel<64, true, 2> : three ? paged_cut_kernel<64, false, 3> : paged_cut_kernel<64, false, 2>);
  if (smem > 16 * 1024) LRSA_CUDA_CHECK(allow_smem<2 * kAppMaxL * (int)sizeof(float)>(cut));
  LRSA_CUDA_CHECK(launch_dependent(cut, dim3((unsigned)grid), dim3(kAppThreads), smem, st, C, a, C));
  launch_counter().n++;
  if (one) return LRSA_OK;
  LRSA_CUDA_CHECK(launch_dependent(g.d == 128 ? paged_rows_kernel<128> : paged_rows_kernel<64>, dim3((unsigned)((long long)a.row_blocks * n_seqs)),
                                   dim3(kAppThreads), 0, st, 1, a));
  launch_counter().n++;
  return LRSA_OK;
}
