// Attention of every sequence's next token, or of a tree of drafted ones, over the paged cache.
//
// The queries of a sequence's m new tokens all see the same rows of the cache (paged_sm100.h) and, of the new tokens, those that they
// continue.  A KV head's group of G query heads and the m tokens make m G rows that share K and V:
//   o_r = sum_j p_rj v_j / sum_j p_rj,  p_rj = exp(scale q_r k_j), j over the visible pages and the row's ancestors.
// The pages of a sequence are read once for 16 rows (few rows: bound by memory; paged_few_kernel, warp-level products) or for 128
// (paged_tile_kernel, tcgen05).  Lengths are on the device and differ from sequence to sequence, so the work is dealt out there: every
// CTA runs over the counts of all sequences (32 at a time), finds how many key tiles there are, how many make an even share, and which share
// is its own.  A share is a range of key tiles of one (sequence, KV head, row tile); where an item has more than one, the shares write
// unnormalised results in fp32 and paged_merge_kernel joins them in a fixed order.  Nothing is added up by atomics: results repeat bit by bit.
#include "attn_common_sm100.h"
#include "infer_sm100.h"
#include "paged_sm100.h"

namespace lrsa {
namespace {

using namespace ptx;

constexpr int kKeys = 128;               // key slots of a tile: 128 / page pages
constexpr int kMaxNew = 128;             // new tokens of a sequence: one key tile
constexpr int kPlaces = 2 * kSms;        // shares that the plan aims at: CTAs that run at a time
constexpr int kMaxParts = 2 * kPlaces;   // shares of items that have several: at most two for every place

struct AttendArgs {
  PageGeom p;
  RopeArgs rope;
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* o;
  long long q_head, q_tok, k_head, k_tok, v_head, v_tok, o_head, o_tok;
  const __nv_bfloat16 *k_pages, *v_pages;
  const int32_t* parent;                 // optional
  float *lse, *part;
  int* status;
  int G, max_new, limit, rows, min_share;   // rows: of a row tile
  float scale, scale_log2;
};

// ---- the plan ----
// Key tiles of a sequence: tile 0 holds its new tokens, the others 128 / page of the pages that it sees, one behind the other.
struct SeqPages { int sinks, w, a, b, ra, rb, pages; };   // rows of the sinks, condensed windows, pages and rows of the recent windows
__device__ __forceinline__ SeqPages seq_pages(const PageGeom& p, int n) {
  SeqPages r;
  const int up = (1 << p.shift) - 1;
  r.sinks = min(n, p.S);
  r.w = cut_windows(p, n);
  const int rest = max(n - p.S - r.w * p.L, 0);
  r.ra = min(rest, p.L);
  r.rb = rest - r.ra;
  r.a = (r.ra + up) >> p.shift;
  r.b = (r.rb + up) >> p.shift;
  r.pages = ((r.sinks + up) >> p.shift) + r.w * p.kp + r.a + r.b;
  return r;
}
// Page f of those: its column, and how many of its rows count (0 behind the last one).
__device__ __forceinline__ int page_column(const PageGeom& p, const SeqPages& r, int f, int& count) {
  const int size = 1 << p.shift, front = (r.sinks + size - 1) >> p.shift;
  int rows, col;
  if (f < front) {
    col = f;
    rows = r.sinks - (f << p.shift);
  } else if ((f -= front) < r.w * p.kp) {
    col = p.sp + 2 * p.lp + f;
    rows = p.kp << p.shift == p.K ? size : p.K - ((f - f / p.kp * p.kp) << p.shift);
  } else if ((f -= r.w * p.kp) < r.a) {
    col = p.sp + (r.w & 1) * p.lp + f;
    rows = r.ra - (f << p.shift);
  } else {
    f -= r.a;
    col = p.sp + ((r.w + 1) & 1) * p.lp + f;
    rows = f < r.b ? r.rb - (f << p.shift) : 0;
  }
  count = min(rows, size);
  return count > 0 ? col : 0;
}

struct Share {
  int s, h, rt;         // sequence, KV head, row tile
  int n, m, tok0;       // its counts
  int tiles, t0, t1;    // key tiles of the item, and those of this share
  int part;             // where a partial result goes, -1: the share is the whole item
};
struct SeqWork { SeqCounts c; int tiles, row_tiles; };
__device__ __forceinline__ SeqWork seq_work(const AttendArgs& a, int s) {
  SeqWork w;
  w.c = seq_counts(a.p, s, a.max_new, a.limit);
  const int per = kKeys >> a.p.shift;
  w.tiles = 1 + (seq_pages(a.p, w.c.n).pages + per - 1) / per;
  w.row_tiles = (w.c.m * a.G + a.rows - 1) / a.rows;
  return w;
}
__device__ __forceinline__ int warp_scan(int x, int lane) {   // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}
// Tiles of a share, by a whole warp: an even share of all tiles over the places, and not so few that a share's start outweighs them.
__device__ __forceinline__ int share_tiles(const AttendArgs& a, int lane) {
  long long total = 0;
  for (int s = lane; s < a.p.n_seqs; s += 32) {
    const SeqWork w = seq_work(a, s);
    total += (long long)w.tiles * w.row_tiles;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  total *= a.p.Hkv;
  const long long even = (total + kPlaces - 1) / kPlaces;
  return (int)max(even, (long long)a.min_share);
}
// Share number `at` of all (by a whole warp); false: there are fewer.  Shares of a sequence: row tiles innermost (they read the same
// pages), then heads, then ranges of tiles.
__device__ __forceinline__ bool find_share(const AttendArgs& a, int at, int lane, Share& out) {
  const int size = share_tiles(a, lane);
  int before = 0, parts = 0;
  for (int s0 = 0; s0 < a.p.n_seqs; s0 += 32) {
    SeqWork w = {};
    if (s0 + lane < a.p.n_seqs) w = seq_work(a, s0 + lane);
    const int splits = (w.tiles + size - 1) / size, mine = splits * w.row_tiles * a.p.Hkv;
    const int incl = warp_scan(mine, lane), split_incl = warp_scan(splits > 1 ? mine : 0, lane);
    const unsigned hit = __ballot_sync(0xffffffffu, at < before + incl);
    if (hit) {
      const int l = __ffs(hit) - 1;
      const int row_tiles = __shfl_sync(0xffffffffu, w.row_tiles, l), n = __shfl_sync(0xffffffffu, splits, l);
      const int i = at - before - __shfl_sync(0xffffffffu, incl - mine, l);
      out.s = s0 + l;
      out.n = __shfl_sync(0xffffffffu, w.c.n, l);
      out.m = __shfl_sync(0xffffffffu, w.c.m, l);
      out.tok0 = __shfl_sync(0xffffffffu, w.c.tok0, l);
      out.tiles = __shfl_sync(0xffffffffu, w.tiles, l);
      out.part = n > 1 ? parts + __shfl_sync(0xffffffffu, split_incl - mine, l) + i : -1;
      out.rt = i % row_tiles;
      out.h = i / row_tiles % a.p.Hkv;
      const int split = i / (row_tiles * a.p.Hkv);
      out.t0 = (int)((long long)out.tiles * split / n);
      out.t1 = (int)((long long)out.tiles * (split + 1) / n);
      return true;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
    parts += __shfl_sync(0xffffffffu, split_incl, 31);
  }
  return false;
}

// A partial result: O [D / 4][rows] of four channels each, then the maxima (log2 domain) and sums of the rows.
__device__ __forceinline__ float* part_at(const AttendArgs& a, int part, int D) { return a.part + (size_t)part * a.rows * (D + 2); }

// The new tokens that token i of a sequence sees: bit j for token j, itself included.  By a whole block of at least m threads; a parent that
// is not in front of its token is none.  (Doubling: after round k a token knows its next 2^k ancestors.)
struct Family { uint4 mask[kMaxNew]; int up[kMaxNew]; };
__device__ __forceinline__ void bit_set(uint4& m, int i) {
  const uint32_t b = 1u << (i & 31);
  if (i < 32) m.x |= b; else if (i < 64) m.y |= b; else if (i < 96) m.z |= b; else m.w |= b;
}
__device__ __forceinline__ void find_family(const AttendArgs& a, int tok0, int m, int tid, Family& f) {
  uint4 own = make_uint4(0, 0, 0, 0);
  int up = -1;
  if (tid < m) {
    if (a.parent) {
      up = a.parent[tok0 + tid];
      if (up < 0 || up >= tid) up = -1;
      bit_set(own, tid);
    } else {
      for (int i = 0; i <= tid; ++i) bit_set(own, i);
    }
    f.mask[tid] = own;
    f.up[tid] = up;
  }
  __syncthreads();
  if (!a.parent) return;
  for (int reach = 1; reach < m; reach <<= 1) {
    uint4 o = make_uint4(0, 0, 0, 0);
    int next = -1;
    if (tid < m && up >= 0) { o = f.mask[up]; next = f.up[up]; }
    __syncthreads();
    if (tid < m) {
      own.x |= o.x; own.y |= o.y; own.z |= o.z; own.w |= o.w;
      up = next;
      f.mask[tid] = own;
      f.up[tid] = up;
    }
    __syncthreads();
  }
}
__device__ __forceinline__ int depth_of(const uint4& m) { return __popc(m.x) + __popc(m.y) + __popc(m.z) + __popc(m.w) - 1; }
__device__ __forceinline__ uint32_t word_of(const uint4& m, int i) { return i == 0 ? m.x : i == 1 ? m.y : i == 2 ? m.z : m.w; }

// Infinities and NaN among the values of new tokens: a product would spread them to the rows that do not see them (0 times infinity), so the
// products get zeros there, and each row adds those of the tokens it sees.
__device__ __forceinline__ bool odd_bits(uint32_t pair) { return (pair & 0x7f80u) == 0x7f80u || (pair & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool odd_chunk(const uint4& v) { return odd_bits(v.x) || odd_bits(v.y) || odd_bits(v.z) || odd_bits(v.w); }
__device__ __forceinline__ uint32_t finite_pair(uint32_t u) {
  if ((u & 0x7f80u) == 0x7f80u) u &= 0xffff0000u;
  if ((u & 0x7f800000u) == 0x7f800000u) u &= 0xffffu;
  return u;
}
__device__ __forceinline__ uint4 finite_chunk(uint4 v) { return make_uint4(finite_pair(v.x), finite_pair(v.y), finite_pair(v.z), finite_pair(v.w)); }
// What channel c of the tokens in `seen` adds to a sum of finite values: 0, or an infinity or NaN.
__device__ __noinline__ float odd_values(const AttendArgs& a, const Share& it, uint4 seen, int c) {
  float sum = 0.f;
  const __nv_bfloat16* v = a.v + it.h * a.v_head + it.tok0 * a.v_tok + c;
  for (int i = 0; i < 4; ++i)
    for (uint32_t left = word_of(seen, i); left; left &= left - 1) {
      const float x = __bfloat162float(v[(32 * i + __ffs(left) - 1) * a.v_tok]);
      if (!(fabsf(x) < INFINITY)) sum += x;
    }
  return sum;
}

// One CTA looks at everything that the others take from the device, and writes the status word.
__device__ void check_attend(const AttendArgs& a) {
  const PageGeom& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  bool bad = false;
  for (int s = warp; s < p.n_seqs; s += blockDim.x / 32) {
    const SeqCounts c = seq_counts(p, s, a.max_new, a.limit);
    bad |= !c.ok;
    if (c.m == 0) continue;
    const SeqPages r = seq_pages(p, c.n);
    const int32_t* row = p.table + (size_t)s * p.width;
#pragma unroll 4
    for (int f = lane; f < r.pages; f += 32) {
      int count;
      bad |= (unsigned)row[page_column(p, r, f, count)] >= (unsigned)p.n_pages;
    }
    if (a.parent)
      for (int i = lane; i < c.m; i += 32) {
        const int up = a.parent[c.tok0 + i];
        bad |= up < -1 || up >= i;
      }
  }
  bad = __syncthreads_or(bad);
  if (tid == 0) *a.status = bad ? LRSA_ERR_INVALID_ARG : LRSA_OK;
}

// ---- few rows ----
__device__ __forceinline__ uint4 load_once(const void* p) {   // read once: no place in L1
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Up to 8 NH rows (query heads and tokens) over a share of a sequence's pages, eight warps.  The work is the transfer of K and V; as in the decode kernel of
// the contiguous cache (lrsa_infer.cu) a warp takes 2048 / D keys at a time straight into the registers that the warp-level products want:
//   S^T = K Q^T    lane (g, t) loads chunks t, t + 4, ... of key rows g, g + 8; Q lies in shared memory in the same order
//   O^T = V^T P^T  lane (g, t) loads chunk g (+ 8) of rows 2t, 2t + 1, 2t + 8, 2t + 9; P^T is turned by movmatrix
// A group of sixteen keys lies in one page; the page number of a warp's next group is asked for while this one is computed.  Rows that do
// not count are not read.  The new tokens are a group of their own, for the first warp of the share that holds tile 0.
template <int D, int NH>
__global__ void __launch_bounds__(256, NH == 1 ? 2 : 1) paged_few_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int U = 128 / D;                // 16-key groups per block
  constexpr int KC = D / 32, VC = D / 64, MT = D / 16, NW = 8;
  constexpr int BPT = kKeys / (16 * U);     // blocks per tile
  __shared__ __align__(16) float sm_o[NW][8][D + 4];
  __shared__ float sm_m[NW][8], sm_l[NW][8];
  __shared__ __align__(16) uint4 sm_q[NH][KC][32];
  __shared__ Family fam;
  __shared__ Share sh;
  __shared__ int found, odd;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  wait_front();
  if (blockIdx.x == gridDim.x - 1) { check_attend(a); return; }
  if (warp == 0) {
    Share mine;
    const bool ok = find_share(a, blockIdx.x, lane, mine);
    if (lane == 0) { found = ok; sh = mine; odd = 0; }
  }
  __syncthreads();
  if (!found) return;
  const Share it = sh;
  const int R = it.m * a.G;
  find_family(a, it.tok0, it.m, tid, fam);
  for (int i = tid; i < NH * KC * 32; i += 256) {   // Q of row 8h + g: the chunks that this lane takes of every key row
    const int h = i / (KC * 32), j = i / 32 % KC, r = 8 * h + (i & 31) / 4, c = (i & 3) + 4 * j;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (r < R) {
      const int tok = r / a.G, head = r - tok * a.G;
      const __nv_bfloat16* row = a.q + (it.h * a.G + head) * a.q_head + (it.tok0 + tok) * a.q_tok;
      x = a.rope.half > 0 ? rotated_chunk(row, c, it.n + depth_of(fam.mask[tok]), a.rope) : *reinterpret_cast<const uint4*>(row + 8 * c);
    }
    sm_q[h][j][i & 31] = x;
  }
  __syncthreads();
  float o[NH][MT][4];        // tile 4j + f: channels 8(g + 8j) + 2f, + 1 of rows 2t, 2t + 1
  float m[NH][2], l[NH][2];  // rows 2t, 2t + 1: maximum (the warp's), sum (this lane's keys)
#pragma unroll
  for (int h = 0; h < NH; ++h) {
    m[h][0] = m[h][1] = -INFINITY;
    l[h][0] = l[h][1] = 0.f;
#pragma unroll
    for (int i = 0; i < MT; ++i) o[h][i][0] = o[h][i][1] = o[h][i][2] = o[h][i][3] = 0.f;
  }
  // one block: the keys of a group that count, and those that rows 2t, 2t + 1 of every eight see, as bits
  auto block = [&](uint4 (&kq)[U][2][KC], uint4 (&vq)[U][4][VC], const uint32_t (&there)[U], const uint32_t (&see)[NH][2]) {
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      float s[U][4];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        s[u][0] = s[u][1] = s[u][2] = s[u][3] = 0.f;
#pragma unroll
        for (int j = 0; j < KC; ++j) {
          uint4 q;
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(smem_u32(&sm_q[h][j][lane])));
          mma_16816(s[u], kq[u][0][j].x, kq[u][1][j].x, kq[u][0][j].y, kq[u][1][j].y, q.x, q.y);
          mma_16816(s[u], kq[u][0][j].z, kq[u][1][j].z, kq[u][0][j].w, kq[u][1][j].w, q.z, q.w);
        }
      }
      float mx[2] = {-INFINITY, -INFINITY};   // e = 0, 1: key g, rows 2t, 2t + 1; e = 2, 3: key g + 8
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[u][e] = ((there[u] & see[h][e & 1]) >> (g + 8 * (e >> 1)) & 1u) ? s[u][e] * a.scale_log2 : -INFINITY;
          mx[e & 1] = fmaxf(mx[e & 1], s[u][e]);
        }
      if (__any_sync(0xffffffffu, mx[0] > m[h][0] + 8.f || mx[1] > m[h][1] + 8.f)) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], x));
          const float mn = fmaxf(m[h][e], mx[e]);
          const float f = m[h][e] == -INFINITY ? 0.f : ex2(m[h][e] - mn);
          m[h][e] = mn;
          l[h][e] *= f;
#pragma unroll
          for (int i = 0; i < MT; ++i) { o[h][i][e] *= f; o[h][i][e + 2] *= f; }
        }
      }
      const float ref[2] = {m[h][0] == -INFINITY ? 0.f : m[h][0], m[h][1] == -INFINITY ? 0.f : m[h][1]};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = ex2(s[u][e] - ref[e & 1]);
          l[h][e & 1] += p[e];
        }
        // the probabilities are rounded to bf16 in front of V, as the product asks for (half a step: 2^-8 of a term)
        const uint32_t b0 = transpose_8x8(pack_bf16(p[0], p[1])), b1 = transpose_8x8(pack_bf16(p[2], p[3]));
#pragma unroll
        for (int j = 0; j < VC; ++j)
#pragma unroll
          for (int f = 0; f < 4; ++f) {
            const uint32_t w0 = word_of(vq[u][0][j], f), w1 = word_of(vq[u][1][j], f), w2 = word_of(vq[u][2][j], f), w3 = word_of(vq[u][3][j], f);
            mma_16816(o[h][4 * j + f], __byte_perm(w0, w1, 0x5410), __byte_perm(w0, w1, 0x7632), __byte_perm(w2, w3, 0x5410),
                      __byte_perm(w2, w3, 0x7632), b0, b1);
          }
      }
    }
  };
  if (it.t0 == 0 && warp == 0) {   // the new tokens: at most 16
    uint4 kq[U][2][KC], vq[U][4][VC];
    bool any = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int j = 16 * u + g + 8 * i;
        const __nv_bfloat16* row = a.k + it.h * a.k_head + (it.tok0 + j) * a.k_tok;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          kq[u][i][c] = make_uint4(0, 0, 0, 0);
          if (j < it.m)
            kq[u][i][c] = a.rope.half > 0 ? rotated_chunk(row, t + 4 * c, it.n + depth_of(fam.mask[j]), a.rope)
                                          : *reinterpret_cast<const uint4*>(row + (t + 4 * c) * 8);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = 16 * u + 2 * t + (i & 1) + 8 * (i >> 1);
        const __nv_bfloat16* row = a.v + it.h * a.v_head + (it.tok0 + j) * a.v_tok;
#pragma unroll
        for (int c = 0; c < VC; ++c) {
          uint4 x = make_uint4(0, 0, 0, 0);
          if (j < it.m) x = *reinterpret_cast<const uint4*>(row + (g + 8 * c) * 8);
          any |= odd_chunk(x);
          vq[u][i][c] = finite_chunk(x);
        }
      }
    }
    if (__any_sync(0xffffffffu, any) && lane == 0) odd = 1;
    uint32_t see[NH][2];   // rows 2t, 2t + 1 of every eight
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) see[h][e] = fam.mask[min((8 * h + 2 * t + e) / a.G, it.m - 1)].x;
    uint32_t there[U] = {0xffffu};   // (the first group holds them all)
    block(kq, vq, there, see);
  }
  // the pages
  const SeqPages pg = seq_pages(a.p, it.n);
  const int32_t* table = a.p.table + (size_t)it.s * a.p.width;
  const int in_page = (1 << a.p.shift) - 1;
  const size_t page_rows = (size_t)a.p.Hkv << a.p.shift, head_row = (size_t)it.h << a.p.shift;
  const int b0 = (max(it.t0, 1) - 1) * BPT, b1 = (it.t1 - 1) * BPT;
  struct Group { int page, count, row; };    // page number, rows that count of this group, first row of it in the page
  auto look = [&](int blk, int u) {
    const int slot = (blk * U + u) * 16;
    Group r;
    r.row = slot & in_page;
    const int col = page_column(a.p, pg, slot >> a.p.shift, r.count);
    r.page = table[col];
    r.count = (unsigned)r.page < (unsigned)a.p.n_pages ? min(r.count - r.row, 16) : 0;
    return r;
  };
  uint32_t all_rows[NH][2];
#pragma unroll
  for (int h = 0; h < NH; ++h) all_rows[h][0] = all_rows[h][1] = 0xffffu;
  Group next[U];
  if (b0 + warp < b1) {
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = look(b0 + warp, u);
  }
  for (int blk = b0 + warp; blk < b1; blk += NW) {
    uint4 kq[U][2][KC], vq[U][4][VC];
    uint32_t there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const Group w = next[u];
      there[u] = (1u << max(w.count, 0)) - 1u;
      const size_t at = ((size_t)(w.count > 0 ? w.page : 0) * page_rows + head_row + w.row) * D;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = g + 8 * i;
#pragma unroll
        for (int j = 0; j < KC; ++j) {
          kq[u][i][j] = make_uint4(0, 0, 0, 0);
          if (r < w.count) kq[u][i][j] = load_once(a.k_pages + at + r * D + (t + 4 * j) * 8);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 2 * t + (i & 1) + 8 * (i >> 1);
#pragma unroll
        for (int j = 0; j < VC; ++j) {
          vq[u][i][j] = make_uint4(0, 0, 0, 0);
          if (r < w.count) vq[u][i][j] = load_once(a.v_pages + at + r * D + (g + 8 * j) * 8);
        }
      }
    }
    if (blk + NW < b1) {
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = look(blk + NW, u);
    }
    block(kq, vq, there, all_rows);
  }
  // the warps' results meet in shared memory, eight rows at a time
  float* part = it.part >= 0 ? part_at(a, it.part, D) : nullptr;
#pragma unroll
  for (int h = 0; h < NH; ++h) {
    if (8 * h >= R) break;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float lh = l[h][e];
#pragma unroll
      for (int y = 4; y < 32; y <<= 1) lh += __shfl_xor_sync(0xffffffffu, lh, y);
      float* dst = sm_o[warp][2 * t + e];
#pragma unroll
      for (int i = 0; i < MT; ++i)
        *reinterpret_cast<float2*>(dst + 8 * (g + 8 * (i >> 2)) + 2 * (i & 3)) = make_float2(o[h][i][e], o[h][i][e + 2]);
      if (g == 0) { sm_m[warp][2 * t + e] = m[h][e]; sm_l[warp][2 * t + e] = lh; }
    }
    __syncthreads();
    for (int i = tid; i < 8 * (D / 4); i += 256) {
      const int r = i / (D / 4), c4 = i % (D / 4), row = 8 * h + r;
      if (row >= R) continue;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) M = fmaxf(M, sm_m[w][r]);
      const float ref = M == -INFINITY ? 0.f : M;
      float4 ov = make_float4(0.f, 0.f, 0.f, 0.f);
      float ls = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float f = ex2(sm_m[w][r] - ref);
        const float4 x = *reinterpret_cast<const float4*>(&sm_o[w][r][4 * c4]);
        ov.x = fmaf(x.x, f, ov.x); ov.y = fmaf(x.y, f, ov.y); ov.z = fmaf(x.z, f, ov.z); ov.w = fmaf(x.w, f, ov.w);
        ls = fmaf(sm_l[w][r], f, ls);
      }
      const int tok = row / a.G, head = it.h * a.G + row - tok * a.G;
      if (odd) {
        const uint4 seen = fam.mask[tok];
        ov.x += odd_values(a, it, seen, 4 * c4); ov.y += odd_values(a, it, seen, 4 * c4 + 1);
        ov.z += odd_values(a, it, seen, 4 * c4 + 2); ov.w += odd_values(a, it, seen, 4 * c4 + 3);
      }
      if (part) {
        reinterpret_cast<float4*>(part)[c4 * a.rows + row] = ov;
        if (c4 == 0) { part[a.rows * D + row] = M; part[a.rows * (D + 1) + row] = ls; }
      } else {
        const float inv = 1.f / ls;
        *reinterpret_cast<uint2*>(a.o + head * a.o_head + (it.tok0 + tok) * a.o_tok + 4 * c4) =
            make_uint2(pack_bf16(ov.x * inv, ov.y * inv), pack_bf16(ov.z * inv, ov.w * inv));
        if (c4 == 0 && a.lse) a.lse[(size_t)head * a.p.n_new + it.tok0 + tok] = (M + log2f(ls)) * 0.6931471805599453f;
      }
    }
    __syncthreads();
  }
}

// ---- joining the shares ----
// A block takes 256 of the float4 of a split item's result at a time: O of the shares brought to one maximum, added in the order of the shares.
template <int D>
__global__ void __launch_bounds__(256) paged_merge_kernel(const __grid_constant__ AttendArgs a) {
  const int tid = threadIdx.x, lane = tid & 31;
  wait_front();
  const int size = share_tiles(a, lane), groups = a.rows * (D / 4) / 256;
  int parts = 0, items = 0;   // of the sequences before
  int at = blockIdx.x;        // number of (split item, group) that is next
  for (int s0 = 0; s0 < a.p.n_seqs; s0 += 32) {
    SeqWork w = {};
    if (s0 + lane < a.p.n_seqs) w = seq_work(a, s0 + lane);
    const int splits = (w.tiles + size - 1) / size, mine = splits > 1 ? w.row_tiles * a.p.Hkv : 0;
    const int item_incl = warp_scan(mine, lane), part_incl = warp_scan(mine * splits, lane);
    const int here = __shfl_sync(0xffffffffu, item_incl, 31);
    for (; at / groups < items + here; at += gridDim.x) {
      const int i = at / groups - items;
      const int l = __ffs(__ballot_sync(0xffffffffu, i < item_incl)) - 1;
      const int n = __shfl_sync(0xffffffffu, splits, l), row_tiles = __shfl_sync(0xffffffffu, w.row_tiles, l), m = __shfl_sync(0xffffffffu, w.c.m, l);
      const int tok0 = __shfl_sync(0xffffffffu, w.c.tok0, l), k = i - __shfl_sync(0xffffffffu, item_incl - mine, l);
      const int part0 = parts + __shfl_sync(0xffffffffu, part_incl - mine * splits, l) + k, step = row_tiles * a.p.Hkv;
      const int rt = k % row_tiles, h = k / row_tiles;
      const int e = at % groups * 256 + tid, row = e % a.rows, c4 = e / a.rows, r = rt * a.rows + row;
      if (r >= m * a.G) continue;
      float M = -INFINITY;
#pragma unroll 4
      for (int j = 0; j < n; ++j) {
        const float* p = part_at(a, part0 + j * step, D) + a.rows * D + row;
        const float pm = __ldcg(p), pl = __ldcg(p + a.rows);
        if (pl != 0.f) M = fmaxf(M, pm);
      }
      float4 ov = make_float4(0.f, 0.f, 0.f, 0.f);
      float ls = 0.f;
#pragma unroll 4
      for (int j = 0; j < n; ++j) {
        const float* p = part_at(a, part0 + j * step, D);
        const float pm = __ldcg(p + a.rows * D + row), pl = __ldcg(p + a.rows * (D + 1) + row);
        const float4 x = __ldcg(reinterpret_cast<const float4*>(p) + c4 * a.rows + row);
        const float f = pl != 0.f ? ex2(pm - M) : 0.f;   // nothing counted in this share: its maximum says nothing
        if (f != 0.f) { ov.x = fmaf(x.x, f, ov.x); ov.y = fmaf(x.y, f, ov.y); ov.z = fmaf(x.z, f, ov.z); ov.w = fmaf(x.w, f, ov.w); }
        ls = fmaf(pl, f, ls);
      }
      const int tok = r / a.G, head = h * a.G + r - tok * a.G;
      const float inv = 1.f / ls;
      *reinterpret_cast<uint2*>(a.o + head * a.o_head + (tok0 + tok) * a.o_tok + 4 * c4) =
          make_uint2(pack_bf16(ov.x * inv, ov.y * inv), pack_bf16(ov.z * inv, ov.w * inv));
      if (c4 == 0 && a.lse) a.lse[(size_t)head * a.p.n_new + tok0 + tok] = (M + log2f(ls)) * 0.6931471805599453f;
    }
    items += here;
    parts += __shfl_sync(0xffffffffu, part_incl, 31);
  }
}

// ---- many rows ----
template <int D>
struct TileCfg {
  static constexpr int kSub = D / 64;                       // 64-column (128-byte) sub-tiles
  static constexpr int kSubBytes = kTile * 128, kTileBytes = kSub * kSubBytes;
  static constexpr int kStages = D == 64 ? 5 : 2;           // ring slots, K and V in turn
  static constexpr int kQRegion = kTileBytes + 2048;        // the output rows are staged there, padded by 16 bytes each
  static constexpr int kSmem = kQRegion + kStages * kTileBytes + 1024;
  static constexpr uint32_t kColO = 0, kColS = 128, kCols = 256;   // tensor memory: O, and S with P over it
};
struct TileMaps { CUtensorMap k, v; };   // [n_pages * Hkv][page][D], box: 64 channels of a page's rows of a head
struct TileBars { uint64_t q_full, kv_full[5], kv_empty[5], s_full, pv_done, p_full[2]; };

// 128 rows (query heads and tokens) over a share of a sequence's key tiles, two CTAs an SM: the structure of the forward's one-tile form
// (attn_fwd_sm100.cu).  Warp 0 brings the pages of a tile, a TMA box for every page and 64 channels, through a ring; warp 1 issues the products;
// warps 4-7 rotate Q and the new tokens into their operand tiles, then do the softmax, a thread a row.  Pages end where they end: the
// slots behind the last row of a page, or of the sequence, get no weight, and their V rows are set to zero in shared memory (what lies
// there belongs to nobody and may be infinite), by the softmax warps of the few tiles that have such slots.
template <int D>
__global__ void __launch_bounds__(256, 2) paged_tile_kernel(const __grid_constant__ TileMaps maps, const __grid_constant__ AttendArgs a) {
  using Cfg = TileCfg<D>;
  constexpr int NS = Cfg::kStages;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) TileBars bars;
  __shared__ Family fam;
  __shared__ Share sh;
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s, found, odd;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u, sQ = smem0, sRing = smem0 + Cfg::kQRegion;
  if (tid == 0) {
    prefetch_tensormap(&maps.k);
    prefetch_tensormap(&maps.v);
    abort_s = odd = 0;
    mbar_init(smem_u32(&bars.q_full), 1);
    for (int i = 0; i < NS; ++i) { mbar_init(smem_u32(&bars.kv_full[i]), 1); mbar_init(smem_u32(&bars.kv_empty[i]), 1); }
    mbar_init(smem_u32(&bars.s_full), 1);
    mbar_init(smem_u32(&bars.pv_done), 1);
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&bars.p_full[i]), 4);
    fence_barrier_init();
  }
  if (warp == 1) { tmem_alloc(smem_u32(&tmem_base_s), Cfg::kCols); tmem_relinquish(); }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = tmem_base_s;
  wait_front();
  const bool checks = blockIdx.x == gridDim.x - 1;
  if (checks) check_attend(a);
  if (warp == 0) {
    Share mine = {};
    const bool ok = !checks && find_share(a, blockIdx.x, lane, mine);
    if (lane == 0) { found = ok; sh = mine; }
  }
  __syncthreads();
  if (!found) {
    if (warp == 1) tmem_dealloc(tmem, Cfg::kCols);
    return;
  }
  const Share it = sh;
  const int n = it.t1 - it.t0, R = it.m * a.G;
  const bool has_new = it.t0 == 0;
  find_family(a, it.tok0, it.m, tid, fam);
  volatile int* abort = &abort_s;
  const SeqPages pg = seq_pages(a.p, it.n);
  const int shift = a.p.shift, per = kKeys >> shift;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 0) {
      // ---------------- TMA producer: a lane a box ----------------
      const int32_t* table = a.p.table + (size_t)it.s * a.p.width;
      const int pi = lane % per, sub = lane / per;      // page of the tile, 64 channels of its rows (128 / 16 pages times 2: at most 16 lanes)
      int page = 0, i = has_new ? 2 : 0;                // the new tokens' tile is written by the softmax warps
      bool ok = true;
      auto page_at = [&](int tile) {
        int count, x = 0;
        if (sub == 0) x = table[page_column(a.p, pg, (tile - 1) * per + pi, count)];
        x = (unsigned)x < (unsigned)a.p.n_pages ? x : 0;
        return __shfl_sync(0xffffffffu, x, pi);
      };
      int next = i < 2 * n ? page_at(it.t0 + (i >> 1)) : 0;
      for (; i < 2 * n; ++i) {
        const int slot = i % NS;
        if (!(i & 1)) {
          page = next;
          if (i + 2 < 2 * n) next = page_at(it.t0 + (i >> 1) + 1);
        }
        if (i >= NS) ok = mbar_wait_warp(smem_u32(&bars.kv_empty[slot]), (i / NS - 1) & 1, abort);
        if (!ok) break;
        const uint32_t full = smem_u32(&bars.kv_full[slot]);
        if (lane == 0) mbar_expect_tx(full, Cfg::kTileBytes);
        __syncwarp();
        if (sub < Cfg::kSub)
          tma_load_3d(sRing + slot * Cfg::kTileBytes + sub * Cfg::kSubBytes + (pi << shift) * 128, i & 1 ? &maps.v : &maps.k, sub * 64, 0,
                      page * a.p.Hkv + it.h, full);
      }
      if (!ok) {
        // loads in flight land before the CTA's shared memory is released (a bounded wait)
        for (int back = 1; back <= NS && i - back >= (has_new ? 2 : 0); ++back) {
          const long long t0 = clock64();
          while (!mbar_try_wait(smem_u32(&bars.kv_full[(i - back) % NS]), ((i - back) / NS) & 1) && clock64() - t0 < 2000000) {}
        }
      }
    } else if (warp == 1) {
      // ---------------- issuer: per key tile j  O += P V_j, then S = Q K_{j+1}^T (they run in this order) ----------------
      constexpr uint32_t idesc_qk = make_idesc_bf16(kTile, kTile, 0, 0), idesc_pv = make_idesc_bf16(kTile, D, 0, 1);
      const uint64_t descK0 = make_smem_desc_sw128(sRing, 16, 1024), descV0 = make_smem_desc_sw128(sRing, Cfg::kSubBytes, 1024);
      const uint64_t descQ = make_smem_desc_sw128(sQ, 16, 1024);
      const uint32_t leader = elect_one();
      bool ok = mbar_wait_warp(smem_u32(&bars.q_full), 0, abort);
      for (int j = -1; j < n && ok; ++j) {
        if (j >= 0) {
          const int i = 2 * j + 1, slot = i % NS;
          ok = mbar_wait_warp(smem_u32(&bars.kv_full[slot]), (i / NS) & 1, abort);
          if (!ok) break;
          const uint64_t dV = desc_advance(descV0, slot * Cfg::kTileBytes);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            if (ok) ok = mbar_wait_warp(smem_u32(&bars.p_full[half]), j & 1, abort);
            if (!ok) break;
            tc_fence_after_sync();
            umma_ts4<8, 16, 24, 2048>(tmem + Cfg::kColO, tmem + Cfg::kColS + half * 32, desc_advance(dV, half * 4 * 2048), idesc_pv,
                                     (half > 0 || j > 0) ? 1u : 0u, leader);
          }
          if (!ok) break;
          umma_commit(smem_u32(&bars.pv_done), leader);
          umma_commit(smem_u32(&bars.kv_empty[slot]), leader);
        }
        if (j + 1 < n) {
          const int i = 2 * j + 2, slot = i % NS;
          ok = mbar_wait_warp(smem_u32(&bars.kv_full[slot]), (i / NS) & 1, abort);
          if (!ok) break;
          tc_fence_after_sync();
          const uint64_t dK = desc_advance(descK0, slot * Cfg::kTileBytes);
#pragma unroll
          for (int h = 0; h < Cfg::kSub; ++h)
            umma_ss4(tmem + Cfg::kColS, desc_advance(descQ, h * Cfg::kSubBytes), desc_advance(dK, h * Cfg::kSubBytes), idesc_qk, h > 0 ? 1u : 0u, leader);
          umma_commit(smem_u32(&bars.s_full), leader);
          umma_commit(smem_u32(&bars.kv_empty[slot]), leader);
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ---------------- softmax + epilogue: one thread per row ----------------
    constexpr int CPR = D / 8;
    const int quad = warp & 3, row = quad * 32 + lane, t = tid - 128;
    unsigned char* gen = smem_raw + (smem0 - smem_u32(smem_raw));
    // Operand tiles: chunk c of row r at sub-tile c / 8, row r, place (c % 8) ^ (r % 8)
    auto place = [&](unsigned char* base, int r, int c) {
      return reinterpret_cast<uint4*>(base + (c >> 3) * Cfg::kSubBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4));
    };
    for (int e = t; e < kTile * CPR; e += 128) {
      const int r = e / CPR, c = e % CPR, rr = it.rt * kTile + r;
      uint4 x = make_uint4(0, 0, 0, 0);
      if (rr < R) {
        const int tok = rr / a.G, head = it.h * a.G + rr - tok * a.G;
        const __nv_bfloat16* src = a.q + head * a.q_head + (it.tok0 + tok) * a.q_tok;
        x = a.rope.half > 0 ? rotated_chunk(src, c, it.n + depth_of(fam.mask[tok]), a.rope) : *reinterpret_cast<const uint4*>(src + 8 * c);
      }
      *place(gen, r, c) = x;
    }
    if (has_new) {
      bool any = false;
      for (int e = t; e < kTile * CPR; e += 128) {
        const int r = e / CPR, c = e % CPR;
        uint4 x = make_uint4(0, 0, 0, 0), y = x;
        if (r < it.m) {
          const __nv_bfloat16 *kr = a.k + it.h * a.k_head + (it.tok0 + r) * a.k_tok, *vr = a.v + it.h * a.v_head + (it.tok0 + r) * a.v_tok;
          x = a.rope.half > 0 ? rotated_chunk(kr, c, it.n + depth_of(fam.mask[r]), a.rope) : *reinterpret_cast<const uint4*>(kr + 8 * c);
          y = *reinterpret_cast<const uint4*>(vr + 8 * c);
          any |= odd_chunk(y);
          y = finite_chunk(y);
        }
        *place(gen + Cfg::kQRegion, r, c) = x;
        *place(gen + Cfg::kQRegion + Cfg::kTileBytes, r, c) = y;
      }
      if (any) odd = 1;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // for the products that read them
    asm volatile("bar.sync 2, 128;" ::: "memory");
    if (t == 0) {
      mbar_arrive(smem_u32(&bars.q_full));
      if (has_new) { mbar_arrive(smem_u32(&bars.kv_full[0])); mbar_arrive(smem_u32(&bars.kv_full[1])); }
    }
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16, S_addr = tmem + lane_addr + Cfg::kColS, O_addr = tmem + lane_addr + Cfg::kColO;
    const float c = a.scale_log2;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int j = 0; j < n && ok; ++j) {
      ok = mbar_wait_warp(smem_u32(&bars.s_full), j & 1, abort);
      if (!ok) break;
      tc_fence_after_sync();
      const int tile = it.t0 + j;
      // the slots that this row sees; the same for all rows but among the new tokens
      bool whole = false;
      uint32_t see[4] = {0, 0, 0, 0};
      if (tile == 0) {
        const uint4 own = fam.mask[min((it.rt * kTile + row) / a.G, it.m - 1)];
        see[0] = own.x; see[1] = own.y; see[2] = own.z; see[3] = own.w;
      } else {
        const int f0 = (tile - 1) * per, front = (pg.sinks + (1 << shift) - 1) >> shift, recent = front + pg.w * a.p.kp;
        whole = (f0 >= front && f0 + per <= recent && a.p.kp << shift == a.p.K) || (f0 >= recent && (f0 + per - recent) << shift <= pg.ra);
        if (!whole) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int key = 32 * q + lane;
            int count;
            page_column(a.p, pg, f0 + (key >> shift), count);
            see[q] = __ballot_sync(0xffffffffu, (key & ((1 << shift) - 1)) < count);
          }
          // rows of V that belong to nobody: zero (the product with them starts behind this thread's arrival below)
          const int i = 2 * j + 1, slot = i % NS;
          ok = mbar_wait_warp(smem_u32(&bars.kv_full[slot]), (i / NS) & 1, abort);
          if (!ok) break;
          const uint32_t mine = quad == 0 ? see[0] : quad == 1 ? see[1] : quad == 2 ? see[2] : see[3];
          if (!(mine >> lane & 1u)) {
            unsigned char* v = gen + Cfg::kQRegion + slot * Cfg::kTileBytes + row * 128;
#pragma unroll
            for (int x = 0; x < CPR; ++x) *reinterpret_cast<uint4*>(v + (x >> 3) * Cfg::kSubBytes + ((x & 7) << 4)) = make_uint4(0, 0, 0, 0);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
      }
      uint32_t s[kTile];
#pragma unroll
      for (int h = 0; h < 4; ++h) tmem_ld32(S_addr + h * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[h * 32]));
      tmem_wait_ld();
      if (!whole) {
#pragma unroll
        for (int i = 0; i < kTile; ++i)
          if (!(see[i >> 5] >> (i & 31) & 1u)) s[i] = 0xff800000u;   // -inf
      }
      float mx4[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) mx4[e] = __uint_as_float(s[e]);
#pragma unroll
      for (int i = 4; i + 8 <= kTile; i += 8)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx4[e] = fmaxf(fmaxf(mx4[e], __uint_as_float(s[i + e])), __uint_as_float(s[i + 4 + e]));
#pragma unroll
      for (int e = 0; e < 4; ++e) mx4[e] = fmaxf(mx4[e], __uint_as_float(s[kTile - 4 + e]));
      const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
      // the maximum is only raised when it grew by more than 2^8 (then O is rescaled in tensor memory); -inf while no score has counted
      const bool need = mx > m && (mx - m) * c > 8.f;
      if (j == 0) {
        m = mx;
      } else if (__any_sync(0xffffffffu, need)) {
        ok = mbar_wait_warp(smem_u32(&bars.pv_done), (j - 1) & 1, abort);   // O holds every earlier tile
        if (!ok) break;
        tc_fence_after_sync();
        const float f = need ? ex2((m - mx) * c) : 1.f;
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          uint32_t o[32];
          tmem_ld32(O_addr + q * 32, o);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
          tmem_st32(O_addr + q * 32, o);
        }
        tmem_wait_st();
        l *= f;
        if (need) m = mx;
      }
      const float nmc = m == -INFINITY ? 0.f : -m * c;
      const uint64_t c2 = f2_pack(c, c), nmc2 = f2_pack(nmc, nmc);
      uint64_t sum2 = f2_pack(0.f, 0.f), sum2b = f2_pack(0.f, 0.f);
      // exponentials as a software pipeline, P over S in two halves, as in the forward; P is rounded to bf16 in front of V (half a step: 2^-8 of a term)
      constexpr int kPairs = kTile / 4, kLag = 4;
      uint32_t pk[kPairs];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int ii = 0; ii < kPairs + kLag; ++ii) {
          if (ii < kPairs) {
            const int i = half * kPairs + ii;
            float x0, x1;
            f2_unpack(f2_fma(f2_pack(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), c2, nmc2), x0, x1);
            s[2 * i] = __float_as_uint(ex2_ordered(x0));
            s[2 * i + 1] = __float_as_uint(ex2_ordered(x1));
          }
          if (ii >= kLag) {
            const int i = half * kPairs + ii - kLag;
            const float p0 = __uint_as_float(s[2 * i]), p1 = __uint_as_float(s[2 * i + 1]);
            if (i & 1) sum2 = f2_add(sum2, f2_pack(p0, p1)); else sum2b = f2_add(sum2b, f2_pack(p0, p1));
            pk[ii - kLag] = pack_bf16(p0, p1);
          }
        }
        tmem_st32(S_addr + half * kPairs, pk);
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.p_full[half]));
      }
      sum2 = f2_add(sum2, sum2b);
      float sum0, sum1;
      f2_unpack(sum2, sum0, sum1);
      l += sum0 + sum1;
    }
    if (ok) ok = mbar_wait_warp(smem_u32(&bars.pv_done), (n - 1) & 1, abort);
    if (ok) {
      tc_fence_after_sync();
      const int rr = it.rt * kTile + row;
      const bool there = rr < R, add_odd = has_new && odd;
      const uint4 seen = fam.mask[min(rr / a.G, it.m - 1)];
      float* part = it.part >= 0 ? part_at(a, it.part, D) : nullptr;
      const float inv = 1.0f / l;
      constexpr int kStride = D * 2 + 16;
      unsigned char* stage = gen + quad * 32 * kStride;   // rows of this warp, over Q, which is no longer needed
#pragma unroll
      for (int q = 0; q < D / 32; ++q) {
        uint32_t o[32];
        tmem_ld32(O_addr + q * 32, o);
        tmem_wait_ld();
        if (add_odd) {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) + odd_values(a, it, seen, 32 * q + i));
        }
        if (part) {
#pragma unroll
          for (int v = 0; v < 8; ++v)
            reinterpret_cast<uint4*>(part)[(8 * q + v) * kTile + row] = make_uint4(o[4 * v], o[4 * v + 1], o[4 * v + 2], o[4 * v + 3]);
        } else {
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(o[8 * v + e]) * inv;
            *reinterpret_cast<uint4*>(stage + lane * kStride + (q * 4 + v) * 16) =
                make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
          }
        }
      }
      if (part) {
        part[kTile * D + row] = m * c;
        part[kTile * (D + 1) + row] = l;
      } else {
        if (there && a.lse) {
          const int tok = rr / a.G, head = it.h * a.G + rr - tok * a.G;
          a.lse[(size_t)head * a.p.n_new + it.tok0 + tok] = m * a.scale + logf(l);
        }
        __syncwarp();
        // whole rows: neighbouring lanes take neighbouring chunks
        for (int r = lane / CPR; r < 32; r += 32 / CPR) {
          const int x = it.rt * kTile + quad * 32 + r;
          if (x >= R) break;
          const int tok = x / a.G, head = it.h * a.G + x - tok * a.G;
          reinterpret_cast<uint4*>(a.o + head * a.o_head + (it.tok0 + tok) * a.o_tok)[lane % CPR] =
              *reinterpret_cast<const uint4*>(stage + r * kStride + (lane % CPR) * 16);
        }
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, Cfg::kCols);
  if (tid == 0 && abort_s) atomicExch(a.status, (int)LRSA_ERR_TIMEOUT);
}

bool rows_ok(const lrsa_rows_t* r) {
  return r && r->data && !(reinterpret_cast<uintptr_t>(r->data) & 15u) && r->head_stride % 8 == 0 && r->token_stride % 8 == 0;
}

// Fewest key tiles of a share.
constexpr int kMinShareFew = 4, kMinShareTile = 4;

size_t attend_ws_bytes(int d) { return sizeof(WsHeader) + (size_t)kMaxParts * kTile * (d + 2) * sizeof(float); }

template <int D>
int launch_attend(AttendArgs a, int max_rows, long long n_new, cudaStream_t st) {
  const bool few = max_rows <= 16;
  a.rows = few ? 16 : kTile;
  a.min_share = few ? kMinShareFew : kMinShareTile;
  const long long seqs = a.p.n_seqs < n_new ? a.p.n_seqs : n_new;
  const long long items = a.p.Hkv * (n_new * a.G / a.rows + seqs), grid = kPlaces + items + 1;   // the last one checks
  if (grid > 0x7fffffffLL) return LRSA_ERR_UNSUPPORTED;
  if (few) {
    LRSA_CUDA_CHECK(launch_dependent(max_rows <= 8 ? paged_few_kernel<D, 1> : paged_few_kernel<D, 2>, dim3((unsigned)grid), dim3(256), 0, st, 1, a));
  } else {
    using Cfg = TileCfg<D>;
    TileMaps maps;
    const long long outer = (long long)a.p.n_pages * a.p.Hkv;
    int rc = make_tmap_bf16(&maps.k, a.k_pages, D, 1 << a.p.shift, outer, 1 << a.p.shift);
    if (rc == LRSA_OK) rc = make_tmap_bf16(&maps.v, a.v_pages, D, 1 << a.p.shift, outer, 1 << a.p.shift);
    if (rc != LRSA_OK) return rc;
    LRSA_CUDA_CHECK(cudaFuncSetAttribute(paged_tile_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem));
    LRSA_CUDA_CHECK(launch_dependent(paged_tile_kernel<D>, dim3((unsigned)grid), dim3(256), Cfg::kSmem, st, 1, maps, a));
  }
  launch_counter().n++;
  LRSA_CUDA_CHECK(launch_dependent(paged_merge_kernel<D>, dim3(4 * kSms), dim3(256), 0, st, 1, a));
  launch_counter().n++;
  return LRSA_OK;
}

}  // namespace
}  // namespace lrsa

using namespace lrsa;

extern "C" {

int lrsa_paged_shape(const lrsa_params_t* params, int32_t page, int32_t* table_width, int32_t* w_cap, size_t* workspace_bytes) {
  lrsa_paged_t paged = {};
  paged.page = page;
  Geom g;
  PageGeom p;
  const int rc = make_pages(params, &paged, &g, &p);
  if (rc != LRSA_OK) return rc;
  if (table_width) *table_width = p.width;
  if (w_cap) *w_cap = p.w_cap;
  if (workspace_bytes) *workspace_bytes = attend_ws_bytes(g.d);
  return LRSA_OK;
}

int lrsa_paged_attend(const lrsa_params_t* params, const lrsa_paged_t* paged, const lrsa_rows_t* q, const lrsa_rows_t* k,
                      const lrsa_rows_t* v, const int32_t* cu_new, int32_t n_new, int32_t max_new, const int32_t* parent,
                      const lrsa_rope_t* rope, const lrsa_rows_t* o, float* lse, void* workspace, size_t workspace_bytes,
                      void* cuda_stream) {
  NvtxRange nvtx_range("lrsa_paged_attend");
  launch_counter().n = 0;
  Geom g;
  AttendArgs a = {};
  int rc = make_pages(params, paged, &g, &a.p);
  if (rc != LRSA_OK) return rc;
  rc = make_rope(rope, g.d, &a.rope);
  if (rc != LRSA_OK) return rc;
  if (max_new > kMaxNew) return LRSA_ERR_UNSUPPORTED;
  if (paged->n_pages < 1 || paged->n_seqs < 1 || paged->table_width != a.p.width || !paged->k_pages || !paged->v_pages || !paged->table ||
      !paged->n_tokens || !cu_new || !workspace || n_new < 0 || max_new < 1)
    return LRSA_ERR_INVALID_ARG;
  if (n_new > 0 && (!rows_ok(q) || !rows_ok(k) || !rows_ok(v) || !rows_ok(o))) return LRSA_ERR_INVALID_ARG;
  auto bits = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if (((bits(paged->k_pages) | bits(paged->v_pages)) & 15u) ||
      ((bits(paged->table) | bits(paged->n_tokens) | bits(cu_new) | bits(parent) | bits(lse)) & 3u) || (bits(workspace) & 255u))
    return LRSA_ERR_INVALID_ARG;
  if (workspace_bytes < attend_ws_bytes(g.d)) return LRSA_ERR_WORKSPACE_TOO_SMALL;
  a.p.cu = cu_new; a.p.n_new = n_new;
  a.k_pages = static_cast<const __nv_bfloat16*>(paged->k_pages); a.v_pages = static_cast<const __nv_bfloat16*>(paged->v_pages);
  if (n_new > 0) {
    auto rows = [](const lrsa_rows_t* r) { return static_cast<__nv_bfloat16*>(r->data); };
    a.q = rows(q); a.k = rows(k); a.v = rows(v); a.o = rows(o);
    a.q_head = q->head_stride; a.q_tok = q->token_stride; a.k_head = k->head_stride; a.k_tok = k->token_stride;
    a.v_head = v->head_stride; a.v_tok = v->token_stride; a.o_head = o->head_stride; a.o_tok = o->token_stride;
  }
  a.parent = parent; a.lse = lse;
  a.status = &static_cast<WsHeader*>(workspace)->status;
  a.part = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + sizeof(WsHeader));
  a.G = g.G; a.max_new = max_new;
  a.limit = a.rope.half > 0 ? a.rope.n_pos : 0x7fffffff;
  a.scale = g.scale; a.scale_log2 = g.scale * 1.4426950408889634f;
  const long long max_rows = (long long)max_new * g.G;
  auto st = static_cast<cudaStream_t>(cuda_stream);
  return g.d == 128 ? launch_attend<128>(a, max_rows > 17 ? 17 : (int)max_rows, n_new, st)
                    : launch_attend<64>(a, max_rows > 17 ? 17 : (int)max_rows, n_new, st);
}

}  // extern "C"
