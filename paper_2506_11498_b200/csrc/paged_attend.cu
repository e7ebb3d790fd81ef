// Attention of every sequence's next token, or of a tree of drafted ones, over the paged cache.
//
// The queries of a sequence's m new tokens all see the same rows of the cache (paged_sm100.h) and, of the new tokens, those that they
// continue.  A KV head's group of G query heads and the m tokens make m G rows that share K and V:
//   o_r = sum_j p_rj v_j / sum_j p_rj,  p_rj = exp(scale q_r k_j), j over the visible pages and the row's ancestors.
// The pages of a sequence are read once for 16 rows (few rows: bound by memory; paged_few_kernel, warp-level products) or for 128 or 256
// (paged_tile_kernel, tcgen05).  Lengths are on the device and differ from sequence to sequence, so the work is dealt out there: the key tiles of
// all (sequence, KV head, row tile) items stand in one line, and every CTA takes an even run of it, which it finds by running over the counts of
// the sequences, 32 at a time.  A run may end one item and begin the next.  Where an item belongs to several CTAs, each writes its unnormalised
// result in fp32 (at most two a CTA: its first item and its last), and paged_merge_kernel joins them in the order of the CTAs.  Nothing is added up
// by atomics: results repeat bit by bit.
// Precision.  A rotated query enters the products as the sum of two bf16 (2^-17 of a channel is lost; rounded to one, the error of o grows from
// 2.0e-3 to 2.9e-3, root mean square, and that of lse to 1e-5 of it), and so does a rotated new key; the keys of the cache are bf16.  Scores, softmax and
// sums are fp32.  The probabilities enter the product with V as sums of two bf16 in the kernel for few, where the tensor pipe has room (16 single tokens
// of 28/4 heads at up to 32K 44.4 and 44.5 us, two tokens each 50.7 and 52.6; the error of o is the rounding of o, 1.7e-3).  In the kernel for many they are
// rounded to bf16 as the forward's are (half a step: 2^-8 of a term; error of o 2.3e-3): in two parts the trees of 32 over 16 sequences took 107 us instead
// of 88, a tree of 48 at 32K 43 instead of 37, the trees at 120K 530 instead of 410.
#include "attn_common_sm100.h"
#include "infer_sm100.h"
#include "paged_sm100.h"

namespace lrsa {
namespace {

using namespace ptx;

constexpr int kKeys = 128;               // key slots of a tile: 128 / page pages
constexpr int kMaxNew = 128;             // new tokens of a sequence: one key tile
constexpr int kFewRows = 16;             // rows of the kernel for few
constexpr int kMaxPlaces = 2 * kSms;     // CTAs of a launch

struct Start;
struct Divided;
struct AttendArgs {
  PageGeom p;
  RopeArgs rope;
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* o;
  long long q_head, q_tok, k_head, k_tok, v_head, v_tok, o_head, o_tok;
  const __nv_bfloat16 *k_pages, *v_pages;
  const int32_t* parent;                 // optional
  float *lse, *part;
  Start* starts;                         // [places]
  Divided* divided;                      // [places]
  // The kernel for many rows: what its first launch makes of the new tokens.
  uint4* family;                         // [n_new] the new tokens that a new token sees
  int* odd;                              // [n_seqs][Hkv] an infinity or NaN among its new values
  __nv_bfloat16 *q_parts[2];             // [Hkv][n_new * G][D] rotated queries: rounded, and what that leaves
  __nv_bfloat16 *k_parts[2], *v_finite;  // [Hkv][n_new][D] the new keys likewise; the new values with zeros for what is not finite
  WsHeader* head;
  int G, max_new, limit, rows;           // rows: of a row tile
  int places, min_tiles, extra;          // CTAs that share the work; the fewest tiles that are a CTA's worth; what beginning an item costs, in tiles
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

// A run of key tiles of one item.
struct Share {
  int s, h, rt;         // sequence, KV head, row tile
  int n, m, tok0;       // its counts
  int t0, t1;           // key tiles
  int part;             // where a partial result goes, -1: the run is the whole item
};
struct SeqWork { SeqCounts c; int tiles, row_tiles; };
__device__ __forceinline__ SeqWork seq_work(const AttendArgs& a, int s, int behind = 0) {
  SeqWork w;
  w.c = seq_counts(a.p, s, a.max_new, a.limit, behind);
  const int per = kKeys >> a.p.shift;
  w.tiles = 1 + (seq_pages(a.p, w.c.n).pages + per - 1) / per;
  w.row_tiles = (w.c.m * a.G + a.rows - 1) / a.rows;
  return w;
}
template <class T>
__device__ __forceinline__ T warp_scan(T x, int lane) {   // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}
// The line of all items, each as long as its tiles and `extra` for what it costs a CTA to begin another one; CTA i takes [i total / ctas,
// (i + 1) total / ctas) of it.
struct Line {
  long long total;
  int ctas;
  __device__ __forceinline__ long long begin(int i) const { return total * i / ctas; }
  // the CTA whose run holds place g
  __device__ __forceinline__ int cta_of(long long g) const { return (int)(((g + 1) * ctas - 1) / total); }
};
// Where a CTA's run begins: item, place in it, length of the run; and the counts of the item's sequence.  Items of a sequence: heads, row tiles
// innermost (they read the same pages).
struct Start { int s, item, t, left, n, m, tok0, tiles; };
// By a whole warp.  left = 0: the CTA has nothing to do.
template <bool BACK>
__device__ __forceinline__ Start find_start_in(const AttendArgs& a, int cta, int lane, Line& line, bool& back) {
  long long total = 0;
  SeqWork w = {};
  back = false;
  if constexpr (BACK) {
    for (int s0 = 0, behind = 0; s0 < a.p.n_seqs; s0 += 32) {
      const int front = largest_in_front(a.p, s0, lane, behind);
      w = SeqWork{};
      if (s0 + lane < a.p.n_seqs) w = seq_work(a, s0 + lane, front);
      total += (long long)(w.tiles + a.extra) * w.row_tiles;
    }
  } else {
    for (int s = lane; s < a.p.n_seqs; s += 32) {
      w = seq_work(a, s);
      total += (long long)(w.tiles + a.extra) * w.row_tiles;
      back |= a.p.cu[s + 1] < a.p.cu[s];
    }
    back = __any_sync(0xffffffffu, back);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  line.total = total * a.p.Hkv;
  line.ctas = (int)min((long long)a.places, (line.total + a.min_tiles - 1) / a.min_tiles);
  Start r = {};
  if (cta >= line.ctas || back) return r;
  const long long g0 = line.begin(cta);
  r.left = (int)(line.begin(cta + 1) - g0);
  long long before = 0;
  for (int s0 = 0, behind = 0; s0 < a.p.n_seqs; s0 += 32) {
    if (a.p.n_seqs > 32) {   // (otherwise w is there)
      const int front = BACK ? largest_in_front(a.p, s0, lane, behind) : 0;
      w = SeqWork{};
      if (s0 + lane < a.p.n_seqs) w = seq_work(a, s0 + lane, front);
    }
    const long long mine = (long long)(w.tiles + a.extra) * w.row_tiles * a.p.Hkv, incl = warp_scan(mine, lane);
    const unsigned hit = __ballot_sync(0xffffffffu, g0 < before + incl);
    if (hit) {
      const int l = __ffs(hit) - 1;
      const long long at = g0 - before - __shfl_sync(0xffffffffu, incl - mine, l);
      r.s = s0 + l;
      r.n = __shfl_sync(0xffffffffu, w.c.n, l);
      r.m = __shfl_sync(0xffffffffu, w.c.m, l);
      r.tok0 = __shfl_sync(0xffffffffu, w.c.tok0, l);
      r.tiles = __shfl_sync(0xffffffffu, w.tiles, l);
      r.item = (int)(at / (r.tiles + a.extra));
      r.t = (int)(at - (long long)r.item * (r.tiles + a.extra));
      return r;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
  r.left = 0;   // (not reached)
  return r;
}
// Where boundaries go back, with those in front of every sequence.  (Apart, so that the others' code stays short.)
__device__ __noinline__ void find_start_back(const AttendArgs& a, int cta, int lane, Line* line, Start* r) {
  bool back;
  *r = find_start_in<true>(a, cta, lane, *line, back);
}
__device__ __forceinline__ Start find_start(const AttendArgs& a, int cta, int lane, Line& line) {
  bool back;
  Start r = find_start_in<false>(a, cta, lane, line, back);
  if (back) {
    Line l;
    Start x;
    find_start_back(a, cta, lane, &l, &x);
    line = l;
    r = x;
  }
  return r;
}
// The runs of a CTA one after the other.  Every role of a CTA has a cursor of its own.
struct Cursor {
  Start at;
  int row_tiles, behind;   // behind: the largest boundary up to that of the sequence at hand
  bool first;
  __device__ __forceinline__ Cursor(const AttendArgs& a, const Start& start) : at(start), behind(start.tok0), first(true) { row_tiles = (at.m * a.G + a.rows - 1) / a.rows; }
  __device__ __forceinline__ bool next(const AttendArgs& a, Share& out) {
    for (;;) {
      if (at.left <= 0) return false;
      while (at.item >= row_tiles * a.p.Hkv) {   // (there is a sequence with work behind this one: left > 0)
        if (++at.s >= a.p.n_seqs) return false;
        const SeqWork w = seq_work(a, at.s, behind);
        behind = max(behind, a.p.cu[at.s]);
        at.n = w.c.n; at.m = w.c.m; at.tok0 = w.c.tok0; at.tiles = w.tiles;
        row_tiles = w.row_tiles;
        at.item = 0;
      }
      out.s = at.s;
      out.h = at.item / row_tiles;
      out.rt = at.item - out.h * row_tiles;
      out.n = at.n; out.m = at.m; out.tok0 = at.tok0;
      const int end = min(at.tiles + a.extra, at.t + at.left);
      out.t0 = max(at.t - a.extra, 0);
      out.t1 = end - a.extra;
      out.part = out.t0 == 0 && out.t1 == at.tiles ? -1 : 2 * (int)blockIdx.x + (first ? 0 : 1);
      at.left -= end - at.t;
      at.t = 0;
      ++at.item;
      first = false;
      if (out.t1 > out.t0) return true;          // (the run may end before the item's first tile)
    }
  }
};

// An item that several CTAs work on, written down by the first of them whose run begins inside of it.
struct alignas(16) Divided {
  int runs, part0, first;   // runs (0: none such); where the first one's result is, and the CTA of the second: those behind it are at 2 first, 2 first + 2, ...
  int h, row0, rows, tok0, pad;   // KV head; first row of the row tile, and how many rows it has
};
// By one thread for every CTA.
__device__ __forceinline__ void note_divided(const AttendArgs& a, const Line& line, const Start& st, int cta) {
  Divided d = {};
  if (st.left > 0 && st.t > a.extra) {
    const long long i0 = line.begin(cta) - st.t;   // the item's place in the line
    const int c0 = line.cta_of(i0 + a.extra), row_tiles = (st.m * a.G + a.rows - 1) / a.rows;
    if (c0 + 1 == cta) {
      d.runs = line.cta_of(i0 + a.extra + st.tiles - 1) - c0 + 1;
      d.part0 = 2 * c0 + (line.begin(c0) >= i0 ? 0 : 1);
      d.first = cta;
      d.h = st.item / row_tiles;
      d.row0 = (st.item - d.h * row_tiles) * a.rows;
      d.rows = min(a.rows, st.m * a.G - d.row0);
      d.tok0 = st.tok0;
    }
  }
  a.divided[cta] = d;
}

// Key tile j of a run in the order in which the kernel for many rows takes them: the new tokens' last (their operands come from the launch in front
// and take three ring slots; the pages' first tile is on its way at once).
__device__ __forceinline__ int tile_of(const Share& it, int j) { return it.t0 > 0 ? it.t0 + j : j + 1 < it.t1 ? j + 1 : 0; }

// A partial result: O [D / 4][rows] of four channels each, then the maxima (log2 domain) and sums of the rows.
__device__ __forceinline__ float* part_at(const AttendArgs& a, int part, int D) { return a.part + (size_t)part * a.rows * (D + 2); }

// The new tokens that token i of a sequence sees: bit j for token j, itself included.  By `threads` threads (128 or more) that meet at named
// barrier 1; a parent that is not in front of its token is none.  (Doubling: after round k a token knows its next 2^k ancestors.)
struct Family { uint4 mask[kMaxNew]; short up[kMaxNew]; };
template <int THREADS>
__device__ __forceinline__ void meet() { asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory"); }
__device__ __forceinline__ void bit_set(uint4& m, int i) {
  const uint32_t b = 1u << (i & 31);
  if (i < 32) m.x |= b; else if (i < 64) m.y |= b; else if (i < 96) m.z |= b; else m.w |= b;
}
template <int THREADS>
__device__ __forceinline__ bool meet_and_vote(bool ok) {   // true: all of them are
  uint32_t bad;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "bar.red.or.pred p, 1, %2, q;\n\tselp.b32 %0, 1, 0, p;\n\t}"
      : "=r"(bad) : "r"(ok ? 0 : 1), "n"(THREADS) : "memory");
  return bad == 0;
}
template <int THREADS>
__device__ __forceinline__ void find_family(const AttendArgs& a, int tok0, int m, int tid, Family& f) {
  uint4 own = make_uint4(0, 0, 0, 0);
  int up = -1;
  if (tid < m) {
    if (a.parent) {
      up = a.parent[tok0 + tid];
      if (up < 0 || up >= tid) up = -1;
      bit_set(own, tid);
    } else {
      auto ones = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; };
      own = make_uint4(ones(tid + 1), ones(tid - 31), ones(tid - 63), ones(tid - 95));
    }
    f.mask[tid] = own;
    f.up[tid] = (short)up;
  }
  meet<THREADS>();
  if (!a.parent) return;
  for (int reach = 1; reach < m; reach <<= 1) {
    uint4 o = make_uint4(0, 0, 0, 0);
    int next = -1;
    if (tid < m && up >= 0) { o = f.mask[up]; next = f.up[up]; }
    meet<THREADS>();
    if (tid < m) {
      own.x |= o.x; own.y |= o.y; own.z |= o.z; own.w |= o.w;
      up = next;
      f.mask[tid] = own;
      f.up[tid] = (short)up;
    }
    meet<THREADS>();
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

// The weight of a part of a row's sum beside the others (l: the sum of its probabilities, x: its maximum above theirs).  Where 32 bits leave it
// none it has the least one there is: in the formula it has some, so an infinity or NaN in it is one of the row's, however the items are dealt out.
__device__ __forceinline__ float weight_of(float l, float x) { return l != 0.f ? fmaxf(ex2(x), 0x1p-149f) : 0.f; }

// The warps of the last launch look at everything that the kernels take from the device, a sequence a warp, the last blocks first.  They read
// inputs only: those were there when the launch in front of this one passed its own wait, so this one need not wait for its end.
__device__ bool attend_inputs_bad(const AttendArgs& a) {
  const PageGeom& p = a.p;
  const int lane = threadIdx.x & 31, warps = blockDim.x / 32;
  bool bad = false;
  for (int s = (gridDim.x - 1 - blockIdx.x) * warps + threadIdx.x / 32; s < p.n_seqs; s += gridDim.x * warps) {
    const SeqCounts c = seq_counts(p, s, a.max_new, a.limit);
    bad |= !c.ok;
    if (c.m == 0) continue;
    const SeqPages r = seq_pages(p, c.n);
    const int32_t* row = p.table + (size_t)s * p.width;
#pragma unroll 8
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
  return bad;
}

// ---- few rows ----
__device__ __forceinline__ uint4 load_once(const void* p) {   // read once: no place in L1
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Up to 8 NH rows (query heads and tokens) over runs of key tiles, eight warps.  The work is the transfer of K and V; as in the decode kernel of
// the contiguous cache (lrsa_infer.cu) a warp takes 2048 / D keys at a time straight into the registers that the warp-level products want:
//   S^T = K Q^T    lane (g, t) loads chunks t, t + 4, ... of key rows g, g + 8; Q lies in shared memory in the same order
//   O^T = V^T P^T  lane (g, t) loads chunk g (+ 8) of rows 2t, 2t + 1, 2t + 8, 2t + 9; P^T is turned by movmatrix
// A group of sixteen keys lies in one page; the page number of a warp's next group is asked for while this one is computed.  Rows that do
// not count are not read.  The new tokens are a group of their own, for the first warp of the run that holds tile 0.
// Bound by the rows it reads where there are many: a token each for 16 sequences of 4K to 32K (28/4 heads, d = 128, 173 MB) takes 44 us, of which the
// loop over the rows is 26 (6.6 TB/s); the others are finding the run 2.2, Q 1.7, joining the warps 3, runs that begin another item up to 5, the merge
// behind it 4.  One sequence of 3.6K (8/8, d = 64) takes 12.5 us in a graph: a chain of round trips, with the merge.
template <int D, int NH>
__global__ void __launch_bounds__(256, NH == 1 ? 2 : 1) paged_few_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int U = 128 / D;                // 16-key groups per block
  constexpr int KC = D / 32, VC = D / 64, MT = D / 16, NW = 8;
  constexpr int BPT = kKeys / (16 * U);     // blocks per tile
  __shared__ __align__(16) float sm_o[NW][8][D + 4];
  __shared__ float sm_m[NW][8], sm_l[NW][8];
  __shared__ __align__(16) uint4 sm_q[2][NH][KC][32];   // rounded, and what that leaves
  __shared__ Family fam;
  __shared__ Start start;
  __shared__ int odd;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  wait_front();
  if (blockIdx.x == 0 && tid == 0) a.head->status = LRSA_OK;
  if (warp == 0) {
    Line line;
    const Start s = find_start(a, blockIdx.x, lane, line);
    if (lane == 0) { start = s; note_divided(a, line, s, blockIdx.x); }
  }
  __syncthreads();
  const bool two = a.rope.half > 0;
  const int in_page = (1 << a.p.shift) - 1;
  const size_t page_rows = (size_t)a.p.Hkv << a.p.shift;
  uint32_t all_rows[NH][2];
  float no_rest[NH][4];
#pragma unroll
  for (int h = 0; h < NH; ++h) {
    all_rows[h][0] = all_rows[h][1] = 0xffffu;
#pragma unroll
    for (int e = 0; e < 4; ++e) no_rest[h][e] = 0.f;
  }
  Cursor cursor(a, start);
  Share it;
  while (cursor.next(a, it)) {
    // the warp's first pages (their numbers are on the way while Q is made)
    const SeqPages pg = seq_pages(a.p, it.n);
    const int32_t* table = a.p.table + (size_t)it.s * a.p.width;
    const size_t head_row = (size_t)it.h << a.p.shift;
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
    Group next[U];
    if (b0 + warp < b1) {
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = look(b0 + warp, u);
    }
    const int R = it.m * a.G;
    if (tid == 0) odd = 0;
    if (it.m > 1) {
      find_family<256>(a, it.tok0, it.m, tid, fam);
    } else {
      if (tid == 0) fam.mask[0] = make_uint4(1, 0, 0, 0);
      __syncthreads();
    }
    for (int i = tid; i < NH * KC * 32; i += 256) {   // Q of row 8h + g: the chunks that this lane takes of every key row
      const int h = i / (KC * 32), j = i / 32 % KC, r = 8 * h + (i & 31) / 4, c = (i & 3) + 4 * j;
      uint4 x = make_uint4(0, 0, 0, 0), rest = x;
      if (r < R) {
        const int tok = r / a.G, head = r - tok * a.G;
        const __nv_bfloat16* row = a.q + (it.h * a.G + head) * a.q_head + (it.tok0 + tok) * a.q_tok;
        x = two ? rotated_chunk(row, c, it.n + depth_of(fam.mask[tok]), a.rope, rest) : *reinterpret_cast<const uint4*>(row + 8 * c);
      }
      sm_q[0][h][j][i & 31] = x;
      sm_q[1][h][j][i & 31] = rest;
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
    auto q_chunk = [&](int which, int h, int j) {
      uint4 q;
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(smem_u32(&sm_q[which][h][j][lane])));
      return q;
    };
    // one block: the keys of a group that count, and those that rows 2t, 2t + 1 of every eight see, as bits; rest: added to the scores of group 0
    auto block = [&](uint4 (&kq)[U][2][KC], uint4 (&vq)[U][4][VC], const uint32_t (&there)[U], const uint32_t (&see)[NH][2], const float (&rest)[NH][4]) {
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        float s[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[u][e] = u == 0 ? rest[h][e] : 0.f;
#pragma unroll
        for (int j = 0; j < KC; ++j) {
          const uint4 q = q_chunk(0, h, j);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            mma_16816(s[u], kq[u][0][j].x, kq[u][1][j].x, kq[u][0][j].y, kq[u][1][j].y, q.x, q.y);
            mma_16816(s[u], kq[u][0][j].z, kq[u][1][j].z, kq[u][0][j].w, kq[u][1][j].w, q.z, q.w);
          }
        }
        if (two) {
#pragma unroll
          for (int j = 0; j < KC; ++j) {
            const uint4 q = q_chunk(1, h, j);
#pragma unroll
            for (int u = 0; u < U; ++u) {
              mma_16816(s[u], kq[u][0][j].x, kq[u][1][j].x, kq[u][0][j].y, kq[u][1][j].y, q.x, q.y);
              mma_16816(s[u], kq[u][0][j].z, kq[u][1][j].z, kq[u][0][j].w, kq[u][1][j].w, q.z, q.w);
            }
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
        // a row's maximum is raised only when it grew by more than 2^8 (then O is rescaled), whatever the other rows' do: a row's bits do not
        // depend on new tokens that it does not see
        if (__any_sync(0xffffffffu, mx[0] > m[h][0] + 8.f || mx[1] > m[h][1] + 8.f)) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], x));
            const float mn = mx[e] > m[h][e] + 8.f ? mx[e] : m[h][e];
            const float f = mn == m[h][e] ? 1.f : m[h][e] == -INFINITY ? 0.f : ex2(m[h][e] - mn);
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
          // P as the sum of two bf16, cut off and what that leaves (not nothing where P is something: an infinite value stays one)
          uint32_t hi[2], lo[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float x = p[2 * i], y = p[2 * i + 1];
            hi[i] = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
            lo[i] = pack_bf16(fmaxf(x - bf16_lo(hi[i]), x * 0x1p-40f), fmaxf(y - bf16_hi(hi[i]), y * 0x1p-40f));
            hi[i] = transpose_8x8(hi[i]);
            lo[i] = transpose_8x8(lo[i]);
          }
#pragma unroll
          for (int j = 0; j < VC; ++j)
#pragma unroll
            for (int f = 0; f < 4; ++f) {
              const uint32_t w0 = word_of(vq[u][0][j], f), w1 = word_of(vq[u][1][j], f), w2 = word_of(vq[u][2][j], f), w3 = word_of(vq[u][3][j], f);
              const uint32_t v0 = __byte_perm(w0, w1, 0x5410), v1 = __byte_perm(w0, w1, 0x7632), v2 = __byte_perm(w2, w3, 0x5410), v3 = __byte_perm(w2, w3, 0x7632);
              mma_16816(o[h][4 * j + f], v0, v1, v2, v3, hi[0], hi[1]);
              mma_16816(o[h][4 * j + f], v0, v1, v2, v3, lo[0], lo[1]);
            }
        }
      }
    };
    if (it.t0 == 0 && warp == 0) {   // the new tokens: at most 16
      uint4 kq[U][2][KC], vq[U][4][VC];
      float rest[NH][4];
#pragma unroll
      for (int h = 0; h < NH; ++h) rest[h][0] = rest[h][1] = rest[h][2] = rest[h][3] = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int c = 0; c < KC; ++c) kq[u][0][c] = kq[u][1][c] = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        uint4 lo[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int j = g + 8 * i;
          const __nv_bfloat16* row = a.k + it.h * a.k_head + (it.tok0 + j) * a.k_tok;
          lo[i] = make_uint4(0, 0, 0, 0);
          if (j < it.m)
            kq[0][i][c] = two ? rotated_chunk(row, t + 4 * c, it.n + depth_of(fam.mask[j]), a.rope, lo[i])
                              : *reinterpret_cast<const uint4*>(row + (t + 4 * c) * 8);
        }
        if (two) {
#pragma unroll
          for (int h = 0; h < NH; ++h) {
            const uint4 q = q_chunk(0, h, c);
            mma_16816(rest[h], lo[0].x, lo[1].x, lo[0].y, lo[1].y, q.x, q.y);
            mma_16816(rest[h], lo[0].z, lo[1].z, lo[0].w, lo[1].w, q.z, q.w);
          }
        }
      }
      bool any = false;
#pragma unroll
      for (int u = 0; u < U; ++u)
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
      if (__any_sync(0xffffffffu, any) && lane == 0) odd = 1;
      uint32_t see[NH][2], there[U] = {0xffffu};   // rows 2t, 2t + 1 of every eight; the first group holds all keys
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) see[h][e] = fam.mask[min((8 * h + 2 * t + e) / a.G, it.m - 1)].x;
      block(kq, vq, there, see, rest);
    }
    // the pages
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
      block(kq, vq, there, all_rows, no_rest);
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
          const float f = weight_of(sm_l[w][r], sm_m[w][r] - ref);
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
}

// ---- joining the runs ----
// A block joins eight rows of a divided item at a time: O of its runs brought to one maximum, added in the order of the CTAs.  The blocks share
// the divided items' row groups, which each of them lists for itself.
template <int D>
__global__ void __launch_bounds__(256, 4) paged_merge_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int kRuns = 64, kRows = 8, kStep = 256 / kRows, kAhead = 4;
  static_assert(D / 4 <= kStep, "a float4 a thread");
  __shared__ float2 ml[kRuns][kRows];      // maxima and sums of so many runs at a time
  __shared__ Divided list[kMaxPlaces];
  __shared__ int before[kMaxPlaces];       // row groups of the items before
  __shared__ int warp_sum[8][2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool bad = attend_inputs_bad(a);
  wait_front();
  if (bad) {
    atomicCAS(&a.head->status, (int)LRSA_OK, (int)LRSA_ERR_INVALID_ARG);
    keep_status(a.head, LRSA_ERR_INVALID_ARG);
  }
  int items = 0, total = 0;
  static_assert(kMaxPlaces <= 512, "two a thread");
  Divided d[2] = {};
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (2 * tid + u < a.places) d[u] = a.divided[2 * tid + u];
  {
    int groups[2], both = 0, n = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      groups[u] = d[u].runs > 0 ? (d[u].rows + kRows - 1) / kRows : 0;
      both += groups[u];
      n += groups[u] > 0;
    }
    const int n_incl = warp_scan(n, lane), g_incl = warp_scan(both, lane);
    if (lane == 31) { warp_sum[warp][0] = n_incl; warp_sum[warp][1] = g_incl; }
    __syncthreads();
    int n0 = n_incl - n, g0 = g_incl - both;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      if (w < warp) { n0 += warp_sum[w][0]; g0 += warp_sum[w][1]; }
      items += warp_sum[w][0];
      total += warp_sum[w][1];
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (groups[u] > 0) { list[n0] = d[u]; before[n0++] = g0; g0 += groups[u]; }
  }
  const int lane_row = tid % kRows, c4 = tid / kRows;   // rows of neighbouring threads are neighbours
  for (int at = blockIdx.x; at < total; at += gridDim.x) {
    __syncthreads();   // the list is there; `ml` has been read
    int lo = 0, hi = items;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before[mid] <= at) lo = mid; else hi = mid;
    }
    const Divided d = list[lo];
    const int row = (at - before[lo]) * kRows + lane_row;
    auto part_of = [&](int i) { return part_at(a, i == 0 ? d.part0 : 2 * (d.first + i - 1), D); };
    auto o_of = [&](int i) {
      return i < d.runs && c4 < D / 4 ? __ldcg(reinterpret_cast<const float4*>(part_of(i)) + c4 * a.rows + row) : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    float M = -INFINITY, ls = 0.f;
    float4 ov = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < d.runs; i0 += kRuns) {
      const int n = min(kRuns, d.runs - i0);
      if (i0 > 0) __syncthreads();
      for (int i = c4; i < n; i += kStep) {
        const float* p = part_of(i0 + i) + a.rows * D + row;
        ml[i][lane_row] = make_float2(__ldcg(p), __ldcg(p + a.rows));
      }
      float4 x[kAhead];   // of the next runs, asked for before the maximum is known
#pragma unroll
      for (int u = 0; u < kAhead; ++u) x[u] = o_of(i0 + u);
      __syncthreads();
      const float was = M;
      for (int i = 0; i < n; ++i) {
        const float2 y = ml[i][lane_row];
        if (y.y != 0.f) M = fmaxf(M, y.x);   // (nothing counted in a run: its maximum says nothing)
      }
      const float f0 = was == -INFINITY ? 0.f : weight_of(1.f, was - M);
      ls *= f0;
      ov.x *= f0; ov.y *= f0; ov.z *= f0; ov.w *= f0;
      for (int i = 0; i < n; i += kAhead) {
        float4 y[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) { y[u] = x[u]; if (i + kAhead < n) x[u] = o_of(i0 + i + kAhead + u); }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          if (i + u >= n) break;
          const float2 w = ml[i + u][lane_row];
          const float f = weight_of(w.y, w.x - M);
          ls = fmaf(w.y, f, ls);
          if (f != 0.f) { ov.x = fmaf(y[u].x, f, ov.x); ov.y = fmaf(y[u].y, f, ov.y); ov.z = fmaf(y[u].z, f, ov.z); ov.w = fmaf(y[u].w, f, ov.w); }
        }
      }
    }
    const int r = d.row0 + row, tok = r / a.G, head = d.h * a.G + r - tok * a.G;
    if (row >= d.rows || c4 >= D / 4) continue;
    const float inv = 1.f / ls;
    *reinterpret_cast<uint2*>(a.o + head * a.o_head + (d.tok0 + tok) * a.o_tok + 4 * c4) =
        make_uint2(pack_bf16(ov.x * inv, ov.y * inv), pack_bf16(ov.z * inv, ov.w * inv));
    if (c4 == 0 && a.lse) a.lse[(size_t)head * a.p.n_new + d.tok0 + tok] = (M + log2f(ls)) * 0.6931471805599453f;
  }
}

// ---- many rows ----
// The operands of the new tokens, once for all CTAs that work on their items (which would each spend 5 to 15 us on it): which new tokens each one
// sees, queries and keys rotated and split in two bf16, values without infinities and NaN.  A block takes a query head of a sequence, or a KV head's
// keys, or its values.  The last blocks find where the runs of the CTAs begin, a warp for each.
template <int D>
__global__ void __launch_bounds__(256) paged_operands_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int UNITS = D / 16, kAhead = 2;
  __shared__ Family fam;
  __shared__ int odd;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  wait_front();
  if (blockIdx.x == 0 && tid == 0) a.head->status = LRSA_OK;
  const int heads = a.p.Hkv * (a.G + 2), plan0 = a.p.n_seqs * heads, s = blockIdx.x / heads, which = blockIdx.x - s * heads;
  if ((int)blockIdx.x >= plan0) {
    const int cta = (blockIdx.x - plan0) * 8 + warp;
    if (cta < a.places) {
      Line line;
      const Start st = find_start(a, cta, lane, line);
      if (lane == 0) { a.starts[cta] = st; note_divided(a, line, st, cta); }
    }
    return;
  }
  const int first = first_boundary(a.p, s);
  const SeqCounts c = seq_counts(a.p, s, a.max_new, a.limit);
  if (begins_early(a.p, s, first) || c.m == 0) return;   // (the whole block)
  const int q_heads = a.p.Hkv * a.G;
  if (which >= q_heads + a.p.Hkv) {
    const int h = which - q_heads - a.p.Hkv;
    if (tid == 0) odd = 0;
    __syncthreads();
    bool any = false;
#pragma unroll 4
    for (int i = tid; i < c.m * (D / 8); i += 256) {
      const int tok = i / (D / 8), ch = i % (D / 8);
      const uint4 y = *reinterpret_cast<const uint4*>(a.v + h * a.v_head + (c.tok0 + tok) * a.v_tok + 8 * ch);
      any |= odd_chunk(y);
      reinterpret_cast<uint4*>(a.v_finite)[((size_t)h * a.p.n_new + c.tok0 + tok) * (D / 8) + ch] = finite_chunk(y);
    }
    if (any) odd = 1;
    __syncthreads();
    if (tid == 0) a.odd[(size_t)s * a.p.Hkv + h] = odd;
    return;
  }
  find_family<256>(a, c.tok0, c.m, tid, fam);
  const bool is_q = which < q_heads, two = a.rope.half > 0;
  const int h = is_q ? which / a.G : which - q_heads, g = which - h * a.G;
  const __nv_bfloat16* src = is_q ? a.q + which * a.q_head + c.tok0 * a.q_tok : a.k + h * a.k_head + c.tok0 * a.k_tok;
  const long long src_tok = is_q ? a.q_tok : a.k_tok;
  // rows of the result: G to a token for the queries
  const size_t row0 = (size_t)h * a.p.n_new * (is_q ? a.G : 1) + (size_t)c.tok0 * (is_q ? a.G : 1) + (is_q ? g : 0);
  __nv_bfloat16 *hi_out = is_q ? a.q_parts[0] : a.k_parts[0], *lo_out = is_q ? a.q_parts[1] : a.k_parts[1];
  for (int i0 = tid; i0 < c.m * UNITS; i0 += kAhead * 256) {
    RotUnit u[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int i = min(i0 + x * 256, c.m * UNITS - 1), tok = i / UNITS;
      load_unit(u[x], src + tok * src_tok, i % UNITS, two ? c.n + depth_of(fam.mask[tok]) : 0, a.rope);
    }
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int i = i0 + x * 256, tok = i / UNITS;
      if (i >= c.m * UNITS) break;
      uint4 hi[2], lo[2];
      turn_unit(u[x], hi, lo);
      const size_t at = (row0 + (size_t)tok * (is_q ? a.G : 1)) * (D / 8);
      reinterpret_cast<uint4*>(hi_out)[at + u[x].c0] = hi[0];
      reinterpret_cast<uint4*>(hi_out)[at + u[x].c1] = hi[1];
      if (two) {
        reinterpret_cast<uint4*>(lo_out)[at + u[x].c0] = lo[0];
        reinterpret_cast<uint4*>(lo_out)[at + u[x].c1] = lo[1];
      }
    }
  }
  if (which == 0 && tid < c.m) a.family[c.tok0 + tid] = fam.mask[tid];
}

template <int D, int TQ>
struct TileCfg {
  static constexpr int kSub = D / 64;                       // 64-column (128-byte) sub-tiles
  static constexpr int kSubBytes = kTile * 128, kTileBytes = kSub * kSubBytes;
  static constexpr int kStages = D == 64 ? 8 : TQ == 1 ? 5 : 3;   // ring slots
  static constexpr int kQRegion = 2 * kTileBytes;           // rounded, and what that leaves
  static constexpr int kRing = TQ * kQRegion, kTail = kRing + kStages * kTileBytes;
  static constexpr int kThreads = 384;
  static constexpr uint32_t kColO = 0, kColS = 256, kCols = 512;   // tensor memory: O of the warpgroups, S with P over it, 128 columns each
};
struct TileMaps {
  CUtensorMap k, v;                // [n_pages * Hkv][page][D], box: 64 channels of a page's rows of a head
  CUtensorMap q[2], kn[2], vn;     // what paged_operands_kernel made, box: 64 channels of 128 rows
};
struct TileTail {                  // behind the operand tiles in shared memory
  uint64_t q_full, q_free, kv_full[8], kv_empty[8], s_full[2], pv_done[2], p_full[2][2];
  Start start;
  uint32_t tmem;
  int abort;
  float2 ml[2][kTile];           // TQ = 1: maxima and sums of the warpgroups' rows
};

// 128 TQ rows (query heads and tokens) over runs of key tiles, one CTA an SM: the structure of the forward (attn_fwd_sm100.cu).  Warp 0 brings Q at
// the start of an item and the key tiles through a ring, of a page tile a TMA box for every page and 64 channels; warp 1 issues the products;
// two warpgroups do the softmax, a thread a row.  S = Q K^T is formed with both parts of Q, for the new tokens (three ring slots) with both of K.
//   TQ = 2: a warpgroup has a row tile, a key tile serves both: per key tile O_t += P_t V_j and then S_t of the next one, for t = 0, 1.
//   TQ = 1: the warpgroups take the key tiles of the one row tile in turns, each with its own S, O, maximum and sum, and their results are
//           joined at the end of an item (both can read all of O in tensor memory).  A tile's chain of products and exponentials takes 2.3 us,
//           so one warpgroup alone would leave the SM waiting: 16 trees of 16 tokens at up to 20K, 16/4 heads, d = 64, 52 us with one, 45 with two (d = 128, 8 of 32/4 at
//           60K: 90 and 89, a tile then takes 1.75 us where its bytes would take 1.46).
// What bounds it.  TQ = 2, d = 128: 2.15 us a key tile (a plain copy's rate would bring it in 1.46, its 48 products take 1.87 at 1965 MHz): beside 128 KB
// of Q the ring has three slots, so K of the next tile but one comes 1.4 us after the slot of V is free, and then its scores take 0.75.  16 trees of 32 tokens at
// up to 32K (28/4) 89 us: launch in front 5, first tile 7, twenty tiles 43 to 60, a second item 8, merge 8.  Four trees of 64 tokens at 120K (32/8): 414 us, at
// 1.65 GHz under the power limit; without the second part of Q 371.
// Pages end where they end: the slots behind the last row of a page, or of the sequence, get no weight, and their V rows are set to zero in
// shared memory (what lies there belongs to nobody and may be infinite) by the softmax warps of the few tiles that have such slots.
template <int D, int TQ>
__global__ void __launch_bounds__(TileCfg<D, TQ>::kThreads, 1) paged_tile_kernel(const __grid_constant__ TileMaps maps, const __grid_constant__ AttendArgs a) {
  using Cfg = TileCfg<D, TQ>;
  constexpr int NS = Cfg::kStages;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  TileTail& sh = *reinterpret_cast<TileTail*>(smem_raw + Cfg::kTail);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sQ = smem_u32(smem_raw), sRing = sQ + Cfg::kRing;
  if (tid == 0) {
    prefetch_tensormap(&maps.k);
    prefetch_tensormap(&maps.v);
    for (int i = 0; i < 2; ++i) { prefetch_tensormap(&maps.q[i]); prefetch_tensormap(&maps.kn[i]); }
    prefetch_tensormap(&maps.vn);
    sh.abort = 0;
    mbar_init(smem_u32(&sh.q_full), 1);
    mbar_init(smem_u32(&sh.q_free), 1);
    for (int i = 0; i < NS; ++i) { mbar_init(smem_u32(&sh.kv_full[i]), 1); mbar_init(smem_u32(&sh.kv_empty[i]), 1); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&sh.s_full[t]), 1);
      mbar_init(smem_u32(&sh.pv_done[t]), 1);
      for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&sh.p_full[t][i]), 4);
    }
    fence_barrier_init();
  }
  if (warp == 1) { tmem_alloc(smem_u32(&sh.tmem), Cfg::kCols); tmem_relinquish(); }
  tc_fence_before_sync();
  wait_front();
  if (tid == 0) {
    sh.start = a.starts[blockIdx.x];
    if (sQ & 1023u) { sh.start.left = 0; sh.abort = 1; }   // (the operand tiles want 1024 bytes, as declared)
  }
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = sh.tmem;
  volatile int* abort = &sh.abort;
  const int shift = a.p.shift, per = kKeys >> shift;
  const bool two = a.rope.half > 0;
  // The ring: a page tile takes two entries (K, V), the new tokens' tile, which is the last of an item's, three (K, rest of K, V).  Entry number i is
  // in slot i % NS, in its i / NS-th use.
  struct Entry {
    int slot, phase;
    __device__ __forceinline__ explicit Entry(int i) : slot(i % NS), phase(i / NS & 1) {}
  };
  Cursor cursor(a, sh.start);
  Share it;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");   // 128 x 72 + 256 x 216 = 384 x 168
    if (warp == 0) {
      // ---------------- TMA producer: a lane a box ----------------
      const int pi = lane % per, sub = lane / per;      // page of the tile, 64 channels of its rows: at most 16 lanes
      int filled = 0, items = 0;                        // entries, items so far
      bool ok = true;
      while (ok && cursor.next(a, it)) {
        const SeqPages pg = seq_pages(a.p, it.n);
        const int32_t* table = a.p.table + (size_t)it.s * a.p.width;
        auto page_at = [&](int tile) {
          int count, x = 0;
          if (sub == 0) x = table[page_column(a.p, pg, (tile - 1) * per + pi, count)];
          x = (unsigned)x < (unsigned)a.p.n_pages ? x : 0;
          return __shfl_sync(0xffffffffu, x, pi);
        };
        // into the next entry: waits for its slot, announces the bytes; lane 0 has done so when the others go on
        auto claim = [&](const Entry& e) {
          if (ok && filled >= NS) ok = mbar_wait_warp(smem_u32(&sh.kv_empty[e.slot]), e.phase ^ 1, abort);
          if (ok && lane == 0) mbar_expect_tx(smem_u32(&sh.kv_full[e.slot]), Cfg::kTileBytes);
          __syncwarp();
          return ok;
        };
        // Q: both parts of the row tiles that have rows (rows behind the item's are other items', and nobody looks at theirs)
        const int row_tiles = TQ == 2 && it.rt * a.rows + kTile < it.m * a.G ? 2 : 1, parts = two ? 2 : 1;
        if (items > 0) ok = mbar_wait_warp(smem_u32(&sh.q_free), (items - 1) & 1, abort);
        if (!ok) break;
        ++items;
        if (lane == 0) mbar_expect_tx(smem_u32(&sh.q_full), row_tiles * parts * Cfg::kTileBytes);
        __syncwarp();
        if (lane < row_tiles * parts * Cfg::kSub) {
          const int x = lane % Cfg::kSub, lo = lane / Cfg::kSub % parts, t = lane / Cfg::kSub / parts;
          tma_load_3d(sQ + t * Cfg::kQRegion + lo * Cfg::kTileBytes + x * Cfg::kSubBytes, &maps.q[lo], x * 64, it.tok0 * a.G + it.rt * a.rows + t * kTile,
                      it.h, smem_u32(&sh.q_full));
        }
        // (Bringing the rows of later tiles into L2 ahead of the ring was slower: 92.0 us without, 93.1 one tile ahead, 99.1 four, of sixteen trees of 32
        // tokens at up to 32K.)
        int next = max(it.t0, 1) < it.t1 ? page_at(max(it.t0, 1)) : 0;
        for (int tile = max(it.t0, 1); tile < it.t1 && ok; ++tile) {
          const int page = next;
          if (tile + 1 < it.t1) next = page_at(tile + 1);
#pragma unroll
          for (int which = 0; which < 2; ++which) {
            const Entry e(filled);
            if (!claim(e)) break;
            if (sub < Cfg::kSub)
              tma_load_3d(sRing + e.slot * Cfg::kTileBytes + sub * Cfg::kSubBytes + (pi << shift) * 128, which ? &maps.v : &maps.k, sub * 64, 0,
                          page * a.p.Hkv + it.h, smem_u32(&sh.kv_full[e.slot]));
            ++filled;
          }
        }
        if (it.t0 == 0 && ok) {
          for (int i = 0; i < 3; ++i, ++filled) {
            const Entry e(filled);
            if (!claim(e)) break;
            const CUtensorMap* map = i == 0 ? &maps.kn[0] : i == 1 ? &maps.kn[two ? 1 : 0] : &maps.vn;   // (unrotated keys leave no rest: never multiplied)
            if (lane < Cfg::kSub)
              tma_load_3d(sRing + e.slot * Cfg::kTileBytes + lane * Cfg::kSubBytes, map, lane * 64, it.tok0, it.h, smem_u32(&sh.kv_full[e.slot]));
          }
        }
      }
      if (!ok) {
        // loads in flight land before the CTA's shared memory is released (bounded waits)
        auto drain = [&](uint64_t* bar, int phase) {
          const long long t0 = clock64();
          while (!mbar_try_wait(smem_u32(bar), phase) && clock64() - t0 < 2000000) {}
        };
        if (items > 0) drain(&sh.q_full, (items - 1) & 1);
        for (int i = max(0, filled - NS); i < filled; ++i) drain(&sh.kv_full[Entry(i).slot], Entry(i).phase);
      }
    } else if (warp == 1) {
      // ---------------- issuer (the products run in the order of issue, sm100_ptx.h) ----------------
      constexpr uint32_t idesc_qk = make_idesc_bf16(kTile, kTile, 0, 0), idesc_pv = make_idesc_bf16(kTile, D, 0, 1);
      const uint64_t descK0 = make_smem_desc_sw128(sRing, 16, 1024), descV0 = make_smem_desc_sw128(sRing, Cfg::kSubBytes, 1024);
      const uint64_t descQ0 = make_smem_desc_sw128(sQ, 16, 1024);
      const uint32_t leader = elect_one();
      bool ok = true;
      int q_phase = 0, base = 0, count[2] = {0, 0};   // base: the item's first entry; count: tiles so far of each warpgroup, the parity of its P
      while (ok && cursor.next(a, it)) {
        const int n = it.t1 - it.t0, tiles = TQ == 2 && it.rt * a.rows + kTile < it.m * a.G ? 2 : 1;
        ok = mbar_wait_warp(smem_u32(&sh.q_full), q_phase, abort);
        q_phase ^= 1;
        // S_t (+)= part `lo` of Q_q times the K tile in a slot
        auto product = [&](int t, int q, int lo, int slot, bool more) {
          const uint64_t dQ = desc_advance(descQ0, q * Cfg::kQRegion + lo * Cfg::kTileBytes), dK = desc_advance(descK0, slot * Cfg::kTileBytes);
#pragma unroll
          for (int h = 0; h < Cfg::kSub; ++h)
            umma_ss4(tmem + Cfg::kColS + t * kTile, desc_advance(dQ, h * Cfg::kSubBytes), desc_advance(dK, h * Cfg::kSubBytes), idesc_qk,
                     more || h > 0 ? 1u : 0u, leader);
        };
        auto is_new = [&](int j) { return tile_of(it, j) == 0; };
        auto entry_k = [&](int j) { return Entry(base + 2 * j); };
        auto entry_rest = [&](int j) { return Entry(base + 2 * j + 1); };
        auto entry_v = [&](int j) { return Entry(base + 2 * j + (is_new(j) ? 2 : 1)); };
        auto wait_k = [&](int j) {
          ok = mbar_wait_warp(smem_u32(&sh.kv_full[entry_k(j).slot]), entry_k(j).phase, abort);
          if (ok && is_new(j)) ok = mbar_wait_warp(smem_u32(&sh.kv_full[entry_rest(j).slot]), entry_rest(j).phase, abort);
          return ok;
        };
        auto scores = [&](int j, int t, int q) {
          tc_fence_after_sync();
          product(t, q, 0, entry_k(j).slot, false);
          if (two) {
            product(t, q, 1, entry_k(j).slot, true);
            if (is_new(j)) product(t, q, 0, entry_rest(j).slot, true);
          }
          umma_commit(smem_u32(&sh.s_full[t]), leader);
        };
        auto free_k = [&](int j) {
          umma_commit(smem_u32(&sh.kv_empty[entry_k(j).slot]), leader);
          if (is_new(j)) umma_commit(smem_u32(&sh.kv_empty[entry_rest(j).slot]), leader);
          if (j + 1 == n) umma_commit(smem_u32(&sh.q_free), leader);   // the item's last scores: the next Q may come while this item ends
        };
        // O_t += P_t V_j, as the halves of P come
        auto values = [&](int j, int t, bool more) {
          const uint64_t dV = desc_advance(descV0, entry_v(j).slot * Cfg::kTileBytes);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            if (ok) ok = mbar_wait_warp(smem_u32(&sh.p_full[t][half]), count[t] & 1, abort);
            if (!ok) return;
            tc_fence_after_sync();
            umma_ts4<8, 16, 24, 2048>(tmem + Cfg::kColO + t * kTile, tmem + Cfg::kColS + t * kTile + half * 32, desc_advance(dV, half * 4 * 2048),
                                     idesc_pv, half > 0 || more ? 1u : 0u, leader);
          }
          umma_commit(smem_u32(&sh.pv_done[t]), leader);
          ++count[t];
        };
        if constexpr (TQ == 2) {
          for (int j = -1; j < n && ok; ++j) {
            if (j >= 0) ok = mbar_wait_warp(smem_u32(&sh.kv_full[entry_v(j).slot]), entry_v(j).phase, abort);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              if (!ok || t >= tiles) break;
              if (j >= 0) values(j, t, j > 0);
              if (ok && j + 1 < n && (t > 0 || wait_k(j + 1))) scores(j + 1, t, t);
            }
            if (!ok) break;
            if (j >= 0) umma_commit(smem_u32(&sh.kv_empty[entry_v(j).slot]), leader);
            if (j + 1 < n) free_k(j + 1);
          }
        } else {
          // tile j is warpgroup j % 2's; two tiles' scores are ahead of the values
          for (int j = -2; j < n && ok; ++j) {
            if (j >= 0) {
              ok = mbar_wait_warp(smem_u32(&sh.kv_full[entry_v(j).slot]), entry_v(j).phase, abort);
              if (!ok) break;
              if (j & 1) values(j, 1, j > 1); else values(j, 0, j > 1);
              if (!ok) break;
              umma_commit(smem_u32(&sh.kv_empty[entry_v(j).slot]), leader);
            }
            if (j + 2 < n) {
              if (!wait_k(j + 2)) break;
              scores(j + 2, j & 1, 0);
              free_k(j + 2);
            }
          }
        }
        base += 2 * n + (it.t0 == 0 ? 1 : 0);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ---------------- softmax + epilogue: one thread per row; warpgroup t has row tile t (TQ = 2) or every other key tile (TQ = 1) ----------------
    constexpr int CPR = D / 8;
    const int t = (warp - 4) >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16, S_addr = tmem + lane_addr + Cfg::kColS + t * kTile, O_addr = tmem + lane_addr + Cfg::kColO + t * kTile;
    const float c = a.scale_log2;
    bool ok = true;
    int base = 0, count = 0, others = 0;   // the item's first entry; tiles so far of this warpgroup, and (TQ = 1) of the other one
    while (ok && cursor.next(a, it)) {
      const int n = it.t1 - it.t0, R = it.m * a.G, r0 = it.rt * a.rows + (TQ == 2 ? t * kTile : 0);
      const bool mine = r0 < R;    // this warpgroup has rows
      const SeqPages pg = seq_pages(a.p, it.n);
      uint4 own = make_uint4(0, 0, 0, 0);
      if (it.t0 == 0 && mine) own = a.family[it.tok0 + min((r0 + row) / a.G, it.m - 1)];
      float m = -INFINITY, l = 0.f;
      const int first = TQ == 2 ? 0 : t, step = TQ == 2 ? 1 : 2;
      for (int j = first; j < n && mine && ok; j += step) {
        const int tile = tile_of(it, j);
        const Entry v(base + 2 * j + (tile == 0 ? 2 : 1));
        ok = mbar_wait_warp(smem_u32(&sh.s_full[t]), count & 1, abort);
        if (!ok) break;
        tc_fence_after_sync();
        // the slots that this row sees; the same for all rows but among the new tokens
        bool whole = false;
        uint32_t see[4] = {own.x, own.y, own.z, own.w};
        bool used = row < it.m;      // V row `row` of the tile belongs to somebody
        if (tile > 0) {
          const int f0 = (tile - 1) * per, front = (pg.sinks + (1 << shift) - 1) >> shift, recent = front + pg.w * a.p.kp;
          whole = (f0 >= front && f0 + per <= recent && a.p.kp << shift == a.p.K) || (f0 >= recent && (f0 + per - recent) << shift <= pg.ra);
          if (!whole) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int key = 32 * q + lane;
              int rows;
              page_column(a.p, pg, f0 + (key >> shift), rows);
              see[q] = __ballot_sync(0xffffffffu, (key & ((1 << shift) - 1)) < rows);
            }
            used = ((quad == 0 ? see[0] : quad == 1 ? see[1] : quad == 2 ? see[2] : see[3]) >> lane & 1u) != 0;
          }
        }
        if (!whole) {
          // rows of V that belong to nobody: zero (the products with them start behind this thread's arrival below)
          ok = mbar_wait_warp(smem_u32(&sh.kv_full[v.slot]), v.phase, abort);
          if (!ok) break;
          if (!used) {
            unsigned char* dst = smem_raw + Cfg::kRing + v.slot * Cfg::kTileBytes + row * 128;
#pragma unroll
            for (int x = 0; x < CPR; ++x) *reinterpret_cast<uint4*>(dst + (x >> 3) * Cfg::kSubBytes + ((x & 7) << 4)) = make_uint4(0, 0, 0, 0);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
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
        for (int i = 0; i < 4; ++i) mx4[i] = __uint_as_float(s[i]);
#pragma unroll
        for (int i = 4; i + 8 <= kTile; i += 8)
#pragma unroll
          for (int x = 0; x < 4; ++x) mx4[x] = fmaxf(fmaxf(mx4[x], __uint_as_float(s[i + x])), __uint_as_float(s[i + 4 + x]));
#pragma unroll
        for (int i = 0; i < 4; ++i) mx4[i] = fmaxf(mx4[i], __uint_as_float(s[kTile - 4 + i]));
        const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
        // the maximum is only raised when it grew by more than 2^8 (then O is rescaled in tensor memory); -inf while no score has counted
        const bool need = mx > m && (mx - m) * c > 8.f;
        if (j == first) {
          m = mx;
        } else if (__any_sync(0xffffffffu, need)) {
          ok = mbar_wait_warp(smem_u32(&sh.pv_done[t]), (count - 1) & 1, abort);   // O holds every earlier tile
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
        // (s - m) c, not s c - m c in one step: there the rounding of m c is left over, and where scores are beyond 2^31 it is an exponent that overflows
        const float nm = m == -INFINITY ? 0.f : -m;
        const uint64_t c2 = f2_pack(c, c), nm2 = f2_pack(nm, nm);
        uint64_t sum2 = f2_pack(0.f, 0.f), sum2b = f2_pack(0.f, 0.f);
        // exponentials as a software pipeline, P over S in two halves, as in the forward
        constexpr int kPairs = kTile / 4, kLag = 4;
        uint32_t pk[kPairs];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
          for (int ii = 0; ii < kPairs + kLag; ++ii) {
            if (ii < kPairs) {
              const int i = half * kPairs + ii;
              float x0, x1;
              f2_unpack(f2_mul(f2_add(f2_pack(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), nm2), c2), x0, x1);
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
          if (lane == 0) mbar_arrive(smem_u32(&sh.p_full[t][half]));
        }
        sum2 = f2_add(sum2, sum2b);
        float sum0, sum1;
        f2_unpack(sum2, sum0, sum1);
        l += sum0 + sum1;
        ++count;
      }
      base += 2 * n + (it.t0 == 0 ? 1 : 0);
      // the products are done: of TQ = 1 both warpgroups', whose maxima and sums meet in shared memory
      if (ok && mine && n > first) ok = mbar_wait_warp(smem_u32(&sh.pv_done[t]), (count - 1) & 1, abort);
      float f0 = 1.f, f1 = 0.f;   // TQ = 1: what brings O of the two to one maximum
      if constexpr (TQ == 1) {
        const int theirs = t == 0 ? n / 2 : (n + 1) / 2;   // the other warpgroup's tiles of the item
        others += theirs;
        if (ok && theirs > 0) ok = mbar_wait_warp(smem_u32(&sh.pv_done[t ^ 1]), (others - 1) & 1, abort);
        sh.ml[t][row] = make_float2(m, l);
        ok = meet_and_vote<256>(ok);
        if (!ok) break;            // (all of them leave together: a warp that left alone would be waited for at the barrier)
        const float2 x = sh.ml[0][row], y = sh.ml[1][row];
        const float mx = x.y != 0.f ? (y.y != 0.f ? fmaxf(x.x, y.x) : x.x) : y.x;
        f0 = weight_of(x.y, (x.x - mx) * c);
        f1 = weight_of(y.y, (y.x - mx) * c);
        m = mx;
        l = fmaf(x.y, f0, y.y * f1);
      }
      if (ok && mine) {
        tc_fence_after_sync();
        const int rr = r0 + row;
        const bool add_odd = it.t0 == 0 && a.odd[(size_t)it.s * a.p.Hkv + it.h];
        float* part = it.part >= 0 ? part_at(a, it.part, D) : nullptr;
        const float inv = 1.0f / l;
        const int tok = rr / a.G, head = it.h * a.G + rr - tok * a.G, part_row = TQ == 2 ? t * kTile + row : row;
        uint4* dst = rr < R ? reinterpret_cast<uint4*>(a.o + head * a.o_head + (it.tok0 + tok) * a.o_tok) : nullptr;
        // columns of this warpgroup: all of its row tile's, or half of the common one's
        constexpr int W = TQ == 2 ? 32 : 16, kParts = (TQ == 2 ? D : D / 2) / W;
#pragma unroll
        for (int qq = 0; qq < kParts; ++qq) {
          const int q = TQ == 2 ? qq : t * kParts + qq;
          uint32_t o[W];
          if constexpr (TQ == 2) {
            tmem_ld32(O_addr + q * W, o);
            tmem_wait_ld();
          } else {
            uint32_t o1[W];
            tmem_ld16(tmem + lane_addr + Cfg::kColO + q * W, o);
            if (n > 1) tmem_ld16(tmem + lane_addr + Cfg::kColO + kTile + q * W, o1);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < W; ++i) {
              const float z = f0 != 0.f ? __uint_as_float(o[i]) * f0 : 0.f;
              o[i] = __float_as_uint(n > 1 && f1 != 0.f ? fmaf(__uint_as_float(o1[i]), f1, z) : z);
            }
          }
          if (add_odd) {
#pragma unroll 1
            for (int i = 0; i < W; ++i) {
              const float add = odd_values(a, it, own, W * q + i);
#pragma unroll
              for (int x = 0; x < W; ++x)
                if (x == i) o[x] = __float_as_uint(__uint_as_float(o[x]) + add);
            }
          }
          if (part) {
#pragma unroll
            for (int x = 0; x < W / 4; ++x)
              reinterpret_cast<uint4*>(part)[(W / 4 * q + x) * a.rows + part_row] = make_uint4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
          } else if (dst) {
            // (a thread writes its own row: staged in shared memory the rows would leave in whole lines, but the only place for them is Q's, where the
            // next item's is on its way by now)
#pragma unroll
            for (int x = 0; x < W / 8; ++x) {
              float f[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(o[8 * x + i]) * inv;
              dst[q * (W / 8) + x] = pack_channels(f);
            }
          }
        }
        if (TQ == 2 || t == 0) {
          if (part) {
            part[a.rows * D + part_row] = m * c;
            part[a.rows * (D + 1) + part_row] = l;
          } else if (dst && a.lse) {
            a.lse[(size_t)head * a.p.n_new + it.tok0 + tok] = m * a.scale + logf(l);
          }
        }
        tc_fence_before_sync();   // O and S have been read: the next item's products may write them
      }
      if constexpr (TQ == 1) meet<256>();   // ... when both warpgroups have
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, Cfg::kCols);
  if (tid == 0 && sh.abort) {
    atomicExch(&a.head->status, (int)LRSA_ERR_TIMEOUT);
    keep_status(a.head, LRSA_ERR_TIMEOUT);
  }
}

bool rows_ok(const lrsa_rows_t* r) {
  return r && r->data && !(reinterpret_cast<uintptr_t>(r->data) & 15u) && r->head_stride % 8 == 0 && r->token_stride % 8 == 0;
}

// Whether |c + y step| < d for a y in [lo, hi].
bool comes_near(long long c, long long step, long long lo, long long hi, long long d) {
  auto near = [=](long long y) { const long long x = c + (y < lo ? lo : y > hi ? hi : y) * step; return x < d && -x < d; };
  if (step == 0) return near(lo);
  const long long y = -c / step;   // (towards zero: the nearest is this one or a neighbour)
  return near(y - 1) || near(y) || near(y + 1);
}
// Whether two of the rows of o lie over one another: heads h, tokens t at h o_head + t o_tok, d elements each.
bool rows_overlap(const AttendArgs& a, long long heads, long long n, long long d) {
  const long long head = a.o_head < 0 ? -a.o_head : a.o_head, tok = a.o_tok < 0 ? -a.o_tok : a.o_tok;
  if (n > 1 && tok < d) return true;
  if (heads == 1 || (n > 1 ? (tok >= (heads - 1) * head + d && head >= d) || head >= (n - 1) * tok + d : head >= d)) return false;   // one inside the other
  for (long long h = 1; h < heads; ++h)
    if (comes_near(h * a.o_head, a.o_tok, 1 - n, n - 1, d)) return true;
  return false;
}
// Whether a row of o lies over one of the rows at p.  Rows of both may take turns in one buffer (the output beside a fused projection's).
bool rows_overlap(const AttendArgs& a, long long heads, long long n, long long d, const __nv_bfloat16* p, long long p_heads, long long p_head, long long p_tok) {
  const long long apart = (reinterpret_cast<intptr_t>(a.o) - reinterpret_cast<intptr_t>(p)) / (long long)sizeof(__nv_bfloat16);
  auto low = [n](long long h, long long head, long long tok) { return (head < 0 ? (h - 1) * head : 0) + (tok < 0 ? (n - 1) * tok : 0); };
  auto high = [n](long long h, long long head, long long tok) { return (head > 0 ? (h - 1) * head : 0) + (tok > 0 ? (n - 1) * tok : 0); };
  if (apart + high(heads, a.o_head, a.o_tok) + d <= low(p_heads, p_head, p_tok) || apart + low(heads, a.o_head, a.o_tok) >= high(p_heads, p_head, p_tok) + d)
    return false;   // (all that is looked at where every tensor has memory of its own)
  if (a.o_tok == p_tok && p_tok > 0 && a.o_head >= 0 && p_head >= 0) {   // side by side within the pitch of a token
    const long long column = (apart % p_tok + p_tok) % p_tok;
    if (column >= (p_heads - 1) * p_head + d && column + (heads - 1) * a.o_head + d <= p_tok) return false;
  }
  for (long long h = 0; h < heads; ++h)
    for (long long g = 0; g < p_heads; ++g) {
      const long long c = apart + h * a.o_head - g * p_head;
      if (a.o_tok == p_tok) {
        if (comes_near(c, a.o_tok, 1 - n, n - 1, d)) return true;
      } else {
        for (long long t = 0; t < n; ++t)
          if (comes_near(c + t * a.o_tok, -p_tok, 0, n - 1, d)) return true;
      }
    }
  return false;
}

// Fewest key tiles that are a CTA's worth.
constexpr int kMinTilesFew = 2, kMinTiles = 2;
// What it costs a CTA to begin another item, in key tiles.
constexpr int kExtraFew = 2, kExtra = 3;

// The parts of the workspace.  few: of a call that the kernel for few rows takes.
struct AttendWs { size_t starts, divided, part, family, odd, q[2], k[2], v, total; };
AttendWs attend_ws(const Geom& g, long long n_seqs, long long n_new, bool few) {
  AttendWs w;
  size_t off = sizeof(WsHeader);
  auto take = [&off](size_t bytes) { const size_t at = off; off += align_up(bytes, 256); return at; };
  w.starts = take(kMaxPlaces * sizeof(Start));
  w.divided = take(kMaxPlaces * sizeof(Divided));
  w.part = take((few ? (size_t)2 * kMaxPlaces * kFewRows : (size_t)2 * kSms * 2 * kTile) * (g.d + 2) * sizeof(float));
  if (few) n_seqs = n_new = 0;
  w.family = take(n_new * sizeof(uint4));
  w.odd = take(n_seqs * g.Hkv * sizeof(int));
  for (size_t& q : w.q) q = take((size_t)n_new * g.Hq * g.d * 2);
  for (size_t& k : w.k) k = take((size_t)n_new * g.Hkv * g.d * 2);
  w.v = take((size_t)n_new * g.Hkv * g.d * 2);
  w.total = off;
  return w;
}

template <int D, int TQ>
int launch_tile(AttendArgs& a, cudaStream_t st) {
  using Cfg = TileCfg<D, TQ>;
  a.rows = TQ * kTile; a.places = kSms; a.min_tiles = kMinTiles; a.extra = kExtra;
  TileMaps maps;
  const long long outer = (long long)a.p.n_pages * a.p.Hkv, Hkv = a.p.Hkv, T = a.p.n_new > 0 ? a.p.n_new : 1;
  int rc = make_tmap_bf16(&maps.k, a.k_pages, D, 1 << a.p.shift, outer, 1 << a.p.shift);
  if (rc == LRSA_OK) rc = make_tmap_bf16(&maps.v, a.v_pages, D, 1 << a.p.shift, outer, 1 << a.p.shift);
  for (int i = 0; i < 2; ++i) {
    if (rc == LRSA_OK) rc = make_tmap_bf16(&maps.q[i], a.q_parts[i], D, T * a.G, Hkv, kTile);
    if (rc == LRSA_OK) rc = make_tmap_bf16(&maps.kn[i], a.k_parts[i], D, T, Hkv, kTile);
  }
  if (rc == LRSA_OK) rc = make_tmap_bf16(&maps.vn, a.v_finite, D, T, Hkv, kTile);
  if (rc != LRSA_OK) return rc;
  const long long grid = (long long)a.p.n_seqs * Hkv * (a.G + 2) + (a.places + 7) / 8;
  if (grid > 0x7fffffffLL) return LRSA_ERR_UNSUPPORTED;
  LRSA_CUDA_CHECK(launch_dependent(paged_operands_kernel<D>, dim3((unsigned)grid), dim3(256), 0, st, 1, a));
  launch_counter().n++;
  constexpr size_t smem = Cfg::kTail + sizeof(TileTail);
  static_assert(smem <= 227 * 1024, "shared memory of a CTA");
  LRSA_CUDA_CHECK((allow_smem<(int)smem>(paged_tile_kernel<D, TQ>)));
  LRSA_CUDA_CHECK(launch_dependent(paged_tile_kernel<D, TQ>, dim3(a.places), dim3(Cfg::kThreads), smem, st, 1, maps, a));
  return LRSA_OK;
}

template <int D, int NH>
int launch_few(AttendArgs& a, cudaStream_t st) {
  a.rows = kFewRows; a.places = NH == 1 ? 2 * kSms : kSms; a.min_tiles = kMinTilesFew; a.extra = kExtraFew;
  LRSA_CUDA_CHECK(launch_dependent(paged_few_kernel<D, NH>, dim3(a.places), dim3(256), 0, st, 1, a));
  return LRSA_OK;
}

template <int D>
int launch_attend(AttendArgs a, long long max_rows, cudaStream_t st) {
  const int rc = max_rows <= 8          ? launch_few<D, 1>(a, st)
                 : max_rows <= kFewRows ? launch_few<D, 2>(a, st)
                 : max_rows <= kTile    ? launch_tile<D, 1>(a, st)
                                        : launch_tile<D, 2>(a, st);
  if (rc != LRSA_OK) return rc;
  launch_counter().n++;
  LRSA_CUDA_CHECK(launch_dependent(paged_merge_kernel<D>, dim3(4 * kSms), dim3(256), 0, st, 1, a));
  launch_counter().n++;
  return LRSA_OK;
}

}  // namespace
}  // namespace lrsa

using namespace lrsa;

extern "C" {

int lrsa_paged_shape(const lrsa_params_t* params, int32_t page, int32_t n_seqs, int32_t n_new, int32_t max_new, int32_t* table_width, int32_t* w_cap,
                     size_t* workspace_bytes) {
  lrsa_paged_t paged = {};
  paged.page = page;
  if (n_seqs < 0 || n_new < 0 || max_new < 0) return LRSA_ERR_INVALID_ARG;
  Geom g;
  PageGeom p;
  const int rc = make_pages(params, &paged, &g, &p);
  if (rc != LRSA_OK) return rc;
  if (table_width) *table_width = p.width;
  if (w_cap) *w_cap = p.w_cap;
  if (workspace_bytes) *workspace_bytes = max_new > 0 ? attend_ws(g, n_seqs, n_new, (long long)max_new * g.G <= kFewRows).total : append_ws_bytes(g, n_seqs, n_new);
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
  const long long max_rows = (long long)max_new * g.G;
  const AttendWs ws = attend_ws(g, paged->n_seqs, n_new, max_rows <= kFewRows);
  if (workspace_bytes < ws.total) return LRSA_ERR_WORKSPACE_TOO_SMALL;
  a.p.cu = cu_new; a.p.n_new = n_new;
  a.k_pages = static_cast<const __nv_bfloat16*>(paged->k_pages); a.v_pages = static_cast<const __nv_bfloat16*>(paged->v_pages);
  if (n_new > 0) {
    auto rows = [](const lrsa_rows_t* r) { return static_cast<__nv_bfloat16*>(r->data); };
    a.q = rows(q); a.k = rows(k); a.v = rows(v); a.o = rows(o);
    a.q_head = q->head_stride; a.q_tok = q->token_stride; a.k_head = k->head_stride; a.k_tok = k->token_stride;
    a.v_head = v->head_stride; a.v_tok = v->token_stride; a.o_head = o->head_stride; a.o_tok = o->token_stride;
    if (rows_overlap(a, g.Hq, n_new, g.d) || rows_overlap(a, g.Hq, n_new, g.d, a.q, g.Hq, a.q_head, a.q_tok) ||
        rows_overlap(a, g.Hq, n_new, g.d, a.k, g.Hkv, a.k_head, a.k_tok) || rows_overlap(a, g.Hq, n_new, g.d, a.v, g.Hkv, a.v_head, a.v_tok))
      return LRSA_ERR_INVALID_ARG;
  }
  a.parent = parent; a.lse = lse;
  a.head = static_cast<WsHeader*>(workspace);
  auto at = [workspace](size_t offset) { return static_cast<void*>(static_cast<unsigned char*>(workspace) + offset); };
  a.starts = static_cast<Start*>(at(ws.starts));
  a.divided = static_cast<Divided*>(at(ws.divided));
  a.part = static_cast<float*>(at(ws.part));
  a.family = static_cast<uint4*>(at(ws.family));
  a.odd = static_cast<int*>(at(ws.odd));
  for (int i = 0; i < 2; ++i) {
    a.q_parts[i] = static_cast<__nv_bfloat16*>(at(ws.q[i]));
    a.k_parts[i] = static_cast<__nv_bfloat16*>(at(ws.k[i]));
  }
  a.v_finite = static_cast<__nv_bfloat16*>(at(ws.v));
  a.G = g.G; a.max_new = max_new;
  a.limit = a.rope.half > 0 ? a.rope.n_pos : 0x7fffffff;
  a.scale = g.scale; a.scale_log2 = g.scale * 1.4426950408889634f;
  auto st = static_cast<cudaStream_t>(cuda_stream);
  return g.d == 128 ? launch_attend<128>(a, max_rows, st) : launch_attend<64>(a, max_rows, st);
}

}  // extern "C"
