// What the kernels of the paged cache and the rotation share: the rotation of a row, where the rows of a sequence lie in its
// pages, and which counts and tables on the device are usable.
#pragma once

#include "lrsa_internal.h"
#include "sm100_ptx.h"

namespace lrsa {

// May be launched before the kernel in front of it has ended.
__device__ __forceinline__ void wait_front() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// What a call found is told by the status word, which the next call on the workspace clears, and by a word that is kept until it is read.
__device__ __forceinline__ void keep_status(WsHeader* head, lrsa_status code) {
  atomicOr(&head->raised, code == LRSA_ERR_TIMEOUT ? kRaisedTimeout : kRaisedInvalid);
}

// ---- rotation ----
struct RopeArgs {
  const float *cos, *sin;   // [n_pos][half]
  int n_pos, half;          // half: rotated pairs of a row (a multiple of 8); 0: no rotation
  int interleaved;          // pairs are neighbours (2i, 2i + 1) instead of (i, i + half)
};
// Checks and takes the caller's description (NULL: no rotation).  An lrsa_status.
int make_rope(const lrsa_rope_t* rope, int d, RopeArgs* out);

__device__ __forceinline__ float bf16_lo(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }

// x c + y s' for the pair (x, y), s' = -sin for the first of a pair: one product rounded, one fused.  Written out, so that a row
// is rotated to the same bits by every kernel (what a draft attends with is what the cache holds when it is accepted).
__device__ __forceinline__ float turn(float x, float y, float c, float s) { return fmaf(x, c, __fmul_rn(y, s)); }

// Eight rotated channels in 32 bits: chunk c (channels 8c .. 8c + 7) of the row at `row`, for position pos; false: the chunk is not among the rotated
// ones and y holds it as it is.  All loads are 16 bytes; the partner's chunk is another lane's too and comes from L1.
__device__ __forceinline__ bool turned_channels(const __nv_bfloat16* row, int c, int pos, const RopeArgs& r, float (&y)[8]) {
  const uint4 x = *reinterpret_cast<const uint4*>(row + 8 * c);
  const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) { y[2 * e] = bf16_lo(xs[e]); y[2 * e + 1] = bf16_hi(xs[e]); }
  if (8 * c >= 2 * r.half) return false;
  const float* cs = r.cos + (size_t)pos * r.half;
  const float* sn = r.sin + (size_t)pos * r.half;
  if (r.interleaved) {
    const float4 c4 = *reinterpret_cast<const float4*>(cs + 4 * c), s4 = *reinterpret_cast<const float4*>(sn + 4 * c);
    const float cc[4] = {c4.x, c4.y, c4.z, c4.w}, ss[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float a = y[2 * e], b = y[2 * e + 1];
      y[2 * e] = turn(a, b, cc[e], -ss[e]);
      y[2 * e + 1] = turn(b, a, cc[e], ss[e]);
    }
  } else {
    const int m = r.half >> 3;
    const bool first = c < m;
    const int i = first ? c : c - m;
    const uint4 v = *reinterpret_cast<const uint4*>(row + 8 * (first ? c + m : c - m));
    const uint32_t vs[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 c4 = *reinterpret_cast<const float4*>(cs + 8 * i + 4 * h), s4 = *reinterpret_cast<const float4*>(sn + 8 * i + 4 * h);
      const float cc[4] = {c4.x, c4.y, c4.z, c4.w}, ss[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int k = 4 * h + e;
        y[k] = turn(y[k], e & 1 ? bf16_hi(vs[k >> 1]) : bf16_lo(vs[k >> 1]), cc[e], first ? -ss[e] : ss[e]);
      }
    }
  }
  return true;
}
__device__ __forceinline__ uint4 pack_channels(const float (&y)[8]) {
  return make_uint4(ptx::pack_bf16(y[0], y[1]), ptx::pack_bf16(y[2], y[3]), ptx::pack_bf16(y[4], y[5]), ptx::pack_bf16(y[6], y[7]));
}
// The chunk rotated and rounded to bf16: what the cache holds.
__device__ __forceinline__ uint4 rotated_chunk(const __nv_bfloat16* row, int c, int pos, const RopeArgs& r) {
  float y[8];
  turned_channels(row, c, pos, r, y);
  return pack_channels(y);
}
// What the rounding to hi left of y, rounded to bf16.
__device__ __forceinline__ uint4 rest_of(const float (&y)[8], const uint4& hi) {
  const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w};
  float z[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float a = y[2 * e] - bf16_lo(h[e]), b = y[2 * e + 1] - bf16_hi(h[e]);
    z[2 * e] = fabsf(a) < INFINITY ? a : 0.f;           // (an infinity or NaN is all in the first)
    z[2 * e + 1] = fabsf(b) < INFINITY ? b : 0.f;
  }
  return pack_channels(z);
}
// The chunk rotated, as the sum of two bf16: rounded, and what that leaves (2^-17 of a channel is lost).  For operands of products.
__device__ __forceinline__ uint4 rotated_chunk(const __nv_bfloat16* row, int c, int pos, const RopeArgs& r, uint4& rest) {
  float y[8];
  turned_channels(row, c, pos, r, y);
  const uint4 hi = pack_channels(y);
  rest = rest_of(y, hi);
  return hi;
}

// The same for two chunks at a time, which is what a row's D / 16 units are: partners of one another, or neighbours.  Loads and arithmetic
// apart, so that a thread may ask for several units before it works on one.
struct RotUnit {
  uint4 x, y;          // chunks c0 and c1
  float4 cs[2], sn[2];
  int c0, c1, kind;    // 0: not rotated, 1: partners, 2: pairs of neighbours
};
__device__ __forceinline__ void place_unit(RotUnit& u, int unit, const RopeArgs& r) {
  const int m = r.half >> 3;
  u.kind = unit >= m ? 0 : r.interleaved ? 2 : 1;
  u.c0 = u.kind == 1 ? unit : 2 * unit;
  u.c1 = u.kind == 1 ? unit + m : u.c0 + 1;
}
__device__ __forceinline__ void load_angles(RotUnit& u, int unit, int pos, const RopeArgs& r) {
  if (u.kind == 0) return;
  const float4* cs = reinterpret_cast<const float4*>(r.cos + (size_t)pos * r.half + 8 * unit);
  const float4* sn = reinterpret_cast<const float4*>(r.sin + (size_t)pos * r.half + 8 * unit);
  u.cs[0] = cs[0]; u.cs[1] = cs[1]; u.sn[0] = sn[0]; u.sn[1] = sn[1];
}
__device__ __forceinline__ void load_unit(RotUnit& u, const __nv_bfloat16* row, int unit, int pos, const RopeArgs& r) {
  place_unit(u, unit, r);
  u.x = *reinterpret_cast<const uint4*>(row + 8 * u.c0);
  u.y = *reinterpret_cast<const uint4*>(row + 8 * u.c1);
  load_angles(u, unit, pos, r);
}
// hi: the chunks rounded to bf16; lo: what that leaves, rounded to bf16
__device__ __forceinline__ void turn_unit(const RotUnit& u, uint4 (&hi)[2], uint4 (&lo)[2]) {
  hi[0] = u.x; hi[1] = u.y;
  lo[0] = lo[1] = make_uint4(0, 0, 0, 0);
  if (u.kind == 0) return;
  const uint32_t xs[4] = {u.x.x, u.x.y, u.x.z, u.x.w}, ys[4] = {u.y.x, u.y.y, u.y.z, u.y.w};
  const float c[8] = {u.cs[0].x, u.cs[0].y, u.cs[0].z, u.cs[0].w, u.cs[1].x, u.cs[1].y, u.cs[1].z, u.cs[1].w};
  const float s[8] = {u.sn[0].x, u.sn[0].y, u.sn[0].z, u.sn[0].w, u.sn[1].x, u.sn[1].y, u.sn[1].z, u.sn[1].w};
  float a[8], b[8];
  if (u.kind == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = e & 1 ? bf16_hi(xs[e >> 1]) : bf16_lo(xs[e >> 1]), q = e & 1 ? bf16_hi(ys[e >> 1]) : bf16_lo(ys[e >> 1]);
      a[e] = turn(p, q, c[e], -s[e]);
      b[e] = turn(q, p, c[e], s[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[2 * e] = turn(bf16_lo(xs[e]), bf16_hi(xs[e]), c[e], -s[e]);
      a[2 * e + 1] = turn(bf16_hi(xs[e]), bf16_lo(xs[e]), c[e], s[e]);
      b[2 * e] = turn(bf16_lo(ys[e]), bf16_hi(ys[e]), c[4 + e], -s[4 + e]);
      b[2 * e + 1] = turn(bf16_hi(ys[e]), bf16_lo(ys[e]), c[4 + e], s[4 + e]);
    }
  }
  hi[0] = pack_channels(a); hi[1] = pack_channels(b);
  lo[0] = rest_of(a, hi[0]); lo[1] = rest_of(b, hi[1]);
}

// ---- pages ----
// A sequence of the cache is a row of the page table:
//   [0, sp)                      pages of the sinks
//   [sp, sp + 2 lp)              two groups of lp pages: the uncompressed window w lies in group w mod 2
//   [sp + 2 lp + w kp, ... kp)   the kept rows of window w
// A cache of n tokens is condensed for the token at position n, the next one: of the windows in front of that token's chunk c all but
// the last are cut to their kept rows (the mask of Section 3.2).  So cut(n) = max((n - S) / L - 1, 0) windows are, and at most 2 L tokens are whole.
struct PageGeom {
  int S, L, K, N;                // N: most tokens of a sequence
  int shift, sp, lp, kp, width;  // page = 1 << shift rows
  int n_pages, n_seqs, Hkv, w_cap;
  const int32_t* table;          // [n_seqs][width]
  const int32_t* n_tokens;       // [n_seqs]
  const int32_t* cu;             // [n_seqs + 1]: where the new tokens of a sequence begin
  int n_new;                     // new tokens that there is room for (cu[n_seqs] may be less)
};
// paged_append.cu : the workspace of an append.
size_t append_ws_bytes(const Geom& g, long long n_seqs, long long n_new);
// Checks the caller's description and fills everything but cu and n_new.  An lrsa_status.
int make_pages(const lrsa_params_t* params, const lrsa_paged_t* paged, Geom* g, PageGeom* out);

__device__ __forceinline__ int cut_windows(const PageGeom& a, int n) { return n >= a.S ? max((n - a.S) / a.L - 1, 0) : 0; }

// The tokens of sequence s in the cache (n) and the new ones [tok0, tok0 + m); m = 0 where the counts on the device are not usable.
// most: new tokens that a sequence may have; limit: tokens it may have together; behind: the largest of the boundaries in front of
// its own (where they go back, the ranges of two sequences could overlap: the later one is left out).
struct SeqCounts { int n, tok0, m; bool ok; };
__device__ __forceinline__ SeqCounts seq_counts(const PageGeom& a, int s, int most, int limit, int behind = 0) {
  SeqCounts q;
  q.n = a.n_tokens[s];
  q.tok0 = a.cu[s];
  const int end = a.cu[s + 1];
  q.ok = q.n >= 0 && q.n <= a.N && q.tok0 >= max(behind, 0) && end >= q.tok0 && end <= a.n_new;
  q.m = q.ok ? end - q.tok0 : 0;
  if (q.m > most || q.m > limit - q.n) { q.ok = false; q.m = 0; }
  if (!q.ok) q.n = q.tok0 = 0;
  return q;
}
// True where a boundary in front of sequence s lies behind its own; by a whole warp.  first: first_boundary, asked for with the counts
// (volatile: the compiler would ask for it where it is used, a round trip later).
__device__ __forceinline__ int first_boundary(const PageGeom& a, int s) {
  int x;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(x) : "l"(a.cu + min((int)threadIdx.x & 31, s)));
  return x;
}
__device__ __forceinline__ bool begins_early(const PageGeom& a, int s, int first) {
  const int begin = a.cu[s];
  bool early = first > begin;
  for (int i0 = 32 + (threadIdx.x & 31); i0 < s; i0 += 256) {
#pragma unroll
    for (int i = i0; i < i0 + 256; i += 32) early |= i < s && a.cu[i] > begin;   // (eight loads on their way)
  }
  return __any_sync(0xffffffffu, early);
}
// The largest boundary in front of every lane's sequence s0 + lane, by a whole warp; `behind`: in front of s0, moved on by 32.
__device__ __forceinline__ int largest_in_front(const PageGeom& a, int s0, int lane, int& behind) {
  int top = s0 + lane < a.n_seqs ? a.cu[s0 + lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) top = max(top, __shfl_up_sync(0xffffffffu, top, o));   // (the lanes below o get their own)
  const int front = __shfl_up_sync(0xffffffffu, top, 1), mine = lane > 0 ? max(behind, front) : behind;
  behind = max(behind, __shfl_sync(0xffffffffu, top, 31));
  return mine;
}

// Column of the table and row of that page of the uncompressed token at position p.
__device__ __forceinline__ int token_column(const PageGeom& a, int p, int& row) {
  int i = p, col = 0;
  if (p >= a.S) {
    const int w = (p - a.S) / a.L;
    i = p - a.S - w * a.L;
    col = a.sp + (w & 1) * a.lp;
  }
  row = i & ((1 << a.shift) - 1);
  return col + (i >> a.shift);
}

}  // namespace lrsa
