// Position rotation of Q and K, and its gradient (the same by the opposite angles).
//
// Pairs (a, b) of a row's channels become (a cos - b sin, b cos + a sin), with the angle of the token's position and of the pair.  Bound
// by memory: every row is read and written once.  The angles of a token are the same for all its heads: a thread takes 16 channels of
// a token (two chunks that make pairs), loads their eight cosines and sines once and walks over heads, four at a time, so
// that the tables cost 1 / heads of what the rows do.
#include <math.h>

#include "paged_sm100.h"

namespace lrsa {

int make_rope(const lrsa_rope_t* rope, int d, RopeArgs* out) {
  *out = RopeArgs{};
  if (!rope) return LRSA_OK;
  if (!rope->cos || !rope->sin || rope->n_pos < 1 || rope->dim < 16 || rope->dim > d || rope->dim % 16 != 0 ||
      (rope->interleaved != 0 && rope->interleaved != 1) || rope->reserved != 0)
    return LRSA_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(rope->cos) | reinterpret_cast<uintptr_t>(rope->sin)) & 15u) return LRSA_ERR_INVALID_ARG;
  out->cos = rope->cos; out->sin = rope->sin; out->n_pos = rope->n_pos; out->half = rope->dim / 2; out->interleaved = rope->interleaved;
  return LRSA_OK;
}

namespace {

constexpr int kCuts = 512;        // sequences of a packed row that one launch knows
constexpr int kRotThreads = 256;

struct RotateArgs {
  const __nv_bfloat16 *x[2];      // Q, K: [slices][N][d]
  __nv_bfloat16* y[2];
  long long slices[2];            // batch * heads
  RopeArgs rope;
  const int32_t* positions;
  int N, tok0, tok1;              // tokens of this launch
  int tok_blocks, per_thread;     // blocks along the tokens; slices a thread walks over
  int inverse, n_seqs;
  int cut[kCuts + 1];             // first tokens of the sequences of this launch (cut[0] <= tok0)
};

template <int D>
__global__ void __launch_bounds__(kRotThreads) rotate_kernel(const __grid_constant__ RotateArgs a) {
  constexpr int UNITS = D / 16, TOK = kRotThreads / UNITS;
  const int unit = threadIdx.x % UNITS, tok = a.tok0 + (blockIdx.x % a.tok_blocks) * TOK + threadIdx.x / UNITS;
  const long long s0 = (long long)(blockIdx.x / a.tok_blocks) * a.per_thread;
  wait_front();
  if (tok >= a.tok1) return;
  const int half = a.rope.half, m = half >> 3;
  // the two chunks of this thread: a pair's partners, or neighbours where the pairs are, or behind the rotated channels
  const bool split = !a.rope.interleaved && unit < m;
  const int c0 = a.rope.interleaved || unit >= m ? 2 * unit : unit, c1 = split ? unit + m : c0 + 1;
  const bool turn0 = 8 * c0 < 2 * half, turn1 = 8 * c1 < 2 * half;
  int pos;
  if (a.positions) {
    pos = a.positions[tok];
  } else {
    int lo = 0, hi = a.n_seqs;   // the last sequence that begins at or before the token
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.cut[mid] <= tok) lo = mid; else hi = mid;
    }
    pos = tok - a.cut[lo];
  }
  const bool there = pos >= 0 && pos < a.rope.n_pos;
  float cs[8], sn[8];   // of the unit's eight pairs
  if (turn0) {
    const size_t at = (size_t)(there ? pos : 0) * half + 8 * unit;   // (interleaved: chunk 2 unit begins with pair 8 unit)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 1 && !turn1) continue;
      const float4 c4 = *reinterpret_cast<const float4*>(a.rope.cos + at + 4 * h), s4 = *reinterpret_cast<const float4*>(a.rope.sin + at + 4 * h);
      cs[4 * h] = c4.x; cs[4 * h + 1] = c4.y; cs[4 * h + 2] = c4.z; cs[4 * h + 3] = c4.w;
      sn[4 * h] = s4.x; sn[4 * h + 1] = s4.y; sn[4 * h + 2] = s4.z; sn[4 * h + 3] = s4.w;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (a.inverse) sn[e] = -sn[e];
      if (!there) cs[e] = sn[e] = NAN;
    }
  }
  const long long total = a.slices[0] + a.slices[1], s1 = min(total, s0 + a.per_thread);
  const long long row = (long long)tok * D, slice = (long long)a.N * D;
  constexpr int AHEAD = 4;
  for (long long s = s0; s < s1; s += AHEAD) {
    uint4 u[AHEAD], v[AHEAD];
    __nv_bfloat16* dst[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const long long t = min(s + i, s1 - 1);
      const int z = t >= a.slices[0];
      const long long at = (z ? t - a.slices[0] : t) * slice + row;
      dst[i] = a.y[z] + at;
      u[i] = __ldcs(reinterpret_cast<const uint4*>(a.x[z] + at) + c0);
      v[i] = __ldcs(reinterpret_cast<const uint4*>(a.x[z] + at) + c1);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (s + i >= s1) break;
      uint32_t x[4] = {u[i].x, u[i].y, u[i].z, u[i].w}, y[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      if (split) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float a0 = bf16_lo(x[e]), a1 = bf16_hi(x[e]), b0 = bf16_lo(y[e]), b1 = bf16_hi(y[e]);
          x[e] = ptx::pack_bf16(turn(a0, b0, cs[2 * e], -sn[2 * e]), turn(a1, b1, cs[2 * e + 1], -sn[2 * e + 1]));
          y[e] = ptx::pack_bf16(turn(b0, a0, cs[2 * e], sn[2 * e]), turn(b1, a1, cs[2 * e + 1], sn[2 * e + 1]));
        }
      } else if (a.rope.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (turn0) x[e] = ptx::pack_bf16(turn(bf16_lo(x[e]), bf16_hi(x[e]), cs[e], -sn[e]), turn(bf16_hi(x[e]), bf16_lo(x[e]), cs[e], sn[e]));
          if (turn1) y[e] = ptx::pack_bf16(turn(bf16_lo(y[e]), bf16_hi(y[e]), cs[4 + e], -sn[4 + e]), turn(bf16_hi(y[e]), bf16_lo(y[e]), cs[4 + e], sn[4 + e]));
        }
      }
      __stcs(reinterpret_cast<uint4*>(dst[i]) + c0, make_uint4(x[0], x[1], x[2], x[3]));
      __stcs(reinterpret_cast<uint4*>(dst[i]) + c1, make_uint4(y[0], y[1], y[2], y[3]));
    }
  }
}

}  // namespace
}  // namespace lrsa

using namespace lrsa;

extern "C" int lrsa_rotate(const lrsa_params_t* params, const void* Q, const void* K, void* Q_out, void* K_out, const lrsa_rope_t* rope,
                           const int32_t* positions, int32_t inverse, void* cuda_stream) {
  NvtxRange nvtx_range("lrsa_rotate");
  launch_counter().n = 0;
  Geom g;
  int rc = make_geom(params, &g);
  if (rc != LRSA_OK) return rc;
  if (!rope || (!Q && !K) || !Q != !Q_out || !K != !K_out || (inverse != 0 && inverse != 1)) return LRSA_ERR_INVALID_ARG;
  RotateArgs a;
  rc = make_rope(rope, g.d, &a.rope);
  if (rc != LRSA_OK) return rc;
  const uintptr_t all = reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(Q_out) |
                        reinterpret_cast<uintptr_t>(K_out);
  if ((all & 15u) || (reinterpret_cast<uintptr_t>(positions) & 3u)) return LRSA_ERR_INVALID_ARG;
  // an output is its own input, or lies over nothing else of the call
  const size_t row = (size_t)g.N * g.d * sizeof(__nv_bfloat16), size[2] = {(size_t)g.B * g.Hq * row, (size_t)g.B * g.Hkv * row};
  const void *in[2] = {Q, K}, *out[2] = {Q_out, K_out};
  auto over = [&](const void* p, int i, const void* r, int j) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(r);
    return p && r && a < b + size[j] && b < a + size[i];
  };
  for (int i = 0; i < 2; ++i)
    if ((out[i] != in[i] && over(out[i], i, in[i], i)) || over(out[i], i, in[1 - i], 1 - i)) return LRSA_ERR_INVALID_ARG;
  if (over(Q_out, 0, K_out, 1)) return LRSA_ERR_INVALID_ARG;
  const int n_seqs = positions || g.n_seqs == 0 ? 1 : g.n_seqs;
  if (!positions) {
    int longest = g.N;
    if (g.n_seqs > 0) {
      longest = 0;
      for (int s = 0; s < g.n_seqs; ++s) longest = g.cu[s + 1] - g.cu[s] > longest ? g.cu[s + 1] - g.cu[s] : longest;
    }
    if (longest > rope->n_pos) return LRSA_ERR_INVALID_ARG;
  }
  a.x[0] = static_cast<const __nv_bfloat16*>(Q); a.x[1] = static_cast<const __nv_bfloat16*>(K);
  a.y[0] = static_cast<__nv_bfloat16*>(Q_out); a.y[1] = static_cast<__nv_bfloat16*>(K_out);
  a.slices[0] = Q ? (long long)g.B * g.Hq : 0;
  a.slices[1] = K ? (long long)g.B * g.Hkv : 0;
  a.positions = positions; a.N = g.N; a.inverse = inverse;
  auto st = static_cast<cudaStream_t>(cuda_stream);
  const long long total = a.slices[0] + a.slices[1];
  const int tok = kRotThreads / (g.d / 16);
  for (int s0 = 0; s0 < n_seqs; s0 += kCuts) {
    const int s1 = s0 + kCuts < n_seqs ? s0 + kCuts : n_seqs;
    a.n_seqs = s1 - s0;
    for (int s = s0; s < s1; ++s) a.cut[s - s0] = n_seqs > 1 ? g.cu[s] : 0;
    a.tok0 = a.cut[0];
    a.tok1 = s1 < n_seqs ? g.cu[s1] : g.N;
    a.tok_blocks = (a.tok1 - a.tok0 + tok - 1) / tok;
    // Slices a thread walks over: all of them reuse its angles, but the grid should hold eight blocks for every SM.
    long long per = (total * a.tok_blocks + 8 * kSms - 1) / (8 * kSms);
    per = per < 4 ? 4 : per > 64 ? 64 : per;
    if (per > total) per = total;
    const long long grid = a.tok_blocks * ((total + per - 1) / per);
    if (grid > 0x7fffffffLL) return LRSA_ERR_UNSUPPORTED;
    a.per_thread = (int)per;
    LRSA_CUDA_CHECK(launch_dependent(g.d == 128 ? rotate_kernel<128> : rotate_kernel<64>, dim3((unsigned)grid), dim3(kRotThreads), 0, st, 1, a));
    launch_counter().n++;
  }
  return LRSA_OK;
}
